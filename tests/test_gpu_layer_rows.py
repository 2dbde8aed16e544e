"""The layer around the several-row operators: head norms, a prompt's attention, sequences
behind a shared prompt, used together."""
import math

import pytest

from tests import rows_ref as R

pytestmark = pytest.mark.gpu
D = 128
HIDDEN = 320


def _weights(torch, device, hq, hkv, seed, dtype):
    g = torch.Generator().manual_seed(seed)
    make = lambda r, c: (torch.randn(r, c, generator=g) / math.sqrt(r)).to(dtype).to(device)  # noqa: E731
    W = [make(HIDDEN, hq * D), make(HIDDEN, hkv * D), make(HIDDEN, hkv * D), make(hq * D, HIDDEN)]
    return W, R.rotations(hkv, seed + 1, device), R.rotations(hkv, seed + 2, device)


def _layer(torch, device, hq=8, hkv=2, batch=2, buffer=16, capacity=600, k=64, seed=1, norms=True,
           dtype=None, **kw):
    from paper_2511_18936_amd.layer import SwanAttentionLayer

    dtype = dtype or torch.float16
    W, P_qk, P_vo = _weights(torch, device, hq, hkv, seed, dtype)
    g = torch.Generator().manual_seed(seed + 5)
    if norms:
        kw.update(q_norm=(1 + 0.2 * torch.randn(D, generator=g)).to(dtype).to(device),
                  k_norm=(1 + 0.2 * torch.randn(D, generator=g)).to(dtype).to(device))
    return SwanAttentionLayer(*W, P_qk, P_vo, hq, hkv, 10000.0, batch, buffer, capacity, [k] * batch,
                              **kw)


def _x(torch, device, batch, n, seed, dtype=None):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(batch, n, HIDDEN, generator=g).to(dtype or torch.float16).to(device)


def _dense(torch, layer, q, k, v, L0):
    """y in float64 of rows q at L0 .. over keys k, v (rotated values) of all tokens so far."""
    B, hq, n, _ = q.shape
    G = hq // k.shape[1]
    out = torch.empty(B, n, hq * D, dtype=torch.float64, device=q.device)
    seen = torch.ones(n, L0 + n, dtype=torch.bool, device=q.device).tril(L0)
    for b in range(B):
        for h in range(hq):
            o, _ = R.softmax_rows(q[b, h], k[b, h // G], v[b, h // G], seen)
            out[b, :, h * D:(h + 1) * D] = o
    return out @ layer.W_o_hat.double()


def _err(got, want):
    """max |y - y_ref| / max |y_ref| per row of the batch"""
    d = (got.double() - want).abs().flatten(1).amax(1)
    return (d / want.abs().flatten(1).amax(1)).max().item()


# y: o is rounded to binary16 (2^-11) after p was (2^-10 at most, see rows_ref.bound), and the
# output GEMM sums 1024 such products and rounds once more
TOL = 2e-3


def test_projections_are_the_separate_steps(gpu_device, swan_mod, torch_mod):
    """Without norms the rows are what GEMM, split, swan.rope gave before, bit for bit."""
    torch = torch_mod
    layer = _layer(torch, gpu_device, norms=False)
    for n in (1, 7, 300):
        x = _x(torch, gpu_device, 2, n, n)
        q, k, v = layer.project(x)
        rows = (x @ layer.W_qkv).view(2, n, 12, D).transpose(1, 2).contiguous()
        assert torch.equal(q, swan_mod.rope(rows[:, :8].contiguous(), layer.cache.seq_len, 10000.0))
        assert torch.equal(k, swan_mod.rope(rows[:, 8:10].contiguous(), layer.cache.seq_len, 10000.0))
        assert torch.equal(v, rows[:, 10:])
        layer(x)
    assert layer.cache.seq_len == [308, 308]


@pytest.mark.parametrize("name", ["float16", "float32"])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (4, 4), (6, 3)])
def test_a_prompt_in_pieces_and_steps(gpu_device, swan_mod, torch_mod, hq, hkv, name):
    """Nothing pruned (the buffer holds all): a prompt at once, in chunks, then decode steps,
    each against dense attention over all rows so far."""
    torch = torch_mod
    dtype = getattr(torch, name)
    tol = TOL if name == "float16" else 1e-5
    chunks = [50, 1, 64, 3, 1, 1]
    layer = _layer(torch, gpu_device, hq, hkv, buffer=256, dtype=dtype)
    whole = _layer(torch, gpu_device, hq, hkv, buffer=256, dtype=dtype)
    x = _x(torch, gpu_device, 2, sum(chunks), 3, dtype)
    q, k, v = whole.project(x)
    at_once = whole(x, attend=True)
    want = _dense(torch, whole, q, k, v, 0)
    assert at_once.shape == (2, sum(chunks), HIDDEN) and _err(at_once, want) < tol
    L = 0
    for n in chunks:
        y = layer(x[:, L:L + n].contiguous(), attend=True)
        y = y[:, None] if n == 1 else y
        # cached rows are rounded once more than the prompt's own: the rotated keys and values
        assert _err(y, want[:, L:L + n]) < 2 * tol, (L, n)
        L += n
    assert layer.cache.seq_len == whole.cache.seq_len == [L, L]
    plain = _layer(torch, gpu_device, hq, hkv, buffer=256, dtype=dtype)
    assert plain(x) is None  # a prompt whose attention is not asked for
    for name in ("k_ring", "v_ring"):
        assert torch.equal(getattr(plain.cache, name), getattr(whole.cache, name))


@pytest.mark.parametrize("values", ["same", "e4m3"])
@pytest.mark.parametrize("k", [128, 40])
def test_sequences_behind_a_shared_prompt(gpu_device, swan_mod, torch_mod, k, values):
    """Two prompts, five sequences behind them, questions, then decode steps: against
    attention over the rows that the caches hold, at the positions after the prompt."""
    torch = torch_mod
    base = _layer(torch, gpu_device, batch=2, buffer=32, k=k, sparse_values=values)
    prompt = _x(torch, gpu_device, 2, 150, 9)
    assert base(prompt, attend=True).shape == (2, 150, HIDDEN)
    of = [0, 1, 1, 0, 1]
    fork = base.fork(of, 16, 200, [k] * 5, sparse_values=values)
    assert fork.positions() == [150] * 5 and fork.W_qkv is base.W_qkv
    L = 0
    for n, seed in ((20, 21), (33, 22), (1, 23), (1, 24)):
        x = _x(torch, gpu_device, 5, n, seed)
        assert fork.positions() == [150 + L] * 5
        q, kk, vv = fork.project(x)
        held = [[torch.cat([R.cached_rows(base.cache, of[b], h, r),
                            R.cached_rows(fork.cache, b, h, r)]) for r in (0, 1)]
                for b in range(5) for h in range(2)]
        y = fork(x, attend=True)
        y = y[:, None] if n == 1 else y
        if n == 1:  # the step appends first: its own token as the cache holds it
            kk, vv = None, None
            held = [[torch.cat([R.cached_rows(base.cache, of[b], h, r),
                                R.cached_rows(fork.cache, b, h, r)]) for r in (0, 1)]
                    for b in range(5) for h in range(2)]
        want = torch.empty(5, n, 8 * D, dtype=torch.float64, device=gpu_device)
        for b in range(5):
            for hq in range(8):
                h = hq // 4
                P = base.P_qk[h].double()
                K, V = held[2 * b + h]
                if kk is not None:  # the chunk's keys in the rotated basis, where K is
                    K = torch.cat([K, kk[b, h].double() @ P])
                    V = torch.cat([V, vv[b, h].double()])
                seen = torch.ones(n, len(K), dtype=torch.bool, device=gpu_device).tril(len(K) - n)
                want[b, :, hq * D:(hq + 1) * D], _ = R.softmax_rows(q[b, hq].double() @ P, K, V, seen)
        assert _err(y, want @ base.W_o_hat.double()) < TOL, n
        L += n
    assert fork.cache.seq_len == [55] * 5 and base.cache.seq_len == [150] * 2
    with pytest.raises(ValueError):
        fork.fork([0], 16, 10, [k])
    with pytest.raises(ValueError):
        base.fork([2], 16, 10, [k])


def test_a_full_cache_leaves_the_layer_as_it_was(gpu_device, swan_mod, torch_mod):
    torch = torch_mod
    layer = _layer(torch, gpu_device, buffer=16, capacity=30)
    layer(_x(torch, gpu_device, 2, 40, 1), attend=True)
    before = [t.clone() for t in (layer.cache.k_pages, layer.cache.v_ring)]
    with pytest.raises(swan_mod.SwanError):
        layer(_x(torch, gpu_device, 2, 7, 2), attend=True)
    torch.cuda.synchronize()
    assert layer.cache.seq_len == [40, 40]
    for a, b in zip(before, (layer.cache.k_pages, layer.cache.v_ring)):
        assert torch.equal(a, b)
    layer(_x(torch, gpu_device, 2, 6, 2), attend=True)
    assert layer.cache.seq_len == [46, 46]
