"""swan_prompt_attention_window against the formula in float64: windows of one key to all,
first keys, lengths and states that leave rows empty, infinities a row does not see, graphs."""
import math

import pytest

from tests import long_ref as LR
from tests import rows_ref as R
from tests import swan_cases as C

pytestmark = pytest.mark.gpu
D = 128


def _inputs(torch, device, B, hq, hkv, n, m, dtype, seed, sharp=1.5):
    g = torch.Generator().manual_seed(seed)
    td = C.torch_dtype(dtype)
    make = lambda h, r, s: (torch.randn(B, h, r, D, generator=g) * s).to(td).to(device)  # noqa: E731
    return make(hq, n, sharp), make(hkv, m, 1.0), make(hkv, m, 1.0)


def _check(torch, got, q, k, v, ns, ms, window, sinks, dtype, state=None):
    B, hq, n, _ = q.shape
    G = hq // k.shape[1]
    sinks = [sinks] * B if isinstance(sinks, int) else sinks
    for b in range(B):
        nb, mb = ns[b], ms[b]
        p = torch.arange(nb, device=q.device) + mb - nb
        seen = LR.seen_mask(p, torch.arange(mb, device=q.device), window, sinks[b])
        for h in range(hq):
            st = None if state is None else (state[0][b, h, :nb], state[1][b, h, :nb])
            kb, vb = k[b, h // G, :mb], v[b, h // G, :mb]
            want, _ = R.softmax_rows(q[b, h, :nb], kb, vb, seen, st)
            fine = vb[torch.isfinite(vb.float())]
            if state is not None:
                fine = torch.cat([fine.reshape(-1).float(), state[0].reshape(-1)])
            tol = R.bound(dtype, q[b, h, :nb], torch.nan_to_num(kb.double(), posinf=0, neginf=0),
                          fine.reshape(-1, 1), torch.nan_to_num(want, posinf=0, neginf=0), mb)
            R.close(got[b, h, :nb], want, tol, f"sequence {b}, head {h}")


CASES = [  # B, hq, hkv, n, m, window, sinks
    (1, 1, 1, 1, 1, 1, 0), (1, 2, 1, 70, 70, 1, 0), (1, 2, 1, 70, 70, 1, 1), (1, 4, 2, 200, 200, 64, 4),
    (2, 3, 1, 130, 130, 65, 64), (1, 8, 2, 300, 300, 63, 65), (1, 1, 1, 500, 500, 100, 0),
    (1, 16, 1, 257, 257, 17, 1), (1, 4, 4, 400, 400, 129, 200), (1, 2, 2, 333, 333, 5000, 3),
    (1, 2, 1, 1, 700, 128, 5), (2, 4, 2, 3, 1025, 300, 70), (1, 2, 1, 40, 640, 200, 0),
    (1, 2, 1, 140, 40, 16, 2), (1, 5, 1, 192, 192, 191, 0), (1, 2, 2, 64, 1000, 2**31 - 1, 0),
    (1, 2, 1, 150, 150, 20, 65535),
]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("B,hq,hkv,n,m,window,sinks", CASES)
def test_attention_is_the_formula(gpu_device, swan_mod, torch_mod, B, hq, hkv, n, m, window, sinks,
                                  dtype):
    torch = torch_mod
    q, k, v = _inputs(torch, gpu_device, B, hq, hkv, n, m, dtype, n + m)
    got = swan_mod.prompt_attention(q, k, v, window=window, sinks=sinks)
    torch.cuda.synchronize()
    _check(torch, got, q, k, v, [n] * B, [m] * B, window, sinks, dtype)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_random_shapes(gpu_device, swan_mod, torch_mod, dtype):
    import random

    torch = torch_mod
    rng = random.Random(3)
    for i in range(14):
        hkv = rng.choice([1, 2, 3])
        hq = hkv * rng.choice([1, 2, 4, 7])
        B, n, m = rng.randint(1, 3), rng.randint(1, 260), rng.randint(1, 400)
        window, sinks = rng.choice([1, 2, 31, 64, 90, 200]), rng.choice([0, 1, 30, 64, 128, 190])
        ns = [rng.randint(0, n) for _ in range(B)]
        ms = [rng.randint(0, m) for _ in range(B)]
        q, k, v = _inputs(torch, gpu_device, B, hq, hkv, n, m, dtype, i)
        print("shape", B, hq, hkv, n, m, window, sinks, ns, ms, flush=True)
        got = swan_mod.prompt_attention(q, k, v, n=ns, m=ms, window=window, sinks=sinks)
        torch.cuda.synchronize()
        _check(torch, got, q, k, v, ns, ms, window, sinks, dtype)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_a_window_over_everything_is_no_window(gpu_device, swan_mod, torch_mod, dtype):
    torch = torch_mod
    q, k, v = _inputs(torch, gpu_device, 2, 4, 2, 300, 300, dtype, 2)
    plain = swan_mod.prompt_attention(q, k, v)
    for window, sinks in ((300, 0), (10**9, 7), (1, 300)):
        got = swan_mod.prompt_attention(q, k, v, window=window, sinks=sinks)
        assert torch.equal(got, plain), (window, sinks)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_ragged_batches_with_nans_behind_them(gpu_device, swan_mod, torch_mod, dtype):
    torch = torch_mod
    n, m = 150, 210
    ns, ms = [150, 0, 1, 64, 65, 130], [210, 9, 1, 0, 65, 64]
    sinks = [4, 0, 1, 2, 64, 0]
    q, k, v = _inputs(torch, gpu_device, 6, 4, 2, n, m, dtype, 77)
    for b in range(6):
        q[b, :, ns[b]:] = math.nan
        k[b, :, ms[b]:] = math.nan
        v[b, :, ms[b]:] = math.nan
    out = torch.full_like(q, 5.0)
    swan_mod.prompt_attention(q, k, v, n=ns, m=ms, out=out, window=33, sinks=sinks)
    torch.cuda.synchronize()
    _check(torch, out, q, k, v, ns, ms, 33, sinks, dtype)
    for b in range(6):
        assert torch.all(out[b, :, ns[b]:] == 5.0)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_continued_from_a_state(gpu_device, swan_mod, torch_mod, dtype):
    """Rows with a state far below, beside and far above their scores, and without one; and rows
    that see no key but have a state (more rows than keys)."""
    torch = torch_mod
    for n, m, window, sinks in ((90, 90, 20, 3), (2, 1000, 100, 0), (70, 3, 2, 0)):
        q, k, v = _inputs(torch, gpu_device, 2, 4, 2, n, m, dtype, 5)
        g = torch.Generator().manual_seed(8)
        o = torch.randn(2, 4, n, D, generator=g).to(gpu_device)
        lse = (torch.randn(2, 4, n, generator=g) * 3).to(gpu_device)
        lse[0, 0], lse[0, 1], lse[1, 2] = -60.0, 60.0, -math.inf
        o[1, 2] = math.nan  # of no weight
        got = swan_mod.prompt_attention(q, k, v, state=(o, lse), window=window, sinks=sinks)
        o = torch.nan_to_num(o)
        _check(torch, got, q, k, v, [n] * 2, [m] * 2, window, sinks, dtype, (o, lse))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("place", ["value", "key"])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_nothing_comes_from_what_a_row_does_not_see(gpu_device, swan_mod, torch_mod, what, place,
                                                    dtype):
    """A bad key before the window, inside it and behind the row."""
    torch = torch_mod
    n, window, sinks = 300, 40, 2
    q, k, v = _inputs(torch, gpu_device, 1, 2, 1, n, n, dtype, 4)
    good = swan_mod.prompt_attention(q, k, v, window=window, sinks=sinks)
    where = k if place == "key" else v
    bad = (10, 70, 200)
    for j in bad:
        where[0, 0, j, 3] = what
    got = swan_mod.prompt_attention(q, k, v, window=window, sinks=sinks)
    torch.cuda.synchronize()
    hit = torch.zeros(n, dtype=torch.bool, device=q.device)
    for j in bad:
        hit[j:j + window] = True
    assert torch.equal(got[:, :, ~hit], good[:, :, ~hit])
    if place == "value":
        keep = [d for d in range(D) if d != 3]
        assert torch.equal(got[..., keep], good[..., keep])
        assert not torch.isfinite(got[0, :, hit, 3]).any()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("sinks", [3, 64, 70])
def test_infinite_first_keys_reach_every_row(gpu_device, swan_mod, torch_mod, dtype, sinks):
    """A first key and one of the windows, in a tile that holds keys of both: infinite in their
    dim for the rows that see them, the other dims as they were."""
    torch = torch_mod
    n, window = 400, 30
    q, k, v = _inputs(torch, gpu_device, 1, 3, 1, n, n, dtype, 14, sharp=0.5)
    good = swan_mod.prompt_attention(q, k, v, window=window, sinks=sinks)
    v[0, 0, sinks - 1, 5] = math.inf
    v[0, 0, 200, 7] = -math.inf
    v[0, 0, 100, 9] = math.nan
    got = swan_mod.prompt_attention(q, k, v, window=window, sinks=sinks)
    torch.cuda.synchronize()
    keep = [d for d in range(D) if d not in (5, 7, 9)]
    assert torch.equal(got[..., keep], good[..., keep])
    assert torch.all(got[:, :, sinks - 1:, 5] == math.inf)
    assert torch.equal(got[:, :, :sinks - 1, 5], good[:, :, :sinks - 1, 5])
    for dim, j in ((7, 200), (9, 100)):
        sees = torch.zeros(n, dtype=torch.bool, device=q.device)
        sees[j:j + window] = True
        assert torch.equal(got[:, :, ~sees, dim], good[:, :, ~sees, dim])
        assert not torch.isfinite(got[0, :, sees, dim]).any()


def test_the_results_repeat_and_do_not_depend_on_neighbours(gpu_device, swan_mod, torch_mod):
    torch = torch_mod
    q, k, v = _inputs(torch, gpu_device, 3, 8, 2, 500, 500, "f16", 9)
    got = swan_mod.prompt_attention(q, k, v, window=100, sinks=4)
    assert torch.equal(swan_mod.prompt_attention(q, k, v, window=100, sinks=4), got)
    q2, k2, v2 = q.clone(), k.clone(), v.clone()
    q2[0] *= 30
    k2[2], v2[2] = 1.0, -1.0
    assert torch.equal(swan_mod.prompt_attention(q2, k2, v2, window=100, sinks=4)[1], got[1])


def test_captured_and_replayed(gpu_device, swan_mod, torch_mod):
    """A captured call (with a join) gives the eager results at each replay, with other work
    between them."""
    torch = torch_mod
    q, k, v = _inputs(torch, gpu_device, 2, 4, 1, 2, 3000, "f16", 6)
    want = swan_mod.prompt_attention(q, k, v, window=2000, sinks=70)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    out = torch.zeros_like(q)
    with torch.cuda.graph(graph, stream=stream):
        swan_mod.prompt_attention(q, k, v, out=out, window=2000, sinks=70)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        swan_mod.prompt_attention(q, k, v, window=64)
