"""Every token found: rows of which each looks for one token of a cache or a prompt and
gets its value row, whatever page, ring slot, split or tile it lies in."""
import math

import pytest

from tests import needles as N
from tests import rows_ref as R
from tests import swan_cases as C

pytestmark = pytest.mark.gpu
D = 128
FORMATS = [("f16", "same"), ("f16", "e4m3"), ("f32", "same")]


def _cache(torch, swan_mod, device, batch, hkv, G, L, buffer, k, k_value, dtype, values, seed, P=None):
    """A cache of `batch` sequences with L tokens each, and what it holds of them as [batch]
    [hkv][L][D] float64."""
    td = C.torch_dtype(dtype)
    P = P or (R.rotations(hkv, seed + 1, device), R.rotations(hkv, seed + 2, device))
    cache = swan_mod.SwanCache(batch, hkv * G, hkv, buffer, max(0, L + 8 - buffer), [k] * batch, td,
                               device, sparse_values=values, k_value=[k_value] * batch)
    g = torch.Generator().manual_seed(seed + 3)
    K = torch.stack([N.rows(torch, hkv, L, k, seed + 10 * b) for b in range(batch)]).to(device)
    V = torch.randn(batch, hkv, L, D, generator=g).to(device)
    cache.append(*[torch.matmul(x, M.transpose(1, 2).contiguous()).to(td).contiguous()
                   for x, M in zip((K, V), P)], *P)
    held = [torch.stack([torch.stack([R.cached_rows(cache, b, h, r) for h in range(hkv)])
                         for b in range(batch)]) for r in (0, 1)]
    return cache, P, held


def _queries(torch, K, k, P, at, td):
    """[..., heads][n][D] queries for tokens `at` ([heads][n]) of K ([hkv][L][D])."""
    hkv = K.shape[0]
    G = len(at) // hkv
    out = [(K[h // G, at[h]] * N.sharpness(k)) @ P[h // G].double().T for h in range(len(at))]
    return torch.stack(out).to(td)


def _check(torch, got, V, at, P_vo, half, what):
    """got [heads][n][D] against the value rows of V ([hkv][L][D]) at `at`."""
    G = len(at) // V.shape[0]
    for h in range(len(at)):
        want = V[h // G, at[h]]
        if P_vo is not None:
            want = want @ P_vo[h // G].double().T
        miss = N.misses(torch, got[h], want, half, P_vo is not None)
        assert miss <= 1, f"{what}, head {h}: {miss:.3g} of the bound"


# kv heads, heads of each, tokens, buffer, k, k of values
CACHES = [(2, 4, 700, 60, 64, 48), (1, 3, 641, 0, 100, 128), (1, 1, 333, 130, 40, 24),
          (2, 2, 300, 16, 128, 128), (1, 8, 193, 64, 8, 77), (3, 1, 130, 200, 64, 64),
          (1, 2, 65, 1, 128, 8)]


@pytest.mark.parametrize("dtype,values", FORMATS)
@pytest.mark.parametrize("hkv,G,L,buffer,k,k_value", CACHES)
@pytest.mark.parametrize("turned", [False, True])
def test_cached_tokens(gpu_device, swan_mod, torch_mod, hkv, G, L, buffer, k, k_value, dtype, values,
                       turned):
    """All tokens in one call (workgroups of 256 rows where a group fills them), then 25 or
    1 at a time (split keys)."""
    torch = torch_mod
    cache, P, (K, V) = _cache(torch, swan_mod, gpu_device, 1, hkv, G, L, buffer, k, k_value, dtype,
                              values, 1)
    K, V = K[0], V[0]
    assert min(N.gap(torch, x) for x in K) > 50
    P_vo = P[1] if turned else None
    order = torch.arange(L, device=gpu_device)
    at = torch.stack([(order + 37 * h) % L for h in range(hkv * G)])
    q = _queries(torch, K, k, P[0], at, cache.dtype)
    o, lse = cache.attend(q[None], P[0], P_vo)
    _check(torch, o[0], V, at, P_vo, 0.0, "all")
    score = (q.double().view(hkv, G, L, D) @ P[0].double()[:, None]).view(hkv * G, L, D)
    score = torch.stack([(score[h] * K[h // G, at[h]]).sum(-1) for h in range(hkv * G)])
    score = score / math.sqrt(D)
    assert ((lse[0].double() - score).abs() <= 181 * 130 * 2.0 ** -23).all()
    for first in list(range(0, L, 25)) if not turned else [0, L - 25]:
        some = q[:, first:first + 25].contiguous()
        o, _ = cache.attend(some[None], P[0], P_vo)
        _check(torch, o[0], V, at[:, first:first + 25], P_vo, 0.0, f"from {first}")
    for t in (0, 63, 64, L - buffer - 1, L - buffer, L - 1):
        t = min(max(t, 0), L - 1)
        o, _ = cache.attend(q[None, :, t:t + 1].contiguous(), P[0], P_vo)
        _check(torch, o[0], V, at[:, t:t + 1], P_vo, 0.0, f"row {t}")


@pytest.mark.parametrize("dtype,values", FORMATS)
@pytest.mark.parametrize("hkv,G,L,buffer,k,k_value", CACHES[:5])
def test_tokens_of_a_prefix_and_own_ones(gpu_device, swan_mod, torch_mod, hkv, G, L, buffer, k,
                                         k_value, dtype, values):
    """Single tokens behind a prefix: 24 sequences a call, each looking for another token of
    it, then for each of the own ones; and rows over both sources at once."""
    torch = torch_mod
    td = C.torch_dtype(dtype)
    past, P, (K, V) = _cache(torch, swan_mod, gpu_device, 1, hkv, G, L, buffer, k, k_value, dtype,
                             values, 2)
    B, most = 24, 90
    own, _, (Ko, Vo) = _cache(torch, swan_mod, gpu_device, B, hkv, G, most, 40, k, k_value, dtype,
                              values, 500, P)
    every = torch.cat([K[0], Ko.transpose(0, 1).reshape(hkv, B * most, D)], 1)
    assert min(N.gap(torch, x) for x in every) > 50
    prefix = swan_mod.Prefix(past)
    half, heads = R.HALF[dtype], hkv * G
    for first in range(0, L, B):
        at = torch.stack([(torch.arange(B, device=gpu_device) + first + 11 * h) % L
                          for h in range(heads)])
        q = _queries(torch, K[0], k, P[0], at, td).transpose(0, 1).contiguous()
        out = own.decode(q, P[0], None, prefix=prefix)
        _check(torch, out.transpose(0, 1), V[0], at, None, half, f"prefix from {first}")
    out = own.decode(q, P[0], P[1], prefix=prefix)
    _check(torch, out.transpose(0, 1), V[0], at, P[1], half, "turned")
    for j in range(most):
        at = torch.stack([torch.full((1,), (j + 7 * h) % most, device=gpu_device)
                          for h in range(heads)])
        q = torch.cat([_queries(torch, Ko[b], k, P[0], at, td) for b in range(B)], 1)
        out = own.decode(q.transpose(0, 1).contiguous(), P[0], None, prefix=prefix)
        for b in range(0, B, 1 if j in (0, 49, 50, 51, 89) else 7):
            _check(torch, out[b][:, None], Vo[b], at, None, half, f"own {j} of {b}")
    # rows over a prefix's tokens and own ones, in turn
    n = 60
    for b in range(0, B, 9):
        atp = torch.stack([(torch.arange(n, device=gpu_device) * 13 + h) % L for h in range(heads)])
        ato = torch.stack([(torch.arange(n, device=gpu_device) * 7 + h) % most for h in range(heads)])
        mixed = torch.stack([_queries(torch, K[0], k, P[0], atp, td),
                             _queries(torch, Ko[b], k, P[0], ato, td)], 2)
        rows = mixed.view(heads, 2 * n, D)[None].contiguous()
        o, _ = swan_mod.attend([swan_mod.Prefix(past, [0]), swan_mod.Prefix(own, [b])], rows, P[0], None)
        o = o[0].view(heads, n, 2, D)
        _check(torch, o[:, :, 0], V[0], atp, None, 0.0, f"both, prefix, {b}")
        _check(torch, o[:, :, 1], Vo[b], ato, None, 0.0, f"both, own, {b}")


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("hkv,G,n,m,causal", [(2, 4, 333, 333, False), (1, 3, 1500, 1500, False),
                                              (2, 1, 333, 333, True), (1, 5, 129, 129, True),
                                              (1, 2, 100, 700, True), (3, 2, 64, 64, False)])
def test_keys_of_a_prompt(gpu_device, swan_mod, torch_mod, hkv, G, n, m, causal, dtype):
    """Each row looks for a key (that it sees); then a few rows at a time (split keys)."""
    torch = torch_mod
    td = C.torch_dtype(dtype)
    K = N.rows(torch, hkv, m, 64, 3).to(gpu_device).to(td)
    V = torch.randn(hkv, m, D, generator=torch.Generator().manual_seed(4)).to(gpu_device).to(td)
    assert min(N.gap(torch, x) for x in K) > 50
    eye = torch.eye(D, device=gpu_device).expand(hkv, D, D)
    i = torch.arange(n, device=gpu_device)
    reach = i + m - n + 1 if causal else torch.full_like(i, m)
    at = torch.stack([(i * 7 + 31 * h) % reach if h % 2 else reach - 1 - (i * 5 + h) % reach
                      for h in range(hkv * G)])
    q = _queries(torch, K.double(), 64, eye, at, td)
    got = swan_mod.prompt_attention(q[None], K[None], V[None], causal=causal)
    _check(torch, got[0], V.double(), at, None, R.HALF[dtype], "all")
    for first in range(0, n, 9):
        end = min(n, first + 9)
        seen = m - n + end if causal else m
        got = swan_mod.prompt_attention(q[None, :, first:end].contiguous(), K[None], V[None],
                                        causal=causal, m=[seen])
        _check(torch, got[0], V.double(), at[:, first:end], None, R.HALF[dtype], f"from {first}")


@pytest.mark.parametrize("dtype,values", FORMATS)
@pytest.mark.parametrize("n", [1, 3, 300])
def test_large_scores_to_float32_precision(gpu_device, swan_mod, torch_mod, n, dtype, values):
    """128 keys that are the rotated basis' axes, a query of one component: scores of up to
    +-150 that are single products, so a component of the rotated queries or of P that lost
    bits (2^-12 of them in one binary16 part) shows in every weight."""
    torch = torch_mod
    td = C.torch_dtype(dtype)
    P = R.rotations(1, 8, gpu_device)
    cache = swan_mod.SwanCache(1, 1, 1, 0, D + 8, [8], td, gpu_device, sparse_values=values)
    axes = torch.eye(D, device=gpu_device)
    eye = axes[None].contiguous()
    g = torch.Generator().manual_seed(9)
    V = torch.randn(1, 1, D, D, generator=g).to(gpu_device).to(td)
    cache.append(axes[None, None].to(td), V, eye, None)
    K, V = (R.cached_rows(cache, 0, 0, r) for r in (0, 1))
    assert torch.equal(K, axes.double())
    q = torch.zeros(n, D, device=gpu_device)
    q[torch.arange(n), torch.arange(n) % D] = 5000.0 + 7 * torch.arange(n, device=gpu_device)
    q = q.to(td)
    o, lse = cache.attend(q[None, None], P, None)
    want, wlse = R.softmax_rows(q.double() @ P[0].double(), K, V)
    size, _ = R.softmax_rows(q.double() @ P[0].double(), K, V.abs())
    most = q.double().abs().max().item() * P.abs().max().item() / math.sqrt(D)
    # a score's parts of P and of q 2^-23 each, four roundings of 2^-24 (P's product, the
    # factor, its constant, the score's own); then 100 steps of 2^-24 as in the weights' test
    score = most * (2 * 2.0 ** -23 + 4 * 2.0 ** -24)
    R.close(lse[0, 0], wlse, wlse.abs() * 2.0 ** -22 + score + 2.0 ** -20, "lse")
    # (in 16 bits a weight's second part is a multiple of 2^-24, so it is off by 2^-25 at most
    # beside a largest weight of 2^7 or more: 2^-32 of the sum for each of 128 keys)
    floor = D * 2.0 ** -32 * V.abs().max().item() if dtype == "f16" else 2.0 ** -60
    R.close(o[0, 0], want, size * (2 * score + 200 * 2.0 ** -24) + floor, "o")
