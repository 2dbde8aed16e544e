"""Windows, key by key: rows that each look for one token, whose value row is the whole result,
for every token that a row sees through a window, so that a single lost or leaked one shows.

Bounds: the token's weight is above 1 - 2^-17 (asserted), so what the scores' rounding (below 2^-12
of an exponent) makes of the other weights is below 2^-17 of the largest value; weights have 23 bits
at least; binary16 results are rounded once."""
import pytest

from tests import long_ref as LR
from tests import rows_ref as R
from tests import swan_cases as C

pytestmark = pytest.mark.gpu
D = 128


def _visible(p, window, sinks):
    first = max(0, p - window + 1)
    return [*range(min(sinks, first)), *range(first, p + 1)]


def _looking(torch, K, target):
    """Rows whose scores are largest for K[target]: K's rows to a norm that leaves the others
    far below, in float64."""
    k = K[target]
    return k * (60.0 * D ** 0.5 / (k * k).sum(-1, keepdim=True))


def _same(torch, got, want, weight, V, half, where):
    assert weight.min().item() > 1 - 2.0 ** -17, where
    bound = half * want.abs() + V.abs().max().item() * 2.0 ** -16 + 2.0 ** -25
    assert ((got.double() - want).abs() <= bound).all(), where


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n,m,window,sinks", [(300, 300, 100, 5), (130, 500, 129, 64), (257, 257, 64, 70),
                                              (90, 700, 333, 3), (200, 200, 1, 2), (33, 900, 512, 130)])
def test_prompts(gpu_device, swan_mod, torch_mod, n, m, window, sinks, dtype):
    torch = torch_mod
    td = C.torch_dtype(dtype)
    g = torch.Generator().manual_seed(m)
    k = torch.randn(1, 1, m, D, generator=g).to(td).to(gpu_device)
    v = torch.randn(1, 1, m, D, generator=g).to(td).to(gpu_device)
    K, V = k[0, 0].double(), v[0, 0].double()
    pos = torch.arange(n, device=gpu_device) + m - n
    seen = LR.seen_mask(pos, torch.arange(m, device=gpu_device), window, sinks)
    tokens = [_visible(p, window, sinks) for p in pos.tolist()]
    heads = 8
    for call in range((max(map(len, tokens)) + heads - 1) // heads):
        target = torch.tensor([[t[(call * heads + h) % len(t)] for t in tokens]
                               for h in range(heads)], device=gpu_device)
        q = _looking(torch, K, target).to(td)
        got = swan_mod.prompt_attention(q[None], k, v, window=window, sinks=sinks)[0]
        s = (q.double() @ K.T) / D ** 0.5
        w = torch.softmax(s.masked_fill(~seen, -float("inf")), -1)
        _same(torch, got, w @ V, w.gather(-1, target[..., None]), V, R.HALF[dtype], call)


CACHES = [([700, 260, 90, 5], 2, 4, 64, 300, 5), ([500, 333], 4, 1, 16, 129, 70),
          ([400, 64], 1, 8, 100, 90, 3), ([330, 129], 2, 2, 0, 200, 64)]


def _cache(swan, device, lengths, hkv, G, buffer, dtype):
    import torch

    g = torch.Generator().manual_seed(sum(lengths))
    td = C.torch_dtype(dtype)
    n = max(lengths)
    cache = swan.SwanCache(len(lengths), hkv * G, hkv, buffer, n, [64] * len(lengths), td, device)
    P = R.rotations(hkv, 3, device)
    rows = [torch.randn(len(lengths), hkv, n, D, generator=g).to(td).to(device) for _ in range(2)]
    cache.append(rows[0], rows[1], P, P, n_new_per_seq=list(lengths))
    return cache, P


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("lengths,hkv,G,buffer,window,sinks", CACHES)
def test_decode(gpu_device, swan_mod, torch_mod, lengths, hkv, G, buffer, window, sinks, dtype):
    torch = torch_mod
    cache, P = _cache(swan_mod, gpu_device, lengths, hkv, G, buffer, dtype)
    held = [[[R.cached_rows(cache, b, h, r).double() for r in (0, 1)] for h in range(hkv)]
            for b in range(len(lengths))]
    tokens = [_visible(L - 1, window, sinks) for L in lengths]
    heads = hkv * G
    for call in range((max(map(len, tokens)) + G - 1) // G):
        q = torch.zeros(len(lengths), heads, D, device=gpu_device, dtype=cache.dtype)
        picked = {}
        for b, t in enumerate(tokens):
            for h in range(hkv):
                target = torch.tensor([t[(call * G + x) % len(t)] for x in range(G)])
                turned = _looking(torch, held[b][h][0], target.to(gpu_device))
                q[b, h * G:(h + 1) * G] = (turned @ P[h].double().T).to(cache.dtype)
                picked[b, h] = target
        got = cache.decode(q, P, None, window=window, sinks=sinks)
        for (b, h), target in picked.items():
            K, V = held[b][h]
            L = lengths[b]
            s = (q[b, h * G:(h + 1) * G].double() @ P[h].double()) @ K.T / D ** 0.5
            seen = LR.seen_mask(torch.tensor([L - 1]), torch.arange(L), window, sinks)
            w = torch.softmax(s.masked_fill(~seen.to(gpu_device), -float("inf")), -1)
            _same(torch, got[b, h * G:(h + 1) * G], w @ V,
                  w.gather(-1, target.to(gpu_device)[:, None]), V, R.HALF[dtype], (call, b, h))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n", [7, 70])
@pytest.mark.parametrize("lengths,hkv,G,buffer,window,sinks", CACHES)
def test_rows_over_a_cache(gpu_device, swan_mod, torch_mod, lengths, hkv, G, buffer, window, sinks, n,
                           dtype):
    torch = torch_mod
    cache, P = _cache(swan_mod, gpu_device, lengths, hkv, G, buffer, dtype)
    held = [[[R.cached_rows(cache, b, h, r).double() for r in (0, 1)] for h in range(hkv)]
            for b in range(len(lengths))]
    # (rows that see no cached token any more look for the last)
    tokens = [[[t for t in _visible(L + i, window, sinks) if t < L] or [L - 1] for i in range(n)]
              for L in lengths]
    most = max(len(t) for rows in tokens for t in rows)
    for call in range(min(40, (most + G - 1) // G)):
        q = torch.zeros(len(lengths), hkv * G, n, D, device=gpu_device, dtype=cache.dtype)
        picked = {}
        for b, rows in enumerate(tokens):
            for h in range(hkv):
                target = torch.tensor([[t[(call * G + x + i) % len(t)] for i, t in enumerate(rows)]
                                       for x in range(G)], device=gpu_device)
                turned = _looking(torch, held[b][h][0], target)
                q[b, h * G:(h + 1) * G] = (turned @ P[h].double().T).to(cache.dtype)
                picked[b, h] = target
        o, lse = cache.attend(q, P, None, window=window, sinks=sinks)
        for (b, h), target in picked.items():
            K, V = held[b][h]
            L = lengths[b]
            s = (q[b, h * G:(h + 1) * G].double() @ P[h].double()) @ K.T / D ** 0.5
            seen = LR.seen_mask(L + torch.arange(n), torch.arange(L), window, sinks).to(gpu_device)
            some = seen.any(-1)
            w = torch.softmax(s.masked_fill(~seen, -float("inf")), -1)[:, some]
            got = o[b, h * G:(h + 1) * G]
            assert (got[:, ~some] == 0).all()
            assert torch.isinf(lse[b, h * G:(h + 1) * G][:, ~some]).all()
            if some.any():
                _same(torch, got[:, some], w @ V, w.gather(-1, target[:, some][..., None]), V,
                      R.HALF["f32"], (call, b, h))
