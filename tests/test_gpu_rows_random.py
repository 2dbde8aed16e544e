"""Random shapes of rows over cached tokens, chunks and decode steps behind a prefix, against
the formula in float64 (the bounds of rows_ref)."""
import random

import pytest

from tests import rows_ref as R
from tests import swan_cases as C
from tests.test_gpu_prefix import _queries, _want

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("seed", range(24))
def test_random_rows(gpu_device, swan_mod, torch_mod, seed):
    torch = torch_mod
    rng = random.Random(1000 + seed)
    dtype, values = rng.choice([("f16", "same"), ("f16", "e4m3"), ("f32", "same")])
    hkv = rng.choice([1, 2, 3, 8])
    G = rng.choice([1, 2, 3, 4, 7, 8, 16])
    hq, B = hkv * G, rng.randint(1, 9)
    length = lambda top: rng.choice([0, 1, 63, 64, 65, rng.randint(0, top)])  # noqa: E731
    few = hkv * G > 24
    shared = [length(600 if few else 3000) for _ in range(rng.randint(1, 3))]
    lens = [length(300) for _ in range(B)]
    n = rng.choice([1, 2, 17, 33, 64, 130])
    ks = lambda count: [rng.randint(1, 128) for _ in range(count)]  # noqa: E731
    past, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, shared, hq, hkv, rng.choice([0, 5, 64, 130]),
                                      ks(len(shared)), dtype, seed, values, ks(len(shared)))
    own, _, _ = R.filled_cache(swan_mod, gpu_device, lens, hq, hkv, rng.choice([0, 16, 100]), ks(B),
                               dtype, seed + 50, "same", P=(P_qk, P_vo))
    of = [rng.randint(-1, len(shared) - 1) for _ in range(B)]
    prefix = swan_mod.Prefix(past, of)
    sources = [(past, of), (own, list(range(B)))]
    used = [rng.randint(0, n) for _ in range(B)]
    q = _queries(torch, gpu_device, (B, hq, n, D), dtype, seed)
    k = _queries(torch, gpu_device, (B, hkv, n, D), dtype, seed + 1, 0.5)
    v = _queries(torch, gpu_device, (B, hkv, n, D), dtype, seed + 2, 1.0)
    state = own.attend(q, P_qk, P_vo, n=used, prefix=prefix)
    chunk = swan_mod.prompt_attention(q, k, v, n=used, m=used, state=state)
    heads = sorted({0, hq - 1, rng.randrange(hq)})
    for b in range(B):
        for h in heads:
            rows = q[b, h, :used[b]]
            if not len(rows):
                continue
            o, lse, K, V = _want(sources, rows, b, h, G, P_qk, P_vo)
            tol = R.bound(dtype, rows, K, V, o, len(K), "f32", turned=True)
            R.close(state[0][b, h, :used[b]], o, tol, f"state {b} {h}")
            kb, vb = k[b, h // G, :used[b]], v[b, h // G, :used[b]]
            seen = torch.ones(used[b], used[b], dtype=torch.bool, device=gpu_device).tril()
            want, _ = R.softmax_rows(rows, kb, vb, seen, (o, lse))
            tol = R.bound(dtype, rows, kb, vb, want, len(K) + used[b])
            if len(K):
                tol = tol + R.bound(dtype, rows, K, V, o, len(K), "f32", turned=True)
            R.close(chunk[b, h, :used[b]], want, tol, f"chunk {b} {h}")
    some = [of[b] >= 0 and shared[of[b]] > 0 or lens[b] > 0 for b in range(B)]
    one = _queries(torch, gpu_device, (B, hq, D), dtype, seed + 3)
    if not all(some):
        with pytest.raises(swan_mod.SwanError):
            own.decode(one, P_qk, P_vo, prefix=prefix)
        return
    out = own.decode(one, P_qk, P_vo, prefix=prefix)
    for b in range(B):
        for h in heads:
            rows = one[b, h][None]
            want, _, K, V = _want(sources, rows, b, h, G, P_qk, P_vo)
            tol = R.bound(dtype, rows, K, V, want, len(K), turned=True)
            R.close(out[b, h][None], want, tol, f"decode {b} {h}")
