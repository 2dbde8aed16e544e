"""Softmax weights of the several-row operators to float32's precision, in storage of 16 bits
too.  Scores are exact (one component of q), so that what is left of the error is the
weights'; values cancel in pairs, so that a 16-bit result is small and its rounding with it."""
import math

import pytest

from tests import rows_ref as R

pytestmark = pytest.mark.gpu
D = 128


def _rows(torch, device, n, m, dtype, seed):
    """q [n][D], k and v [m][D]: row i of q scores -i/n * 3 on key 1, 0 on key 0 and far less
    on the others; dimension i of the values cancels keys 0 and 1 for row i (of 128)."""
    g = torch.Generator().manual_seed(seed)
    q, k = torch.zeros(n, D), torch.zeros(m, D)
    q[:, 0] = torch.arange(n) / n * 3 * math.sqrt(D)
    q[:, 1] = 32.0
    k[:, 1] = -7.25  # -20.5 in the exponent
    k[:2, 1] = 0
    k[1, 0] = -1.0
    q, k = q.to(dtype).to(device), k.to(dtype).to(device)
    v = torch.randn(m, D, generator=g).to(device)
    v[0] = 1.0
    s = (q[:, :1].double() @ k[1:2, :1].double().T)[:D, 0] / math.sqrt(D)
    v[1, :len(s)] = -torch.exp(-s).float()
    # somewhere among the others, side by side: each its own part's maximum would be exact
    return q, k.roll(2 * (m // 5), 0), v.to(dtype).roll(2 * (m // 5), 0)


def _want(q, k, v, out, seen=None):
    """The formula, and a bound on a kernel's error, in units of 2^-24 of the weighted sum of
    the values' magnitudes: an exponent of 12 at most beside its reference, off by 20 (its
    own rounding, its factor's, log2 e's and the reference's), 14 after ln 2; a weight's two
    parts and exp2's result 2 each; all that twice, for the sum and what it is divided by; 64
    for the sums and joins in float32.  Then the result's rounding."""
    want, lse = R.softmax_rows(q, k, v, seen)
    size, _ = R.softmax_rows(q, k, v.abs(), seen)
    return want, R.HALF[out] * want.abs() + size * (2 * 18 + 64) * 2.0 ** -24, lse


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n,m,causal", [(128, 200, False), (3, 1500, False), (1, 2, False),
                                        (128, 340, True)])
def test_prompt(gpu_device, swan_mod, torch_mod, n, m, causal, dtype):
    torch = torch_mod
    td = torch.float16 if dtype == "f16" else torch.float32
    q, k, v = _rows(torch, gpu_device, n, m, td, 1)
    if causal:  # the keys that matter before the first row's end
        top = k[:, 1] == 0
        first = torch.argsort(top.logical_not().to(torch.uint8), stable=True)
        k, v = k[first].contiguous(), v[first].contiguous()
    got = swan_mod.prompt_attention(q[None, None], k[None, None], v[None, None], causal=causal)
    seen = None
    if causal:
        seen = torch.ones(n, m, dtype=torch.bool, device=gpu_device).tril(m - n)
    want, tol, _ = _want(q, k, v, dtype, seen)
    R.close(got[0, 0], want, tol, "prompt")


FORMATS = [("f16", "same"), ("f16", "e4m3"), ("f32", "same")]


@pytest.mark.parametrize("dtype,values", FORMATS)
@pytest.mark.parametrize("heads", [1, 4])
def test_cached_rows(gpu_device, swan_mod, torch_mod, dtype, values, heads):
    """Unpruned pages (and a buffer) without rotations: few rows, then rows that fill
    workgroups of 256, then single tokens behind a prefix and their own."""
    torch = torch_mod
    td = torch.float16 if dtype == "f16" else torch.float32
    m, n = 500, 128
    q, k, v = _rows(torch, gpu_device, n, m, td, 2)
    eye = torch.eye(D, device=gpu_device)[None].contiguous()
    cache = swan_mod.SwanCache(1, heads, 1, 40, m, [D], td, gpu_device, sparse_values=values)
    cache.append(k[None, None], v[None, None], eye, eye)
    K, V = (R.cached_rows(cache, 0, 0, r) for r in (0, 1))
    for rows in (q[:5], q, q[100:101]):
        want, tol, wlse = _want(rows, K, V, "f32")
        many = rows[None, None].expand(1, heads, -1, -1).contiguous()
        o, lse = cache.attend(many, eye, None)
        for h in range(heads):
            R.close(o[0, h], want, tol, f"rows {len(rows)}, head {h}")
            R.close(lse[0, h], wlse, 2.0 ** -20 + 0 * wlse, "lse")
    # 32 sequences behind it, a row of q for each, with one own token far below
    B = 32
    own = swan_mod.SwanCache(B, heads, 1, 40, 10, [D] * B, td, gpu_device, sparse_values=values)
    far = k[k[:, 1] != 0][:1]
    own.append(far.expand(B, 1, 1, D).contiguous(), torch.ones(B, 1, 1, D, device=gpu_device, dtype=td),
               eye, eye)
    for first in range(0, n, B):
        rows = q[first:first + B]
        out = own.decode(rows[:, None].expand(-1, heads, -1).contiguous(), eye, None,
                         prefix=swan_mod.Prefix(cache))
        k1 = torch.cat([K, R.cached_rows(own, 0, 0, 0)])
        v1 = torch.cat([V, R.cached_rows(own, 0, 0, 1)])
        want, tol, _ = _want(rows, k1, v1, dtype)
        for h in range(heads):
            R.close(out[:, h], want, tol, f"decode, head {h}")


@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("far", [False, True])
def test_values_that_are_no_numbers(gpu_device, swan_mod, torch_mod, what, far):
    """One such value reaches its own dimension of every row, also with a weight of 2^-40 of
    the largest; the others keep their bits.  (Cached ones stand in the buffer and a page.)"""
    torch = torch_mod
    g = torch.Generator().manual_seed(3)
    n, m = 200, 300
    q = torch.zeros(n, D, dtype=torch.float16, device=gpu_device)
    q[:, 0] = 16.0 + torch.arange(n, device=gpu_device) / 64
    k = torch.zeros(m, D, dtype=torch.float16, device=gpu_device)
    k[:, 0] = torch.rand(m, generator=g).to(gpu_device)
    for at in (77, 290):
        k[at, 0] = -20.0 if far else 0.5  # 2^-41 at most of the others' weights
    v = torch.randn(m, D, generator=g).half().to(gpu_device)
    eye = torch.eye(D, device=gpu_device)[None].contiguous()
    rows = q[None, None]

    def all_of(v):
        cache = swan_mod.SwanCache(1, 1, 1, 40, m, [D], torch.float16, gpu_device)
        cache.append(k[None, None], v[None, None], eye, None)
        own = swan_mod.SwanCache(n // 8, 1, 1, 40, 10, [D] * (n // 8), torch.float16, gpu_device)
        first = k[:1].expand(n // 8, 1, 1, D).contiguous()
        own.append(first, first, eye, eye)
        return {"rows": swan_mod.prompt_attention(rows, k[None, None], v[None, None], causal=False),
                "few": swan_mod.prompt_attention(rows[:, :, :2].contiguous(), k[None, None],
                                                 v[None, None], causal=False),
                "cached": cache.attend(rows, eye, None)[0],
                "few cached": cache.attend(rows[:, :, :7].contiguous(), eye, None)[0],
                "decode": own.decode(q[::8, None].contiguous(), eye, None,
                                     prefix=swan_mod.Prefix(cache))[:, None]}

    good = all_of(v)
    v[77, 5] = what
    v[290, 9] = what
    got = all_of(v)
    other = [d for d in range(D) if d not in (5, 9)]
    for name in good:
        assert torch.equal(got[name][..., other], good[name][..., other]), name
        for d in (5, 9):
            x = got[name][..., d]
            assert torch.isnan(x).all() if math.isnan(what) else (x == what).all(), (name, d)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("power", [-60, -20, -10, 12])
def test_rotations_of_any_size(gpu_device, swan_mod, torch_mod, dtype, power):
    """P_qk times a power of two and the scale times its inverse: the same bits, few or many
    rows."""
    torch = torch_mod
    cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [300, 77], 8, 2, 16, [64, 128], dtype, 5)
    g = torch.Generator().manual_seed(6)
    q = torch.randn(2, 8, 70, D, generator=g).to(cache.dtype).to(gpu_device)
    for rows in (q, q[:, :, :1].contiguous()):
        want = cache.attend(rows, P_qk, P_vo, scale=0.11)
        got = cache.attend(rows, P_qk * 2.0 ** power, P_vo, scale=0.11 * 2.0 ** -power)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
