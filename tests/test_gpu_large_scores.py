"""Prompt attention where scores are far larger than float32's steps of one: finite inputs
give the formula's finite results."""
import math

import pytest

from tests import rows_ref as R

pytestmark = pytest.mark.gpu
D = 128
SIZES = {"f16": [300.0, 1000.0, 2048.0, 10000.0, 30000.0, 65504.0],
         "f32": [300.0, 30000.0, 1e6, 1e9, 1e15]}
CASES = [("f16", s) for s in SIZES["f16"]] + [("f32", s) for s in SIZES["f32"]]


def _signs(torch, device, seed, *shape):
    g = torch.Generator().manual_seed(seed)
    return (torch.randint(0, 2, shape, generator=g) * 2 - 1).to(device)


def _inputs(torch, device, dtype, size, n, m, seed):
    """Rows of +-size times up to 1, keys likewise; row i is key at[i] (the others score an
    eighth of it or so), values of any size that the type holds."""
    td = torch.float16 if dtype == "f16" else torch.float32
    g = torch.Generator().manual_seed(seed + 1)
    k = _signs(torch, device, seed, m, D) * size * (0.5 + 0.5 * torch.rand(m, D, generator=g).to(device))
    at = torch.randint(0, m, (n,), generator=g).to(device)
    v = torch.randn(m, D, generator=g).to(device) * 100
    return k[at].to(td), k.to(td), v.to(td), at


def _same(torch, got, want, dtype):
    """Weights of 1 and 0 leave the value itself; a float32 one divided by the sum it was
    multiplied with, half a step each."""
    if dtype == "f16":
        assert torch.equal(got, want)
    else:
        assert ((got - want).abs() <= 2.0 ** -22 * want.abs()).all()


@pytest.mark.parametrize("dtype,size", CASES)
@pytest.mark.parametrize("n,m", [(150, 150), (3, 1500), (300, 70), (1, 1)])
def test_a_row_finds_its_key(gpu_device, swan_mod, torch_mod, n, m, dtype, size):
    torch = torch_mod
    for seed in range(3):
        q, k, v, at = _inputs(torch, gpu_device, dtype, size, n, m, seed)
        got = swan_mod.prompt_attention(q[None, None], k[None, None], v[None, None], causal=False)
        _same(torch, got[0, 0], v[at], dtype)


@pytest.mark.parametrize("dtype,size", CASES)
@pytest.mark.parametrize("sign", [1, -1])
def test_causal_rows_of_one_direction(gpu_device, swan_mod, torch_mod, sign, dtype, size):
    """Keys grow (or, for sign = -1, scores fall below zero) along the prompt by more than a
    step of the scores: each row has its own key, its first for falling ones."""
    torch = torch_mod
    td = torch.float16 if dtype == "f16" else torch.float32
    n = 130
    way = _signs(torch, gpu_device, 5, D)
    grow = (torch.arange(1, n + 1, device=gpu_device) / n)[:, None]
    k = (way * size * grow).to(td)
    q = (sign * way * size).expand(n, D).to(td).contiguous()
    g = torch.Generator().manual_seed(6)
    v = torch.randn(n, D, generator=g).to(gpu_device).to(td)
    got = swan_mod.prompt_attention(q[None, None], k[None, None], v[None, None])
    _same(torch, got[0, 0], v if sign == 1 else v[:1].expand(n, D), dtype)


@pytest.mark.parametrize("dtype,size", CASES)
@pytest.mark.parametrize("n,m", [(1, 1), (140, 1), (2, 1000)])
def test_equal_keys_share(gpu_device, swan_mod, torch_mod, n, m, dtype, size):
    """All keys alike, in rows of any size: the mean of the values, which are +-1 in pairs
    but for the first."""
    torch = torch_mod
    td = torch.float16 if dtype == "f16" else torch.float32
    g = torch.Generator().manual_seed(7)
    way = _signs(torch, gpu_device, 8, D)
    q = (torch.randn(n, 1, generator=g).to(gpu_device) * way * size).clamp(-65504, 65504) \
        if dtype == "f16" else torch.randn(n, 1, generator=g).to(gpu_device) * way * size
    q = q.to(td)
    k = (way * size).to(td).expand(m, D).contiguous()
    v = torch.ones(m, D, device=gpu_device, dtype=td)
    v[1::2] = -1
    got = swan_mod.prompt_attention(q[None, None], k[None, None], v[None, None], causal=False)
    want = v.double().mean(0).expand(n, D)
    # equal weights, whose sums are exact or end in one rounding each of their float32 parts
    assert ((got[0, 0].double() - want).abs() <= R.HALF[dtype] * want.abs() + m * 2.0 ** -22).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("lse", [1e6, 3e8, 2.0 ** 33, 1e20, -3e8, -1e20])
@pytest.mark.parametrize("n,m", [(70, 70), (2, 1200), (5, 0)])
def test_states_far_from_the_scores(gpu_device, swan_mod, torch_mod, n, m, lse, dtype):
    """A state with a sum of e^(+-lse) beside scores of ordinary size: it alone, or none of it."""
    torch = torch_mod
    td = torch.float16 if dtype == "f16" else torch.float32
    g = torch.Generator().manual_seed(9)
    q, k, v = (torch.randn(1, 1, r, D, generator=g).to(td).to(gpu_device) for r in (n, m, m))
    o = torch.randn(1, 1, n, D, generator=g).to(gpu_device)
    at = lse * (1 + torch.rand(1, 1, n, generator=g).to(gpu_device))
    got = swan_mod.prompt_attention(q, k, v, causal=False, state=(o, at))
    if lse > 0 or m == 0:
        _same(torch, got, o.to(td), dtype)
    else:
        alone = swan_mod.prompt_attention(q, k, v, causal=False)
        # both rounded, of weights with other references (100 steps of 2^-24 of the values each)
        tol = 2 * R.HALF[dtype] * alone.double().abs() + v.abs().max().item() * 200 * 2.0 ** -24
        assert ((got.double() - alone.double()).abs() <= tol).all()


def test_a_far_row_beside_others(gpu_device, swan_mod, torch_mod):
    """A row's bits do not depend on whether its neighbours' scores are far."""
    torch = torch_mod
    g = torch.Generator().manual_seed(10)
    q, k, v = (torch.randn(1, 2, 150, D, generator=g).half().to(gpu_device) for _ in range(3))
    want = swan_mod.prompt_attention(q, k, v)
    changed = q.clone()
    changed[:, :, 1::2] *= 30000
    changed = changed.clamp(-65504, 65504)
    got = swan_mod.prompt_attention(changed, k * 1, v)
    assert torch.equal(got[:, :, 0::2], want[:, :, 0::2])
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("n,m", [(3, 20), (150, 100), (2, 1500), (140, 5)])
def test_float32_values_near_the_end_of_their_range(gpu_device, swan_mod, torch_mod, n, m):
    """Values and states of up to 3e38 whose weighted means are as large and finite: over a
    prompt's keys, cached ones, and single tokens behind a prefix."""
    torch = torch_mod
    g = torch.Generator().manual_seed(11)
    q, k = (torch.randn(1, 1, r, D, generator=g).to(gpu_device) for r in (n, m))
    v = torch.zeros(1, 1, m, D, device=gpu_device)
    v[0, 0, 2] = 3e38
    v[0, 0, 3] = -1e38
    o = torch.full((1, 1, n, D), 3e38, device=gpu_device)
    lse = torch.full((1, 1, n), math.log(m), device=gpu_device)
    eye = torch.eye(D, device=gpu_device)[None].contiguous()
    cache = swan_mod.SwanCache(1, 1, 1, 8, m, [D], torch.float32, gpu_device)
    cache.append(k, v, eye, None)
    B = min(n, 64)  # a batch's sequences
    own = swan_mod.SwanCache(B, 1, 1, 8, 8, [D] * B, torch.float32, gpu_device)
    own.append(k[:, :, :1].expand(B, 1, 1, D).contiguous(),
               v[:, :, :1].expand(B, 1, 1, D).contiguous(), eye, None)
    # 2^-60 of the values for the formula, which adds them up first
    small = (v[0, 0].double() * 2.0 ** -60)
    for name, got, state, keys, values in (
            ("prompt", swan_mod.prompt_attention(q, k, v, causal=False)[0, 0], None, k[0, 0], small),
            ("state", swan_mod.prompt_attention(q, k, v, causal=False, state=(o, lse))[0, 0],
             (o[0, 0].double() * 2.0 ** -60, lse[0, 0]), k[0, 0], small),
            ("cached", cache.attend(q, eye, None)[0][0, 0], None, k[0, 0], small),
            ("decode", own.decode(q[0, :, :B].transpose(0, 1).contiguous(), eye, None,
                                  prefix=swan_mod.Prefix(cache))[:, 0], None,
             torch.cat([k[0, 0], k[0, 0, :1]]), torch.cat([small, small[:1]]))):
        want, _ = R.softmax_rows(q[0, 0, :len(got)], keys, values, None, state)
        # as float32 attention anywhere: scores of 128 products of up to |q| |k| / sqrt(D) in
        # the exponent, twice, sums of m terms
        most = q.norm(dim=-1).max().item() * k.norm(dim=-1).max().item() / math.sqrt(D)
        rel = 2 * most * 130 * 2.0 ** -24 + (m + 64) * 2.0 ** -24
        tol = values.abs().max() * rel if state is None else 3e38 * 2.0 ** -60 * rel
        assert torch.isfinite(got).all(), name
        assert ((got.double() * 2.0 ** -60 - want).abs() <= tol).all(), name
