"""What a window hides does not reach a result, in the forms whose pages hold something of
their own: 8-bit values (a NaN code), a prefix, the workgroups of 256 rows; and a window that
hides nothing, for single tokens and every storage."""
import math

import pytest

from tests import rows_ref as R
from tests.test_gpu_window_cache import _check_decode, _poison, _queries

pytestmark = pytest.mark.gpu
D = 128


def _spoil(torch, cache, b, tokens, what):
    """Every value of these pruned tokens becomes `what`: of 8-bit values their NaN code, the only
    one that is no number."""
    if cache.sparse_values != "e4m3":
        return _poison(torch, cache, b, tokens, what)
    hkv, npc = cache.desc.n_kv_heads, (cache.desc.sparse_capacity + 63) // 64
    up = lambda k: (k + 7) // 8 * 8  # noqa: E731
    for pages, ks in ((cache.k_pages, cache.k_active), (cache.v_pages, cache.k_value or cache.k_active)):
        page = [up(k) * 64 * 2 for k in ks]
        first = sum(page[:b]) * npc * hkv
        unit = pages[first:first + page[b] * npc * hkv].view(hkv, npc, -1)
        vals = unit[..., :64 * up(ks[b])].view(hkv, npc, up(ks[b]) // 8, 64, 8)
        for t in tokens:
            vals[:, t // 64, :, t % 64] = 0x7F


FORMS = [("f16", 4, 4, "e4m3"), ("f16", 8, 2, "e4m3"), ("f16", 4, 4, "same"), ("f16", 8, 2, "same"),
         ("f32", 4, 2, "same")]


@pytest.mark.parametrize("dtype,hq,hkv,values", FORMS)
def test_hidden_codes_and_numbers(gpu_device, swan_mod, torch_mod, dtype, hq, hkv, values):
    """Pages of a cache: the tokens are hidden from decode and all rows, then one from the last
    rows alone."""
    torch = torch_mod
    window, sinks, L, what = 40, 4, 400, math.nan
    made = lambda: R.filled_cache(swan_mod, gpu_device, [90, L], hq, hkv, 16, [33, 64], dtype, 7,  # noqa: E731
                                  values)
    good, P_qk, P_vo = made()
    bad, _, _ = made()
    q = _queries(torch, gpu_device, dtype, 2, hq, D, seed=3)
    rows = _queries(torch, gpu_device, dtype, 2, hq, 60, D, seed=4)
    _spoil(torch, bad, 1, [4, 63, 64, 200, L - window - 1], what)
    if values == "e4m3":
        spoilt = R.cached_rows(bad, 1, 0, 1)
        assert torch.isnan(spoilt[200]).any() and torch.isfinite(spoilt[201]).all()
    want = good.decode(q, P_qk, P_vo, window=window, sinks=sinks)
    assert torch.equal(bad.decode(q, P_qk, P_vo, window=window, sinks=sinks), want)
    want = good.attend(rows, P_qk, P_vo, window=window, sinks=sinks)
    got = bad.attend(rows, P_qk, P_vo, window=window, sinks=sinks)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    at = L - 20
    _spoil(torch, bad, 1, [at], what)
    want = good.attend(rows, P_qk, None, window=window, sinks=sinks)
    got = bad.attend(rows, P_qk, None, window=window, sinks=sinks)
    last = at + window - 1 - L
    assert torch.equal(got[0][1, :, last + 1:], want[0][1, :, last + 1:])
    assert torch.equal(got[0][0], want[0][0])
    assert torch.isnan(got[0][1, :, :last + 1]).any(-1).all()
    assert torch.isnan(bad.decode(q, P_qk, P_vo, window=window, sinks=sinks)[1]).any(-1).all()


@pytest.mark.parametrize("dtype,hq,hkv,values", FORMS)
def test_hidden_tokens_of_a_prefix(gpu_device, swan_mod, torch_mod, dtype, hq, hkv, values):
    torch = torch_mod
    window, sinks, L = 40, 4, 300
    made = lambda: R.filled_cache(swan_mod, gpu_device, [70, L], hq, hkv, 16, [40, 64], dtype, 7,  # noqa: E731
                                  values)
    good, P_qk, P_vo = made()
    bad, _, _ = made()
    _spoil(torch, bad, 1, [4, 63, 64, 200, L + 10 - window - 1], math.nan)
    own, _, _ = R.filled_cache(swan_mod, gpu_device, [10, 10, 25], hq, hkv, 16, [64] * 3, dtype, 9,
                               values, P=(P_qk, P_vo))
    of = [1, -1, 1]
    q = _queries(torch, gpu_device, dtype, 3, hq, D, seed=3)
    rows = _queries(torch, gpu_device, dtype, 3, hq, 60, D, seed=4)
    kw = dict(window=window, sinks=sinks)
    pg, pb = swan_mod.Prefix(good, of), swan_mod.Prefix(bad, of)
    assert torch.equal(own.decode(q, P_qk, P_vo, prefix=pb, **kw),
                       own.decode(q, P_qk, P_vo, prefix=pg, **kw))
    want = own.attend(rows, P_qk, P_vo, prefix=pg, **kw)
    got = own.attend(rows, P_qk, P_vo, prefix=pb, **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    at = L - 20  # seen by the first rows of sequence 0, by fewer of sequence 2
    _spoil(torch, bad, 1, [at], math.nan)
    want = own.attend(rows, P_qk, None, prefix=pg, **kw)[0]
    got = own.attend(rows, P_qk, None, prefix=pb, **kw)[0]
    for b, before in ((0, 10), (2, 25)):
        last = at + window - 1 - (L + before)
        assert (last >= 0) == (b == 0)
        assert torch.equal(got[b, :, max(last + 1, 0):], want[b, :, max(last + 1, 0):])
        if last >= 0:
            assert torch.isnan(got[b, :, :last + 1]).any(-1).all()
    assert torch.equal(got[1], want[1])


@pytest.mark.parametrize("values,k", [("same", 64), ("same", 128), ("e4m3", 64)])
@pytest.mark.parametrize("what", [math.inf, math.nan])
def test_workgroups_of_256_rows(gpu_device, swan_mod, torch_mod, values, k, what):
    """4 x 256 rows of 32 heads on 8: row tiles of 256, whose rows see parts of a tile.  Rows that
    see a value which is no number get it in its dim, the others keep their bits."""
    torch = torch_mod
    window, sinks, L, n = 2000, 4, 2500, 256
    made = lambda: R.filled_cache(swan_mod, gpu_device, [L] * 4, 32, 8, 64, [k] * 4, "f16", 7,  # noqa: E731
                                  values)
    good, P_qk, P_vo = made()
    bad, _, _ = made()
    rows = _queries(torch, gpu_device, "f16", 4, 32, n, D, seed=4, sharp=1)
    kw = dict(window=window, sinks=sinks)
    want = good.attend(rows, P_qk, None, **kw)[0]
    at = [L - window + 1 + x for x in (20, 150)]  # hidden from row 20 on, from 150 on
    if values == "e4m3":
        _spoil(torch, bad, 2, at, what)
    else:
        for t in at:  # (the values alone: their keys stay)
            keys = bad.k_pages.clone()
            _poison(torch, bad, 2, [t], what)
            bad.k_pages.copy_(keys)
    bad.v_ring[1, :, (L - 30) % 64, 9] = what  # a ring's: seen by every row
    got = bad.attend(rows, P_qk, None, **kw)[0]
    for b in (0, 3):
        assert torch.equal(got[b], want[b])
    assert torch.equal(got[2, :, 151:], want[2, :, 151:])
    assert not torch.isfinite(got[2, :, :150]).all(-1).any()
    keep = [d for d in range(D) if d != 9]
    assert torch.equal(got[1][..., keep], want[1][..., keep])
    assert torch.all(got[1, :, :, 9] == what) if what == math.inf else torch.isnan(got[1, :, :, 9]).all()


@pytest.mark.parametrize("dtype,hq,hkv,values", FORMS)
def test_a_window_that_hides_nothing(gpu_device, swan_mod, torch_mod, dtype, hq, hkv, values):
    """Rows over a cache: the bits of the call without a window.  Single tokens: both calls within
    the bound of the formula (their splits differ)."""
    torch = torch_mod
    cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [500, 90], hq, hkv, 64, [64, 64], dtype,
                                       7, values)
    rows = _queries(torch, gpu_device, dtype, 2, hq, 30, D, seed=4)
    q = _queries(torch, gpu_device, dtype, 2, hq, D, seed=3)
    a = cache.attend(rows, P_qk, P_vo)
    plain = cache.decode(q, P_qk, P_vo)
    for window, sinks in ((1000, 0), (1, 530)):
        b = cache.attend(rows, P_qk, P_vo, window=window, sinks=sinks)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        out = cache.decode(q, P_qk, P_vo, window=window, sinks=sinks)
        torch.cuda.synchronize()
        for got in (out, plain):
            _check_decode(torch, cache, q, P_qk, P_vo, got, window, sinks, dtype)
