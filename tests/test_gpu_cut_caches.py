"""Caches cut to a window by outside() and select: what they answer is what the whole cache
answers, for the rows that outside() was asked about; other calls are refused."""
import pytest

from tests import rows_ref as R
from tests.test_gpu_window_cache import _check_decode, _queries

pytestmark = pytest.mark.gpu
D = 128

CUT = [  # lengths, hq, hkv, buffer, window, sinks, values
    ([500, 80, 300], 4, 4, 32, 100, 3, "same"),
    ([500, 80, 300], 8, 2, 32, 33, 0, "same"),  # a window of the buffer and one
    ([500, 131, 64], 8, 2, 0, 64, 64, "same"),
    ([300, 200], 4, 2, 100, 40, 4, "same"),  # a window within the buffer
    ([257, 65], 2, 2, 16, 1, 0, "same"),
    ([400, 399], 8, 2, 16, 150, 5, "e4m3"),
]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("lengths,hq,hkv,buffer,window,sinks,values", CUT)
def test_decode_of_a_cut_cache(gpu_device, swan_mod, torch_mod, lengths, hq, hkv, buffer, window,
                               sinks, values, dtype):
    """decode() stands at the last cached token, one before the rows of step() and attend()."""
    torch = torch_mod
    if values == "e4m3" and dtype == "f32":
        return
    src, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, lengths, hq, hkv, buffer,
                                     [48] * len(lengths), dtype, 7, values, spare=20)
    q = _queries(torch, gpu_device, dtype, len(lengths), hq, D, seed=3)
    every = range(len(lengths))
    cut = src.select(every, sinks, src.outside(window, sinks, decode=True))
    assert sum(cut.seq_len) < sum(src.seq_len)
    out = cut.decode(q, P_qk, P_vo, window=window, sinks=sinks)
    torch.cuda.synchronize()
    _check_decode(torch, src, q, P_qk, P_vo, out, window, sinks, dtype)
    # cut for later rows: refused where the last row misses a token, and a step is the source's
    cut = src.select(every, sinks, src.outside(window, sinks))
    short = [b for b in every if src.seq_len[b] - cut.seq_len[b] >
             src.seq_len[b] - src.select(every, sinks, src.outside(window, sinks, decode=True)).seq_len[b]]
    assert bool(short) == (window > buffer)
    if short:
        with pytest.raises(swan_mod.SwanError, match="left out"):
            cut.decode(q, P_qk, P_vo, window=window, sinks=sinks)
        same = cut.select(every)  # a copy of it is cut as it is
        with pytest.raises(swan_mod.SwanError, match="left out"):
            same.decode(q, P_qk, P_vo, window=window, sinks=sinks)
        if window > 1:
            cut.decode(q, P_qk, P_vo, window=window - 1, sinks=sinks)
    else:
        out = cut.decode(q, P_qk, P_vo, window=window, sinks=sinks)
        torch.cuda.synchronize()
        _check_decode(torch, src, q, P_qk, P_vo, out, window, sinks, dtype)
    k = _queries(torch, gpu_device, dtype, len(lengths), hkv, 1, D, seed=5, sharp=1)
    for c in (src, cut):
        out = c.step(k, k, q, P_qk, P_vo, window=window, sinks=sinks)
        torch.cuda.synchronize()
        _check_decode(torch, src if c is src else cut, q, P_qk, P_vo, out, window, sinks, dtype)
    _check_decode(torch, src, q, P_qk, P_vo, out, window, sinks, dtype)
    out = cut.decode(q, P_qk, P_vo, window=window, sinks=sinks)
    torch.cuda.synchronize()
    _check_decode(torch, src, q, P_qk, P_vo, out, window, sinks, dtype)


def test_decode_at_the_end_of_a_cut_prefix(gpu_device, swan_mod, torch_mod):
    """A sequence without tokens of its own stands at its prefix's last token."""
    torch = torch_mod
    window, sinks = 100, 3
    src, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [500], 8, 2, 16, [64], "f16", 7)
    own, _, _ = R.filled_cache(swan_mod, gpu_device, [0, 6], 8, 2, 16, [64] * 2, "f16", 9,
                               P=(P_qk, P_vo))
    q = _queries(torch, gpu_device, "f16", 2, 8, D, seed=3)
    whole = swan_mod.Prefix(src, [0, 0])
    kw = dict(window=window, sinks=sinks)
    cut = src.select([0], sinks, src.outside(window, sinks, decode=True))
    out = own.decode(q, P_qk, P_vo, prefix=swan_mod.Prefix(cut, [0, 0]), **kw)
    torch.cuda.synchronize()
    _check_decode(torch, own, q, P_qk, P_vo, out, window, sinks, "f16", whole)
    later = src.select([0], sinks, src.outside(window, sinks))
    with pytest.raises(swan_mod.SwanError, match="left out"):
        own.decode(q, P_qk, P_vo, prefix=swan_mod.Prefix(later, [0, 0]), **kw)
    with pytest.raises(swan_mod.SwanError, match="left out"):
        own.decode(q, P_qk, P_vo, prefix=swan_mod.Prefix(later), **kw)
    prefix = swan_mod.Prefix(later, [0, 0])
    k = _queries(torch, gpu_device, "f16", 2, 2, 1, D, seed=5, sharp=1)
    out = own.step(k, k, q, P_qk, P_vo, prefix=prefix, **kw)
    torch.cuda.synchronize()
    _check_decode(torch, own, q, P_qk, P_vo, out, window, sinks, "f16", whole)
    out = own.decode(q, P_qk, P_vo, prefix=prefix, **kw)
    torch.cuda.synchronize()
    _check_decode(torch, own, q, P_qk, P_vo, out, window, sinks, "f16", whole)
