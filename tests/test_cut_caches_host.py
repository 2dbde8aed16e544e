"""SwanCache.outside() against its definition, and which decode calls a cut cache refuses (on
the CPU: the lengths alone)."""
import pytest
import torch

from paper_2511_18936_amd import swan


def _cache(lengths, buffer, capacity=2000):
    cache = swan.SwanCache(len(lengths), 2, 2, buffer, capacity, [64] * len(lengths), torch.float16,
                           "cpu")
    cache.seq_len = list(lengths)
    return cache


@pytest.mark.parametrize("window", [1, 5, 16, 17, 18, 63, 64, 100, 499, 500, 501, 10**9])
@pytest.mark.parametrize("buffer", [0, 16, 100])
@pytest.mark.parametrize("sinks", [0, 4, 70])
def test_what_rows_do_not_see(window, buffer, sinks):
    lengths = [0, 1, 15, 64, 100, 101, 130, 500]
    cache = _cache(lengths, buffer)
    for decode, row in ((False, 0), (True, -1)):
        drop = cache.outside(window, sinks, decode=decode)
        for L, d in zip(lengths, drop):
            p = L + row  # the first row to come
            hidden = [j for j in range(sinks, max(0, L - buffer)) if j <= p - window]
            assert d == len(hidden)
            assert hidden == list(range(sinks, sinks + d))


def _cut(monkeypatch, src, of, first, drop):
    """copy_from, but for the copy itself."""
    dst = _cache([0] * len(of), src.desc.buffer_tokens)
    monkeypatch.setattr(swan, "copy_sequences", lambda *a: None)
    monkeypatch.setattr(swan, "_same_gpu", lambda **kw: torch.device("cuda", 0))
    monkeypatch.setattr(swan, "_CallsOn", lambda *a: __import__("contextlib").nullcontext())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: None)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda *a: None)
    dst.copy_from(src, of, first, drop)
    return dst


def _refused(cache, window, sinks=0, prefix=None):
    try:
        cache._check_last_row(window, sinks, prefix)
    except swan.SwanError as e:
        assert e.status == swan.SWAN_ERR_INVALID_ARG and "left out" in str(e)
        return True
    return False


def test_which_decode_calls_are_refused(monkeypatch):
    src = _cache([500, 300, 40], 32)
    cut = _cut(monkeypatch, src, [0, 1, 2], 4, src.outside(100, 4))
    assert cut.seq_len == [4 + 99, 4 + 99, 40]
    assert _refused(cut, 100, 4)
    assert not _refused(cut, 99, 4)
    assert not _refused(_cut(monkeypatch, src, [2, 2], 4, [0, 0]), 100, 4)
    assert not _refused(_cut(monkeypatch, src, [0, 1], 4, src.outside(100, 4, decode=True)[:2]), 100, 4)
    # the buffer holds the last row's window: nothing that it shows is left out
    assert not _refused(_cut(monkeypatch, src, [0, 1], 4, src.outside(30, 4)[:2]), 30, 4)
    # a copy of a cut sequence; a sequence that grows, or takes another copy
    again = _cut(monkeypatch, cut, [-1, 2, 1], 0, None)
    assert _refused(again, 100, 4)
    again._grow([0, 40, 103])
    assert _refused(again, 100, 4)
    again._grow([1, 41, 104])
    assert not _refused(again, 100, 4)
    again = _cut(monkeypatch, cut, [1], 0, None)
    again.copy_from(src, [2])
    assert not _refused(again, 100, 4)
    # emptied and filled again to the same length
    cut.seq_len = [0, 0, 0]
    cut._grow([103, 103, 40])
    assert not _refused(cut, 100, 4)


def test_behind_a_prefix_that_was_cut(monkeypatch):
    src = _cache([500, 300], 32)
    cut = _cut(monkeypatch, src, [0, 1], 4, src.outside(100, 4))
    own = _cache([0, 3], 32)
    for of, refused in (([0, 0], True), ([1, 1], True), ([-1, 0], False), (None, True)):
        prefix = swan.Prefix(cut, of)
        assert _refused(own, 100, 4, prefix) == refused
    assert not _refused(own, 99, 4, swan.Prefix(cut, [0, 0]))
    own._grow([1, 4])
    assert not _refused(own, 100, 4, swan.Prefix(cut, [0, 0]))


def test_what_is_no_window_stays_an_error(monkeypatch):
    src = _cache([500], 32)
    cut = _cut(monkeypatch, src, [0], 4, src.outside(100, 4))
    for window, sinks in ((None, 4), (True, 0), (2.0, 0), (0, 0), (5, [1])):
        with pytest.raises(swan.SwanError):
            cut._check_last_row(window, sinks, None)
