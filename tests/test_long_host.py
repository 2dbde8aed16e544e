"""Refusals of the calls of swan_long.h: every bad call is turned down on the host, before
anything is enqueued (the pointers below are never dereferenced); and the host's part of
rotary positions and of what a window leaves."""
import ctypes
import math

import pytest

swan = pytest.importorskip("paper_2511_18936_amd.swan")

FAKE = 0x10000
BIG = 1 << 40
INVALID, UNSUPPORTED = swan.SWAN_ERR_INVALID_ARG, swan.SWAN_ERR_UNSUPPORTED
CAPACITY, WORKSPACE = swan.SWAN_ERR_CAPACITY, swan.SWAN_ERR_WORKSPACE
LIB = swan.lib()


def _i32(*v):
    return (ctypes.c_int32 * len(v))(*v)


def test_the_header_is_exported():
    import os
    import re

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "include", "swan_long.h")) as f:
        names = re.findall(r"^swan_status (swan_\w+)\(", f.read(), re.M)
    assert len(names) == 10 and len(set(names)) == 10
    for name in names:
        assert hasattr(LIB, name), name


# ---- rotary -----------------------------------------------------------------------------
def _rotary(dims=64, interleaved=0, magnitude=1.0, freqs=None):
    n = max(dims, 2) // 2
    f = (ctypes.c_double * n)(*(freqs or [0.5] * n))
    return swan.RotaryDesc(dims, interleaved, magnitude, f)


def _rope(r, **kw):
    a = dict(x=FAKE, y=FAKE, dtype=swan.SWAN_F16, batch=1, heads=2, n=3, d=128, pos0=_i32(0))
    a.update(kw)
    return LIB.swan_rope_rotary(a["x"], a["y"], a["dtype"], a["batch"], a["heads"], a["n"], a["d"],
                                a["pos0"], None if r is None else ctypes.byref(r), None)


def _rows(r, **kw):
    a = dict(batch=1, n=3, d=128, pos0=_i32(0), q=FAKE + (1 << 20))
    a.update(kw)
    return LIB.swan_qkv_rows_rotary(FAKE, 0, 12 * 128, swan.SWAN_F16, a["batch"], 8, 2, a["n"],
                                    a["d"], a["pos0"], None if r is None else ctypes.byref(r), None,
                                    None, 0, 0, 1e-6, a["q"], FAKE + (2 << 20), FAKE + (3 << 20),
                                    None)


BAD_FORMS = [dict(dims=0), dict(dims=-8), dict(dims=4), dict(dims=12), dict(dims=136),
             dict(interleaved=2), dict(interleaved=-1), dict(magnitude=0.0), dict(magnitude=-1.0),
             dict(magnitude=math.inf), dict(magnitude=math.nan), dict(freqs=[math.nan] * 32),
             dict(freqs=[1.0] * 31 + [math.inf])]


@pytest.mark.parametrize("kw", BAD_FORMS)
def test_rotary_forms_are_checked(kw):
    r = _rotary(**kw)
    assert _rope(r) == INVALID and "rotary" in swan.last_error()
    assert _rows(r) == INVALID
    assert _rope(r, n=0) == INVALID  # also where there is nothing to do


def test_rotary_calls_refuse():
    r = _rotary()
    assert _rope(None) == INVALID and _rows(None) == INVALID
    assert _rope(swan.RotaryDesc(64, 0, 1.0, None)) == INVALID
    assert _rope(r, n=0) == swan.SWAN_OK and _rows(r, n=0) == swan.SWAN_OK
    for kw in (dict(x=None), dict(y=None), dict(batch=0), dict(batch=65), dict(heads=0), dict(n=-1),
               dict(pos0=None), dict(pos0=_i32(-1)), dict(pos0=_i32(2**31 - 2)), dict(x=FAKE + 8)):
        assert _rope(r, **kw) == INVALID, kw
    assert _rope(r, d=64) == UNSUPPORTED and _rope(r, dtype=9) == UNSUPPORTED
    for kw in (dict(batch=0), dict(n=-1), dict(pos0=_i32(-1)), dict(q=None), dict(q=FAKE)):
        assert _rows(r, **kw) == INVALID, kw


def test_rotary_of_python():
    r = swan.Rotary(10000.0, dims=32)
    assert r.freqs == tuple(10000.0 ** (-j / 16) for j in range(16)) and r.magnitude == 1.0
    s = r.stretched(4.0)
    assert s.freqs == tuple(f / 4 for f in r.freqs) and s.dims == 32 and not s.interleaved
    p = swan.Rotary(500000.0, interleaved=True).by_parts(8.0, 8192, low=1, high=4, magnitude=1.0)
    assert p.interleaved and p.magnitude == 1.0
    for f, g in zip(swan.Rotary(500000.0).freqs, p.freqs):
        turns = 8192 * f / (2 * math.pi)
        if turns <= 1:
            assert g == f / 8
        elif turns >= 4:
            assert g == f
        else:
            assert f / 8 < g < f
            mix = (turns - 1) / 3
            assert math.isclose(g, f * mix + f / 8 * (1 - mix), rel_tol=1e-14)
    assert math.isclose(swan.Rotary().by_parts(8.0, 8192).magnitude, 0.1 * math.log(8) + 1)
    for kw in (dict(dims=0), dict(dims=12), dict(dims=136), dict(base=1.0), dict(base=math.nan),
               dict(base=math.inf), dict(freqs=[1.0] * 63), dict(freqs=[math.nan] * 64),
               dict(magnitude=0.0), dict(magnitude=math.nan), dict(magnitude=math.inf)):
        with pytest.raises(swan.SwanError):
            swan.Rotary(**kw)
    for low, high in ((0, 4), (4, 4), (5, 1)):
        with pytest.raises(swan.SwanError):
            swan.Rotary().by_parts(8.0, 8192, low, high)
    for factor in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(swan.SwanError):
            swan.Rotary().stretched(factor)
        with pytest.raises(swan.SwanError):
            swan.Rotary().by_parts(factor, 8192)


# ---- prompts with a window --------------------------------------------------------------
def _prompt(**kw):
    a = dict(q=FAKE, k=FAKE + (1 << 30), v=FAKE + (2 << 30), dtype=swan.SWAN_F16, batch=2, hq=8,
             hkv=2, n=4, m=300, d=128, ns=None, ms=None, window=10, sinks=None, scale=0.0, o0=None,
             lse0=None, out=FAKE + (3 << 30), ws=FAKE, wsb=BIG)
    a.update(kw)
    return LIB.swan_prompt_attention_window(
        a["q"], a["k"], a["v"], a["dtype"], a["batch"], a["hq"], a["hkv"], a["n"], a["m"], a["d"],
        a["ns"], a["ms"], a["window"], a["sinks"], a["scale"], a["o0"], a["lse0"], a["out"], a["ws"],
        a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(window=0), INVALID), (dict(window=-5), INVALID), (dict(sinks=_i32(0, -1)), INVALID),
    (dict(sinks=_i32(65536, 0)), INVALID), (dict(dtype=7), UNSUPPORTED), (dict(batch=0), INVALID),
    (dict(hq=7), INVALID), (dict(d=64), UNSUPPORTED), (dict(n=-1), INVALID),
    (dict(ns=_i32(5, 0)), INVALID), (dict(ms=_i32(0, 301)), INVALID), (dict(q=None), INVALID),
    (dict(k=None), INVALID), (dict(out=None), INVALID), (dict(q=FAKE + 8), INVALID),
    (dict(scale=math.nan), INVALID), (dict(scale=2.0 ** -70), INVALID), (dict(o0=FAKE), INVALID),
    (dict(out=FAKE), INVALID), (dict(out=FAKE + (1 << 30)), INVALID),
])
def test_windowed_prompts_are_checked(kw, status):
    assert _prompt(**kw) == status


def test_windowed_prompts_workspace():
    need = ctypes.c_size_t()
    args = (swan.SWAN_F16, 1, 8, 2, 1, 100000, 128, None, None)
    assert LIB.swan_prompt_window_workspace_bytes(*args, 50000, None, ctypes.byref(need)) == 0
    assert need.value > 0
    call = dict(batch=1, n=1, m=100000, window=50000)
    assert _prompt(**call, wsb=need.value - 1) == WORKSPACE
    assert _prompt(**call, ws=None) == WORKSPACE
    assert _prompt(**call, ws=FAKE + 16) == INVALID
    assert LIB.swan_prompt_window_workspace_bytes(*args, 64, None, None) == INVALID
    assert LIB.swan_prompt_window_workspace_bytes(*args, 0, None, ctypes.byref(need)) == INVALID
    # nothing to do
    assert _prompt(n=0) == swan.SWAN_OK


# ---- rows and single tokens over a cache ------------------------------------------------
def _desc(at=FAKE, **kw):
    d = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, buffer_tokens=16, sparse_capacity=1000,
             dtype=swan.SWAN_F16, reserved=0, k_pages=at, v_pages=at + (1 << 30),
             k_ring=at + (2 << 30), v_ring=at + (3 << 30))
    d.update(kw)
    return swan.CacheDesc(**d)


def _prefix(desc, lens, of, ks=(64, 64), keep=[]):
    keep[:] = [desc]
    return swan.PrefixDesc(ctypes.pointer(desc), _i32(*lens), _i32(*ks), None, _i32(*of))


def _attend(**kw):
    a = dict(src=_prefix(_desc(), (500, 20), (0, 1)), count=1, batch=2, n=4, ns=None, window=10,
             sinks=2, q=FAKE, P=FAKE, scale=0.0, o=FAKE, lse=FAKE + (1 << 30), ws=FAKE, wsb=BIG)
    a.update(kw)
    return LIB.swan_attend_window(ctypes.byref(a["src"]), a["count"], a["batch"], a["n"], a["ns"],
                                  a["window"], a["sinks"], a["q"], a["P"], None, a["scale"], a["o"],
                                  a["lse"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(window=0), INVALID), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID),
    (dict(sinks=65536), INVALID), (dict(count=0), INVALID), (dict(count=3), INVALID),
    (dict(batch=0), INVALID), (dict(n=-1), INVALID), (dict(q=None), INVALID), (dict(o=None), INVALID),
    (dict(scale=math.inf), INVALID), (dict(wsb=100), WORKSPACE), (dict(ws=FAKE + 16), INVALID),
    (dict(lse=FAKE), INVALID),
])
def test_windowed_rows_are_checked(kw, status):
    assert _attend(**kw) == status


def test_windowed_rows_positions_fit():
    big = _desc(sparse_capacity=2**30)
    src = _prefix(big, (2**30, 20), (0, 1))
    two = (swan.PrefixDesc * 2)(src, src)
    need = ctypes.c_size_t()
    call = lambda n: LIB.swan_attend_window_workspace_bytes(two, 2, 2, n, None, 10, 0,  # noqa: E731
                                                            ctypes.byref(need))
    assert call(1) == INVALID  # a length above 2^30 - 1 / 2, as without a window
    src = _prefix(big, (2**30 - 1, 20), (0, 1))
    two = (swan.PrefixDesc * 2)(src, src)
    assert call(1) == swan.SWAN_OK
    assert call(3) == UNSUPPORTED


def _decode(step=False, **kw):
    a = dict(prefix=None, c=_desc(), lens=_i32(500, 20), k=_i32(64, 64), kv=None, window=10, sinks=2,
             q=FAKE, P=FAKE, scale=0.0, out=FAKE, ws=FAKE, wsb=BIG, kn=FAKE)
    a.update(kw)
    p = None if a["prefix"] is None else ctypes.byref(a["prefix"])
    head = (p, ctypes.byref(a["c"]), a["lens"], a["k"], a["kv"], a["window"], a["sinks"])
    tail = (a["q"], a["P"], None, a["scale"], a["out"], a["ws"], a["wsb"], None)
    if step:
        return LIB.swan_decode_step_window(*head, a["kn"], a["kn"], *tail)
    return LIB.swan_decode_attention_window(*head, *tail)


@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(window=0), INVALID), (dict(sinks=-1), INVALID), (dict(sinks=65536), INVALID),
    (dict(lens=None), INVALID), (dict(lens=_i32(-2, 5)), INVALID),
    (dict(lens=_i32(1017, 5)), CAPACITY), (dict(k=_i32(64, 129)), INVALID), (dict(k=None), INVALID),
    (dict(kv=_i32(0, 64)), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID),
    (dict(P=None), INVALID), (dict(P=FAKE + 4), INVALID), (dict(scale=math.nan), INVALID),
    (dict(scale=2.0 ** -70), INVALID), (dict(ws=None), WORKSPACE), (dict(wsb=100), WORKSPACE),
    (dict(ws=FAKE + 64), INVALID), (dict(c=_desc(batch=65)), INVALID),
    (dict(c=_desc(k_pages=None)), INVALID), (dict(c=_desc(k_ring=None)), INVALID),
    (dict(c=_desc(head_dim=64)), UNSUPPORTED), (dict(c=_desc(buffer_tokens=5000)), UNSUPPORTED),
    (dict(prefix=_prefix(_desc(n_kv_heads=4), (5, 5), (0, 1))), INVALID),
    (dict(prefix=_prefix(_desc(dtype=swan.SWAN_F32), (5, 5), (0, 1))), INVALID),
    (dict(prefix=_prefix(_desc(), (5, 5), (0, 2))), INVALID),
    (dict(prefix=_prefix(_desc(), (-1, 5), (0, 0))), INVALID),
    (dict(prefix=_prefix(_desc(), (2000, 5), (0, 0))), CAPACITY),
])
def test_windowed_decode_is_checked(kw, status, step):
    assert _decode(step, **kw) == status


def test_windowed_decode_needs_a_token():
    assert _decode(lens=_i32(5, 0)) == INVALID and "no token" in swan.last_error()
    assert _decode(step=True, kn=None) == INVALID
    far = _desc(at=1 << 36)
    p = _prefix(far, (7, 0), (0, 1))
    assert _decode(lens=_i32(5, 0), prefix=p) == INVALID  # its prefix is empty too
    own = _desc()
    assert _decode(step=True, c=own, prefix=_prefix(own, (5, 5), (0, 1))) == INVALID
    assert "appended to" in swan.last_error()


# ---- copies -----------------------------------------------------------------------------
def _copy(**kw):
    a = dict(src=_desc(), dst=_desc(at=1 << 36), lens=_i32(500, 20), ks=_i32(64, 64), kvs=None,
             kd=_i32(64, 64), kvd=None, of=_i32(1, 0), first=_i32(0, 0), drop=_i32(0, 0))
    a.update(kw)
    return LIB.swan_copy_sequences(ctypes.byref(a["src"]), a["lens"], a["ks"], a["kvs"],
                                   ctypes.byref(a["dst"]), a["kd"], a["kvd"], a["of"], a["first"],
                                   a["drop"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dst=_desc()), INVALID),
    (dict(dst=_desc(at=1 << 36, v_ring=FAKE + 64)), INVALID),
    (dict(dst=_desc(at=1 << 36, n_kv_heads=4)), INVALID),
    (dict(dst=_desc(at=1 << 36, n_q_heads=4)), INVALID),
    (dict(dst=_desc(at=1 << 36, buffer_tokens=8)), INVALID),
    (dict(dst=_desc(at=1 << 36, dtype=swan.SWAN_F32)), INVALID),
    (dict(dst=_desc(at=1 << 36, k_pages=None)), INVALID),
    (dict(of=None), INVALID), (dict(lens=None), INVALID), (dict(of=_i32(2, 0)), INVALID),
    (dict(of=_i32(-2, 0)), INVALID), (dict(lens=_i32(-1, 0)), INVALID),
    (dict(lens=_i32(1017, 0)), CAPACITY), (dict(kd=_i32(64, 48)), INVALID),
    (dict(kvd=_i32(64, 48)), INVALID), (dict(drop=_i32(5, 0)), INVALID),
    (dict(drop=_i32(0, 485)), INVALID), (dict(drop=_i32(0, -1)), INVALID),
    (dict(first=_i32(0, 400), drop=_i32(0, 85)), INVALID), (dict(first=_i32(-1, 0)), INVALID),
    (dict(dst=_desc(at=1 << 36, sparse_capacity=100)), CAPACITY),
    (dict(dst=_desc(at=1 << 36, sparse_capacity=100), drop=_i32(0, 383)), CAPACITY),
])
def test_copies_are_checked(kw, status):
    assert _copy(**kw) == status


def test_a_copy_of_nothing():
    assert _copy(of=_i32(-1, -1)) == swan.SWAN_OK


def test_what_a_window_leaves():
    cache = swan.SwanCache(4, 2, 2, 16, 1000, [64] * 4, __import__("torch").float16, "cpu")
    cache.seq_len = [500, 100, 20, 0]
    assert cache.outside(100, 4) == [397, 0, 0, 0]
    assert cache.outside(5, 4) == [480, 80, 0, 0]  # the ring's tokens stay
    assert cache.outside(1, [0, 1, 0, 0]) == [484, 83, 4, 0]
    with pytest.raises(swan.SwanError):
        cache.outside(0)


def test_sinks_and_windows_of_python():
    for window, sinks in ((None, 3), (None, [0, 1]), (2.0, 0), (True, 0), (5, 1.0), (2**31, 0),
                          (5, 2**32)):
        with pytest.raises(swan.SwanError):
            swan._window(window, sinks)
    swan._window(5, [1, 2])


@pytest.mark.parametrize("window,sinks", [(0, 0), (-1, 0), (-2**31 - 1, 0), (-2**32 + 5, 0), (5, -1),
                                          (5, -2**32 + 1), (5, [1, -2**32]), (5, [2**32, 0])])
def test_numbers_that_32_bits_would_wrap(window, sinks):
    """ctypes takes a number's low 32 bits: -2^31 - 1 would be a window of 2^31 - 1."""
    with pytest.raises(swan.SwanError):
        swan._window(window, sinks)
    cache = swan.SwanCache(2, 2, 2, 16, 1000, [64] * 2, __import__("torch").float16, "cpu")
    cache.seq_len = [500, 100]
    with pytest.raises(swan.SwanError):
        cache.outside(window, sinks)


def test_what_a_window_leaves_takes_whole_lists():
    cache = swan.SwanCache(3, 2, 2, 16, 1000, [64] * 3, __import__("torch").float16, "cpu")
    cache.seq_len = [500, 100, 7]
    for sinks in ([0], [0] * 4, -1, 1.0):
        with pytest.raises(swan.SwanError):
            cache.outside(50, sinks)
    with pytest.raises(swan.SwanError):
        cache.outside(None)


@pytest.mark.parametrize("of,first,drop", [([2**32, 1], 0, None), ([0, 1], 2**32, [3, 3]),
                                           ([0, 1], [0, -2**32], [3, 3]), ([0, 1], 0, [2**32 + 1, 0])])
def test_copies_that_32_bits_would_wrap(of, first, drop):
    torch = __import__("torch")
    src, dst = (swan.SwanCache(2, 2, 2, 16, 1000, [64] * 2, torch.float16, "cpu") for _ in range(2))
    src.seq_len = [500, 100]
    with pytest.raises(swan.SwanError, match="out of range"):
        dst.copy_from(src, of, first, drop)
    assert dst.seq_len == [0, 0]


@pytest.mark.parametrize("original", [0, -4096, float("nan"), float("inf")])
def test_the_original_context_is_one(original):
    with pytest.raises(swan.SwanError):
        swan.Rotary(10000.0).by_parts(4.0, original)
