"""Refusals of the several-row operators: every bad call is turned down on the host, before
anything is enqueued (the pointers below are never dereferenced)."""
import ctypes
import math

import pytest

swan = pytest.importorskip("paper_2511_18936_amd.swan")

FAKE = 0x10000
BIG = 1 << 40
INVALID, UNSUPPORTED = swan.SWAN_ERR_INVALID_ARG, swan.SWAN_ERR_UNSUPPORTED
CAPACITY, WORKSPACE = swan.SWAN_ERR_CAPACITY, swan.SWAN_ERR_WORKSPACE


def _i32(*v):
    return (ctypes.c_int32 * len(v))(*v)


def _header(name):
    import os

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "include", name)) as f:
        return f.read()


def test_the_layer_header_is_exported():
    import re

    names = re.findall(r"^swan_status (swan_\w+)\(", _header("swan_layer.h"), re.M)
    assert len(names) == 9 and len(set(names)) == 9
    for name in names:
        assert hasattr(swan.lib(), name), name


# ---- swan_qkv_rows ----------------------------------------------------------------------
def _qkv(**kw):
    a = dict(qkv=FAKE, seq=12 * 128 * 4, row=12 * 128, dtype=swan.SWAN_F16, batch=2, hq=8, hkv=2,
             n=4, d=128, pos0=_i32(0, 5), base=10000.0, qw=None, kw=None, per_head=0, w32=0,
             eps=1e-6, q=FAKE + (1 << 20), k=FAKE + (2 << 20), v=FAKE + (3 << 20))
    a.update(kw)
    return swan.lib().swan_qkv_rows(a["qkv"], a["seq"], a["row"], a["dtype"], a["batch"], a["hq"],
                                    a["hkv"], a["n"], a["d"], a["pos0"], a["base"], a["qw"],
                                    a["kw"], a["per_head"], a["w32"], a["eps"], a["q"], a["k"],
                                    a["v"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), UNSUPPORTED), (dict(d=64), UNSUPPORTED), (dict(batch=0), INVALID),
    (dict(batch=65), INVALID), (dict(n=-1), INVALID), (dict(hq=-1), INVALID),
    (dict(hq=0, hkv=0), INVALID), (dict(hq=70000), INVALID), (dict(base=1.0), INVALID),
    (dict(base=math.inf), INVALID), (dict(base=math.nan), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=math.nan), INVALID), (dict(pos0=None), INVALID), (dict(pos0=_i32(0, -1)), INVALID),
    (dict(pos0=_i32(0, 2**31 - 3)), INVALID), (dict(row=12 * 128 - 8), INVALID),
    (dict(row=12 * 128 + 4), INVALID), (dict(seq=4), INVALID), (dict(seq=-8), INVALID),
    (dict(qkv=None), INVALID), (dict(q=None), INVALID), (dict(v=None), INVALID),
    (dict(qkv=FAKE + 8), INVALID), (dict(qw=FAKE + 2), INVALID), (dict(per_head=2), INVALID),
    (dict(w32=-1), INVALID), (dict(q=FAKE), INVALID), (dict(v=FAKE + (2 << 20) + 512), INVALID),
    (dict(batch=64, n=2**26, pos0=_i32(*[0] * 64)), INVALID),
])
def test_qkv_rows_refuses(kw, status):
    assert _qkv(**kw) == status and swan.last_error()


def test_no_rows_of_qkv_are_fine():
    assert _qkv(n=0, qkv=None, q=None, k=None, v=None) == swan.SWAN_OK


# ---- swan_prompt_attention --------------------------------------------------------------
def _prompt(**kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, dtype=swan.SWAN_F16, batch=2, hq=8, hkv=2, n=4, m=9, d=128,
             ns=None, ms=None, causal=1, scale=0.0, o0=None, lse0=None, out=FAKE, ws=None,
             bytes=0)
    a.update(kw)
    return swan.lib().swan_prompt_attention(a["q"], a["k"], a["v"], a["dtype"], a["batch"],
                                            a["hq"], a["hkv"], a["n"], a["m"], a["d"], a["ns"],
                                            a["ms"], a["causal"], a["scale"], a["o0"], a["lse0"],
                                            a["out"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=9), UNSUPPORTED), (dict(batch=0), INVALID), (dict(batch=65), INVALID),
    (dict(hq=7), INVALID), (dict(hkv=0), INVALID), (dict(d=64), UNSUPPORTED),
    (dict(n=-1), INVALID), (dict(m=-1), INVALID), (dict(n=2**30), INVALID),
    (dict(ns=_i32(4, 5)), INVALID), (dict(ns=_i32(-1, 4)), INVALID), (dict(ms=_i32(9, 10)), INVALID),
    (dict(causal=2), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID),
    (dict(scale=1e-30), INVALID), (dict(o0=FAKE), INVALID), (dict(lse0=FAKE), INVALID),
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(out=None), INVALID),
    (dict(v=FAKE + 4), INVALID), (dict(o0=FAKE + 4, lse0=FAKE), INVALID),
    (dict(n=2**28, hq=16, hkv=2), UNSUPPORTED),
    (dict(n=1, m=5000, causal=0), WORKSPACE), (dict(n=1, m=5000, causal=0, ws=FAKE, bytes=64), WORKSPACE),
    (dict(n=1, m=5000, causal=0, ws=FAKE + 16, bytes=BIG), INVALID),
])
def test_prompt_attention_refuses(kw, status):
    assert _prompt(**kw) == status and swan.last_error()


@pytest.mark.parametrize("name", ["q", "k", "v", "o0", "lse0"])
def test_prompt_attention_refuses_an_out_over_its_inputs(name):
    """The last bytes of an input, 2 x 8 x 4 rows of q, 2 x 2 x 9 of k, or the state's."""
    far = {x: FAKE + (i << 24) for i, x in enumerate(("q", "k", "v", "o0", "lse0"), 1)}
    size = {"q": 64 * 256, "k": 36 * 256, "v": 36 * 256, "o0": 64 * 512, "lse0": 64 * 4}[name]
    assert _prompt(**far, out=far[name] + size - 16) == INVALID
    assert "overlaps" in swan.last_error()


def test_no_rows_of_a_prompt_are_fine():
    none = dict(q=None, k=None, v=None, out=None)
    assert _prompt(n=0, **none) == swan.SWAN_OK
    assert _prompt(ns=_i32(0, 0), **none) == swan.SWAN_OK


def test_prompt_workspace():
    def need(n, m, causal, hq=8, hkv=2, dtype=swan.SWAN_F16, ns=None):
        out = ctypes.c_size_t(7)
        st = swan.lib().swan_prompt_workspace_bytes(dtype, 1, hq, hkv, n, m, 128, ns, None, causal,
                                                    ctypes.byref(out))
        assert st == swan.SWAN_OK, swan.last_error()
        return out.value

    assert need(4096, 4096, 1, 32, 8) == 0  # row tiles enough to fill the GPU
    parts = need(1, 20000, 0) / (8 * 132 * 4)  # a single token: its keys are split
    assert parts == int(parts) and 16 <= parts <= 256
    assert need(1, 20000, 0, ns=_i32(0)) == 0
    assert swan.lib().swan_prompt_workspace_bytes(swan.SWAN_F16, 1, 8, 2, 1, 1, 128, None, None, 1,
                                                  None) == INVALID


# ---- swan_attend and decode behind a prefix ---------------------------------------------
def _desc(**kw):
    d = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, buffer_tokens=16,
             sparse_capacity=1000, dtype=swan.SWAN_F16, reserved=0,
             k_pages=FAKE, v_pages=FAKE, k_ring=FAKE, v_ring=FAKE)
    d.update(kw)
    return swan.CacheDesc(**d)


def _prefix(desc=None, lens=(300, 5), k=(32, 32), kv=None, of=(0, 1, -1)):
    arr = lambda v: None if v is None else ctypes.cast(_i32(*v), ctypes.POINTER(ctypes.c_int32))  # noqa: E731
    return swan.PrefixDesc(ctypes.pointer(desc or _desc()), arr(lens), arr(k), arr(kv), arr(of))


def _attend(sources, batch=3, n=4, ns=None, q=FAKE, P=FAKE, Pvo=None, scale=0.0, o=FAKE, lse=FAKE,
            ws=FAKE, size=BIG, count=None):
    arr = (swan.PrefixDesc * max(1, len(sources)))(*sources)
    return swan.lib().swan_attend(arr, len(sources) if count is None else count, batch, n, ns, q, P,
                                  Pvo, scale, o, lse, ws, size, None)


BAD_PREFIXES = [
    (dict(lens=None), INVALID), (dict(of=None), INVALID), (dict(k=None), INVALID),
    (dict(k=(32, 0)), INVALID), (dict(kv=(32, 129)), INVALID), (dict(lens=(-1, 5)), INVALID),
    (dict(lens=(1017, 5)), CAPACITY), (dict(of=(0, 2, 0)), INVALID), (dict(of=(-2, 0, 0)), INVALID),
    (dict(desc=_desc(head_dim=64)), UNSUPPORTED), (dict(desc=_desc(batch=0)), INVALID),
    (dict(desc=_desc(k_pages=None)), INVALID), (dict(desc=_desc(k_ring=FAKE + 4)), INVALID),
]


@pytest.mark.parametrize("kw,status", BAD_PREFIXES)
def test_attend_refuses_a_bad_source(kw, status):
    assert _attend([_prefix(**kw)]) == status and swan.last_error()
    assert _attend([_prefix(), _prefix(**kw)]) == status


@pytest.mark.parametrize("kw,status", [
    (dict(count=0), INVALID), (dict(count=3), INVALID), (dict(batch=0), INVALID),
    (dict(batch=65), INVALID), (dict(n=-1), INVALID), (dict(ns=_i32(1, 2, 5)), INVALID),
    (dict(q=None), INVALID), (dict(P=None), INVALID), (dict(o=None), INVALID),
    (dict(lse=None), INVALID), (dict(q=FAKE + 2), INVALID), (dict(Pvo=FAKE + 4), INVALID),
    (dict(scale=math.nan), INVALID), (dict(scale=1e-38), INVALID), (dict(ws=None), WORKSPACE),
    (dict(size=1000), WORKSPACE), (dict(ws=FAKE + 16), INVALID), (dict(n=2**28), UNSUPPORTED),
])
def test_attend_refuses(kw, status):
    assert _attend([_prefix()], **kw) == status and swan.last_error()


def test_attend_refuses_a_state_over_itself():
    assert _attend([_prefix()], o=FAKE, lse=FAKE + 3 * 8 * 4 * 512 - 4) == INVALID
    assert "overlap" in swan.last_error()


def test_attend_refuses_sources_that_differ():
    other = _desc(n_kv_heads=4)
    assert _attend([_prefix(), _prefix(desc=other)]) == INVALID
    assert _attend([_prefix(), _prefix(desc=_desc(dtype=swan.SWAN_F32))]) == INVALID


def test_attend_without_rows_is_fine():
    assert _attend([_prefix()], ns=_i32(0, 0, 0), q=None, P=None, o=None, lse=None, ws=None,
                   size=0) == swan.SWAN_OK


def _decode(prefix, desc=None, lens=(10, 20, 0), k=(32, 32, 32), step=False, ws=FAKE, size=BIG,
            new=FAKE, q=FAKE, scale=0.0):
    desc = desc or _desc(batch=3, k_pages=2 * FAKE, v_pages=2 * FAKE, k_ring=2 * FAKE, v_ring=2 * FAKE)
    head = (ctypes.byref(prefix), ctypes.byref(desc), None if lens is None else _i32(*lens),
            _i32(*k), None)
    tail = (q, FAKE, None, scale, FAKE, ws, size, None)
    if step:
        return swan.lib().swan_decode_step_prefix(*head, new, new, *tail)
    return swan.lib().swan_decode_attention_prefix(*head, *tail)


@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("kw,status", BAD_PREFIXES)
def test_decode_refuses_a_bad_prefix(kw, status, step):
    kw = dict(kw)
    assert _decode(_prefix(**kw), step=step, lens=(10, 20, 30)) == status and swan.last_error()


@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(lens=None), INVALID), (dict(lens=(-1, 5, 5)), INVALID), (dict(k=(0, 32, 32)), INVALID),
    (dict(lens=(10, 20, 2000)), CAPACITY), (dict(q=None), INVALID), (dict(scale=math.inf), INVALID),
    (dict(ws=None), WORKSPACE), (dict(size=4096), WORKSPACE), (dict(ws=FAKE + 64), INVALID),
    (dict(desc=_desc(batch=3, n_kv_heads=4)), INVALID),
    (dict(desc=_desc(batch=3, dtype=swan.SWAN_F32)), INVALID),
])
def test_decode_behind_a_prefix_refuses(kw, status, step):
    kw = dict(lens=(10, 20, 30)) | kw
    assert _decode(_prefix(), step=step, **kw) == status and swan.last_error()


def test_decode_wants_a_token_and_another_cache():
    assert _decode(_prefix(lens=(300, 5))) == INVALID  # sequence 2: no prefix, no own token
    assert "no token" in swan.last_error()
    assert _decode(_prefix(lens=(300, 0), of=(0, 1, 0)), lens=(1, 0, 1)) == INVALID
    same = _desc(batch=3)
    assert _decode(_prefix(desc=same, lens=(5, 5, 5), k=(32, 32, 32)), desc=same, step=True,
                   lens=(5, 5, 5)) == INVALID
    assert "appended" in swan.last_error()
    assert _decode(_prefix(), step=True, new=None, lens=(1, 1, 1)) == INVALID


def test_workspace_queries_refuse():
    out = ctypes.c_size_t()
    p, c = _prefix(), _desc(batch=3)
    lib = swan.lib()
    assert lib.swan_prefix_workspace_bytes(ctypes.byref(p), ctypes.byref(c), _i32(1, 1, 1),
                                           _i32(8, 8, 8), None, None) == INVALID
    assert lib.swan_prefix_workspace_bytes(None, ctypes.byref(c), _i32(1, 1, 1), _i32(8, 8, 8), None,
                                           ctypes.byref(out)) == INVALID
    assert lib.swan_attend_workspace_bytes(None, 1, 3, 4, None, ctypes.byref(out)) == INVALID
    arr = (swan.PrefixDesc * 1)(p)
    assert lib.swan_attend_workspace_bytes(arr, 1, 3, 4, None, None) == INVALID
    assert lib.swan_attend_workspace_bytes(arr, 1, 3, 4, None, ctypes.byref(out)) == swan.SWAN_OK
    assert out.value >= 3 * 8 * 4 * (128 + 132) * 4


# ---- the binding ------------------------------------------------------------------------
def test_the_binding_refuses_what_the_library_cannot_see():
    import torch

    x = torch.zeros(2, 3, 12 * 128, dtype=torch.float16)
    with pytest.raises(swan.SwanError, match="GPU"):
        swan.qkv_rows(x, 8, 2, [0, 0], 10000.0)
    with pytest.raises(swan.SwanError, match="elements"):
        swan.qkv_rows(x, 8, 4, [0, 0], 10000.0)
    with pytest.raises(swan.SwanError, match="dtype"):
        swan.qkv_rows(x.bfloat16(), 8, 2, [0, 0], 10000.0)
    with pytest.raises(swan.SwanError, match="qkv must be"):
        swan.qkv_rows(x[0], 8, 2, [0, 0], 10000.0)
    with pytest.raises(swan.SwanError, match="contiguous"):
        swan.qkv_rows(torch.zeros(2, 12 * 128, 3, dtype=torch.float16).transpose(1, 2), 8, 2, [0, 0],
                      10000.0)
    with pytest.raises(swan.SwanError, match="q_weight"):
        swan.qkv_rows(x, 8, 2, [0, 0], 10000.0, torch.ones(64, dtype=torch.float16))
    with pytest.raises(swan.SwanError, match="differ"):
        swan.qkv_rows(x, 8, 2, [0, 0], 10000.0, torch.ones(128, dtype=torch.float16),
                      torch.ones(128))
    q, k = torch.zeros(2, 8, 3, 128).half(), torch.zeros(2, 2, 3, 128).half()
    with pytest.raises(swan.SwanError, match="GPU"):
        swan.prompt_attention(q, k, k)
    with pytest.raises(swan.SwanError, match="shape"):
        swan.prompt_attention(q, k, k[:, :, :2])
    with pytest.raises(swan.SwanError, match="contiguous"):
        swan.prompt_attention(q.transpose(1, 2).contiguous().transpose(1, 2), k, k)
    with pytest.raises(swan.SwanError, match="dtype"):
        swan.prompt_attention(q, k, k.float())
    with pytest.raises(swan.SwanError, match="lse"):
        swan.prompt_attention(q, k, k, state=(torch.zeros(2, 8, 3, 128), torch.zeros(2, 8, 4)))
