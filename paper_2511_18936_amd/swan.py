"""ctypes binding of libswan (include/swan.h, include/swan_layer.h, include/swan_long.h), plus
a small cache holder.

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  PyTorch provides device memory and the current stream.  If the
library is missing the import fails loudly; there is no fallback.
"""
from __future__ import annotations

import copy
import ctypes
import math
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SWAN_LIB", os.path.join(_HERE, "libswan.so"))

SWAN_OK = 0
SWAN_ERR_INVALID_ARG = 1
SWAN_ERR_UNSUPPORTED = 2
SWAN_ERR_CAPACITY = 3
SWAN_ERR_WORKSPACE = 4
SWAN_ERR_HIP = 5
SWAN_ERR_NO_CONVERGENCE = 6
SWAN_F32 = 0
SWAN_F16 = 1
SWAN_F16_E4M3 = 2  # fp16 everywhere, sparse values as OCP FP8 E4M3
MAX_BATCH = 64
HEAD_DIM = 128
PAGE_TOKENS = 64

EXPORTED = (
    "swan_last_error", "swan_version", "swan_page_bytes", "swan_cache_bytes",
    "swan_calibrate_workspace_bytes", "swan_calibrate_rotation", "swan_compress_append",
    "swan_decode_workspace_bytes", "swan_decode_attention", "swan_decode_attention_noalloc",
    "swan_decode_step", "swan_change_k", "swan_rope", "swan_set_decode_tuning", "swan_set_profile_events",
)
NOALLOC_SCRATCH_BYTES = 16 << 20


class SwanError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"swan status {status}: {message}")
        self.status = status


class DecodeTuning(ctypes.Structure):
    _fields_ = [
        ("target_waves", ctypes.c_int32),
        ("short_split_pages", ctypes.c_int32),
        ("merge_pct", ctypes.c_int32),
        ("side_streams", ctypes.c_int32),
    ]


class CacheDesc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("buffer_tokens", ctypes.c_int32),
        ("sparse_capacity", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("k_pages", ctypes.c_void_p),
        ("v_pages", ctypes.c_void_p),
        ("k_ring", ctypes.c_void_p),
        ("v_ring", ctypes.c_void_p),
    ]


class PrefixDesc(ctypes.Structure):
    """swan_prefix: a cache, its lengths and k, and the sequence of it per query sequence."""
    _fields_ = [
        ("cache", ctypes.POINTER(CacheDesc)),
        ("seq_len_host", ctypes.POINTER(ctypes.c_int32)),
        ("k_active_host", ctypes.POINTER(ctypes.c_int32)),
        ("k_value_host", ctypes.POINTER(ctypes.c_int32)),
        ("of_host", ctypes.POINTER(ctypes.c_int32)),
    ]


class RotaryDesc(ctypes.Structure):
    """swan_rotary: dims turned, pairs of neighbours or not, magnitude, frequencies."""
    _fields_ = [
        ("dims", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
        ("magnitude", ctypes.c_double),
        ("freq_host", ctypes.POINTER(ctypes.c_double)),
    ]


def _load() -> ctypes.CDLL:
    # torch first: its HIP runtime (soname libamdhip64.so.7) then also serves
    # libswan, so the process holds a single runtime and a single device context
    import torch  # noqa: F401

    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"libswan.so not found at {LIB_PATH}; build it with "
            "`python -m paper_2511_18936_amd.build` (there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    i32, i64, sz, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p
    pi32, psz, pdesc = ctypes.POINTER(i32), ctypes.POINTER(sz), ctypes.POINTER(CacheDesc)
    pprefix, protary = ctypes.POINTER(PrefixDesc), ctypes.POINTER(RotaryDesc)
    lib.swan_last_error.restype = ctypes.c_char_p
    lib.swan_last_error.argtypes = []
    lib.swan_version.restype = i32
    lib.swan_version.argtypes = []
    sigs = {
        "swan_page_bytes": [i32, i32, psz],
        "swan_cache_bytes": [pdesc, pi32, pi32, psz, psz, psz],
        "swan_calibrate_workspace_bytes": [i32, psz],
        "swan_calibrate_rotation": [vp, i64, i32, vp, vp, vp, sz, vp],
        "swan_calibrate_rotations": [vp, i32, ctypes.POINTER(i64), i32, vp, vp, vp, sz, vp],
        "swan_compress_append": [pdesc, pi32, pi32, pi32, vp, vp, i32, pi32, vp, vp, vp],
        "swan_decode_workspace_bytes": [pdesc, pi32, pi32, pi32, psz],
        "swan_decode_attention": [pdesc, pi32, pi32, pi32, vp, vp, vp, ctypes.c_float, vp, vp, sz,
                                  vp],
        "swan_decode_attention_noalloc": [pdesc, pi32, pi32, pi32, vp, vp, vp, ctypes.c_float,
                                          vp, vp],
        "swan_decode_step": [pdesc, pi32, pi32, pi32, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp,
                             sz, vp],
        "swan_change_k": [pdesc, pi32, pi32, pdesc, pi32, pi32, pi32, vp],
        "swan_rope": [vp, vp, i32, i32, i32, i32, i32, pi32, ctypes.c_double, vp],
        "swan_qkv_rows": [vp, i64, i64, i32, i32, i32, i32, i32, i32, pi32, ctypes.c_double, vp,
                          vp, i32, i32, ctypes.c_double, vp, vp, vp, vp],
        "swan_attend_workspace_bytes": [pprefix, i32, i32, i32, pi32, psz],
        "swan_attend": [pprefix, i32, i32, i32, pi32, vp, vp, vp, ctypes.c_float, vp, vp, vp, sz,
                        vp],
        "swan_prompt_workspace_bytes": [i32, i32, i32, i32, i32, i32, i32, pi32, pi32, i32, psz],
        "swan_prompt_attention": [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, pi32, pi32, i32,
                                  ctypes.c_float, vp, vp, vp, vp, sz, vp],
        "swan_prefix_workspace_bytes": [pprefix, pdesc, pi32, pi32, pi32, psz],
        "swan_decode_attention_prefix": [pprefix, pdesc, pi32, pi32, pi32, vp, vp, vp,
                                         ctypes.c_float, vp, vp, sz, vp],
        "swan_decode_step_prefix": [pprefix, pdesc, pi32, pi32, pi32, vp, vp, vp, vp, vp,
                                    ctypes.c_float, vp, vp, sz, vp],
        "swan_rope_rotary": [vp, vp, i32, i32, i32, i32, i32, pi32, protary, vp],
        "swan_qkv_rows_rotary": [vp, i64, i64, i32, i32, i32, i32, i32, i32, pi32, protary, vp, vp,
                                 i32, i32, ctypes.c_double, vp, vp, vp, vp],
        "swan_prompt_window_workspace_bytes": [i32, i32, i32, i32, i32, i32, i32, pi32, pi32, i32,
                                               pi32, psz],
        "swan_prompt_attention_window": [vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, pi32, pi32,
                                         i32, pi32, ctypes.c_float, vp, vp, vp, vp, sz, vp],
        "swan_attend_window_workspace_bytes": [pprefix, i32, i32, i32, pi32, i32, i32, psz],
        "swan_attend_window": [pprefix, i32, i32, i32, pi32, i32, i32, vp, vp, vp, ctypes.c_float,
                               vp, vp, vp, sz, vp],
        "swan_decode_window_workspace_bytes": [pprefix, pdesc, pi32, pi32, pi32, i32, i32, psz],
        "swan_decode_attention_window": [pprefix, pdesc, pi32, pi32, pi32, i32, i32, vp, vp, vp,
                                         ctypes.c_float, vp, vp, sz, vp],
        "swan_decode_step_window": [pprefix, pdesc, pi32, pi32, pi32, i32, i32, vp, vp, vp, vp, vp,
                                    ctypes.c_float, vp, vp, sz, vp],
        "swan_copy_sequences": [pdesc, pi32, pi32, pi32, pdesc, pi32, pi32, pi32, pi32, pi32, vp],
        "swan_set_decode_tuning": [ctypes.POINTER(DecodeTuning)],
        "swan_set_profile_events": [vp, vp],
    }
    for name, args in sigs.items():
        f = getattr(lib, name)
        f.restype = i32
        f.argtypes = args
    return lib


_lib = _load()


def lib() -> ctypes.CDLL:
    return _lib


def last_error() -> str:
    return _lib.swan_last_error().decode()


def _check(status: int) -> None:
    if status != SWAN_OK:
        raise SwanError(status, last_error())


_I32_TYPES: dict = {}


def _i32_array(values: Sequence[int]):
    n = len(values)
    ty = _I32_TYPES.get(n)
    if ty is None:
        ty = _I32_TYPES[n] = ctypes.c_int32 * n
    return ty(*values)


def _opt_i32_array(values: Optional[Sequence[int]]):
    return None if values is None else _i32_array(values)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream, device_index: Optional[int] = None) -> Optional[int]:
    """The HIP stream handle: the given torch stream's, else the current stream of
    device_index (default: the current device)."""
    import torch

    if stream is not None:
        return stream.cuda_stream
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is not None:
        return raw(torch.cuda.current_device() if device_index is None else device_index)
    return torch.cuda.current_stream().cuda_stream


def _elem_torch_dtype(code: int):
    import torch

    return torch.float32 if code == SWAN_F32 else torch.float16


def _tensor(t, name: str, dtype, shape) -> None:
    """The library sees only a device pointer: check what it assumes about the
    tensor behind it (dtype, shape, dense row-major layout, a GPU) before the call.
    A None entry of `shape` matches any size."""
    if t is None:
        raise SwanError(SWAN_ERR_INVALID_ARG, f"{name} is None")
    if t.dtype != dtype:
        raise SwanError(SWAN_ERR_INVALID_ARG, f"{name} has dtype {t.dtype}, expected {dtype}")
    ts = tuple(t.shape)
    if ts != shape and (len(ts) != len(shape) or
                        any(w is not None and g != w for g, w in zip(ts, shape))):
        want = "x".join("*" if w is None else str(w) for w in shape)
        raise SwanError(SWAN_ERR_INVALID_ARG,
                        f"{name} has shape {ts}, expected [{want}]")
    if not t.is_contiguous():
        raise SwanError(SWAN_ERR_INVALID_ARG, f"{name} must be contiguous (row-major)")


def _on_gpu(**tensors) -> None:
    for name, t in tensors.items():
        if t is not None and not t.is_cuda:
            raise SwanError(SWAN_ERR_INVALID_ARG, f"{name} is on {t.device}, not on a GPU")


def _rotations(desc: CacheDesc, P_qk, P_vo) -> None:
    import torch

    shape = (desc.n_kv_heads, desc.head_dim, desc.head_dim)
    _tensor(P_qk, "P_qk", torch.float32, shape)
    if P_vo is not None:
        _tensor(P_vo, "P_vo", torch.float32, shape)


def dtype_code(torch_dtype, sparse_values: str = "same") -> int:
    import torch

    if sparse_values not in ("same", "e4m3"):
        raise SwanError(SWAN_ERR_INVALID_ARG, f"sparse_values {sparse_values!r}")
    if sparse_values == "e4m3":
        if torch_dtype != torch.float16:
            raise SwanError(SWAN_ERR_UNSUPPORTED, "E4M3 sparse values need float16 storage")
        return SWAN_F16_E4M3
    if torch_dtype == torch.float16:
        return SWAN_F16
    if torch_dtype == torch.float32:
        return SWAN_F32
    raise SwanError(SWAN_ERR_UNSUPPORTED, f"dtype {torch_dtype} not supported")


def page_bytes(dtype: int, k_active: int) -> int:
    out = ctypes.c_size_t()
    _check(_lib.swan_page_bytes(dtype, k_active, ctypes.byref(out)))
    return out.value


def cache_bytes(desc: CacheDesc, k_active: Sequence[int],
                k_value: Optional[Sequence[int]] = None):
    """(key page bytes, value page bytes, ring bytes); k_value None: as k_active."""
    kb, vb, rb = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check(_lib.swan_cache_bytes(ctypes.byref(desc), _i32_array(k_active),
                                 _opt_i32_array(k_value), ctypes.byref(kb), ctypes.byref(vb),
                                 ctypes.byref(rb)))
    return kb.value, vb.value, rb.value


def calibrate_workspace_bytes(d: int = HEAD_DIM) -> int:
    out = ctypes.c_size_t()
    _check(_lib.swan_calibrate_workspace_bytes(d, ctypes.byref(out)))
    return out.value


def calibrate_rotation(rows, P_out, sigma_out=None, workspace=None, stream=None) -> None:
    """Sec. 4.1.2 basis of `rows` ([n][d] float32, cuda) into P_out ([d][d] float32)."""
    n, d = rows.shape
    if workspace is None:
        workspace = _made("empty", (calibrate_workspace_bytes(d),), "uint8", rows.device, stream)
    _check(_lib.swan_calibrate_rotation(_ptr(rows), n, d, _ptr(P_out), _ptr(sigma_out),
                                        _ptr(workspace), workspace.numel(), _stream(stream)))


def calibrate_rotations(rows, n_rows: Sequence[int], P_out, sigma_out=None, workspace=None,
                        stream=None) -> None:
    """calibrate_rotation of several problems at once: `rows` ([sum(n_rows)][d] float32,
    cuda) holds n_rows[i] rows of problem i, one problem after another; into P_out
    ([len(n_rows)][d][d] float32)."""
    import torch

    count, d = len(n_rows), rows.shape[1]
    _tensor(rows, "rows", torch.float32, (sum(n_rows), d))
    _tensor(P_out, "P_out", torch.float32, (count, d, d))
    if sigma_out is not None:
        _tensor(sigma_out, "sigma_out", torch.float32, (count, d))
    _on_gpu(rows=rows, P_out=P_out, sigma_out=sigma_out)
    if workspace is None:
        workspace = _made("empty", (count * calibrate_workspace_bytes(d),), "uint8", rows.device,
                          stream)
    _check(_lib.swan_calibrate_rotations(_ptr(rows), count, (ctypes.c_int64 * count)(*n_rows), d,
                                         _ptr(P_out), _ptr(sigma_out), _ptr(workspace),
                                         workspace.numel(), _stream(stream, rows.get_device())))


def compress_append(desc: CacheDesc, seq_len: Sequence[int], k_active: Sequence[int], k_new,
                    v_new, P_qk, P_vo, n_new_per_seq: Optional[Sequence[int]] = None,
                    stream=None, k_value: Optional[Sequence[int]] = None) -> None:
    n_new = 0 if k_new is None else int(k_new.shape[2])
    if k_new is not None or v_new is not None:
        et = _elem_torch_dtype(desc.dtype)
        shape = (desc.batch, desc.n_kv_heads, n_new, desc.head_dim)
        _tensor(k_new, "k_new", et, shape)
        _tensor(v_new, "v_new", et, shape)
    _rotations(desc, P_qk, P_vo)
    _on_gpu(k_new=k_new, v_new=v_new, P_qk=P_qk, P_vo=P_vo)
    per = None if n_new_per_seq is None else _i32_array(n_new_per_seq)
    _check(_lib.swan_compress_append(ctypes.byref(desc), _i32_array(seq_len),
                                     _i32_array(k_active), _opt_i32_array(k_value), _ptr(k_new),
                                     _ptr(v_new), n_new, per, _ptr(P_qk), _ptr(P_vo),
                                     _stream(stream, P_qk.get_device())))


def decode_workspace_bytes(desc: CacheDesc, seq_len: Sequence[int], k_active: Sequence[int],
                           k_value: Optional[Sequence[int]] = None) -> int:
    out = ctypes.c_size_t()
    _check(_lib.swan_decode_workspace_bytes(ctypes.byref(desc), _i32_array(seq_len),
                                            _i32_array(k_active), _opt_i32_array(k_value),
                                            ctypes.byref(out)))
    return out.value


def decode_attention(desc: CacheDesc, seq_len: Sequence[int], k_active: Sequence[int], q,
                     P_qk, P_vo, out, workspace, scale: float = 0.0, stream=None,
                     k_value: Optional[Sequence[int]] = None) -> None:
    _decode_tensors(desc, q, P_qk, P_vo, out)
    if workspace is None or not workspace.is_cuda or not workspace.is_contiguous():
        raise SwanError(SWAN_ERR_WORKSPACE, "workspace must be a contiguous GPU tensor")
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(_lib.swan_decode_attention(ctypes.byref(desc), _i32_array(seq_len),
                                      _i32_array(k_active), _opt_i32_array(k_value), _ptr(q),
                                      _ptr(P_qk), _ptr(P_vo), float(scale), _ptr(out),
                                      _ptr(workspace), ws_bytes, _stream(stream, q.get_device())))


def _decode_tensors(desc: CacheDesc, q, P_qk, P_vo, out) -> None:
    et = _elem_torch_dtype(desc.dtype)
    shape = (desc.batch, desc.n_q_heads, desc.head_dim)
    _tensor(q, "q", et, shape)
    _tensor(out, "out", et, shape)
    _rotations(desc, P_qk, P_vo)
    _on_gpu(q=q, out=out, P_qk=P_qk, P_vo=P_vo)


def decode_attention_noalloc(desc: CacheDesc, seq_len: Sequence[int], k_active: Sequence[int],
                             q, P_qk, P_vo, out, scale: float = 0.0, stream=None,
                             k_value: Optional[Sequence[int]] = None) -> None:
    """swan_decode_attention with the library's own scratch instead of a workspace."""
    _decode_tensors(desc, q, P_qk, P_vo, out)
    _check(_lib.swan_decode_attention_noalloc(ctypes.byref(desc), _i32_array(seq_len),
                                              _i32_array(k_active), _opt_i32_array(k_value),
                                              _ptr(q), _ptr(P_qk), _ptr(P_vo), float(scale),
                                              _ptr(out), _stream(stream, q.get_device())))


def decode_step(desc: CacheDesc, seq_len: Sequence[int], k_active: Sequence[int], k_new, v_new,
                q, P_qk, P_vo, out, workspace, scale: float = 0.0, stream=None,
                k_value: Optional[Sequence[int]] = None) -> None:
    """swan_decode_step: append one token per sequence (seq_len: lengths before it), then
    decode q over the cache with it; workspace sized for the lengths after the step."""
    et = _elem_torch_dtype(desc.dtype)
    shape = (desc.batch, desc.n_kv_heads, 1, desc.head_dim)
    _tensor(k_new, "k_new", et, shape)
    _tensor(v_new, "v_new", et, shape)
    _decode_tensors(desc, q, P_qk, P_vo, out)
    _on_gpu(k_new=k_new, v_new=v_new)
    if workspace is None or not workspace.is_cuda or not workspace.is_contiguous():
        raise SwanError(SWAN_ERR_WORKSPACE, "workspace must be a contiguous GPU tensor")
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(_lib.swan_decode_step(ctypes.byref(desc), _i32_array(seq_len), _i32_array(k_active),
                                 _opt_i32_array(k_value), _ptr(k_new), _ptr(v_new), _ptr(q),
                                 _ptr(P_qk), _ptr(P_vo), float(scale), _ptr(out),
                                 _ptr(workspace), ws_bytes, _stream(stream, q.get_device())))


def change_k(src: CacheDesc, k_active_src: Sequence[int], k_value_src: Optional[Sequence[int]],
             dst: CacheDesc, k_active_dst: Sequence[int], k_value_dst: Optional[Sequence[int]],
             seq_len: Sequence[int], stream=None) -> None:
    """Lay src's sparse caches out again in dst for the new k (see swan_change_k)."""
    _check(_lib.swan_change_k(ctypes.byref(src), _i32_array(k_active_src),
                              _opt_i32_array(k_value_src), ctypes.byref(dst),
                              _i32_array(k_active_dst), _opt_i32_array(k_value_dst),
                              _i32_array(seq_len), _stream(stream)))


class Rotary:
    """How rows are turned to their positions: of a head's first `dims` dims (a multiple of 8)
    dims j and j + dims/2 are pair j, or with interleaved=True dims 2j and 2j + 1; a pair turns
    by pos * freqs[j] (None: base^(-2j/dims)) and is multiplied by `magnitude`.  The other dims
    stay as they are.  Taken by rope, qkv_rows and the layer in the place of a base."""

    def __init__(self, base: float = 10000.0, dims: int = HEAD_DIM, interleaved: bool = False,
                 freqs: Optional[Sequence[float]] = None, magnitude: float = 1.0):
        self.dims, self.interleaved = int(dims), bool(interleaved)
        self.magnitude = float(magnitude)
        if self.dims < 8 or self.dims > HEAD_DIM or self.dims % 8:
            raise SwanError(SWAN_ERR_INVALID_ARG,
                            f"dims {dims}: a multiple of 8 within 8..{HEAD_DIM}")
        if not self.magnitude > 0 or math.isinf(self.magnitude):
            raise SwanError(SWAN_ERR_INVALID_ARG, f"magnitude {magnitude}")
        half = self.dims // 2
        if freqs is None:
            if not base > 1 or math.isinf(base):
                raise SwanError(SWAN_ERR_INVALID_ARG, f"base {base} must be > 1")
            freqs = [float(base) ** (-j / half) for j in range(half)]
        freqs = [float(f) for f in freqs]
        if len(freqs) != half or not all(math.isfinite(f) for f in freqs):
            raise SwanError(SWAN_ERR_INVALID_ARG, f"freqs must be {half} finite numbers")
        self.freqs = tuple(freqs)
        self._freqs = (ctypes.c_double * half)(*freqs)
        self._desc = RotaryDesc(self.dims, int(self.interleaved), self.magnitude, self._freqs)

    def stretched(self, factor: float) -> "Rotary":
        """Positions interpolated: every frequency divided by `factor`."""
        self._check_factor(factor)
        return self._with([f / factor for f in self.freqs], self.magnitude)

    def by_parts(self, factor: float, original: int, low: float = 1.0, high: float = 32.0,
                 magnitude: Optional[float] = None) -> "Rotary":
        """Stretched to `factor` times the `original` context by parts: frequencies that turn
        fewer than `low` times in it are divided by `factor`, those that turn more than `high`
        times stay, those between are mixed linearly in their turns.  magnitude: what the
        present one is multiplied by (None: 0.1 ln(factor) + 1)."""
        self._check_factor(factor)
        if not 0 < low < high:
            raise SwanError(SWAN_ERR_INVALID_ARG, f"low {low} and high {high}: 0 < low < high")
        if not original > 0 or math.isinf(original):
            raise SwanError(SWAN_ERR_INVALID_ARG, f"original {original} must be finite, > 0")
        if magnitude is None:
            magnitude = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
        freqs = []
        for f in self.freqs:
            keep = min(1.0, max(0.0, (original * f / (2 * math.pi) - low) / (high - low)))
            freqs.append(keep * f + (1 - keep) * f / factor)
        return self._with(freqs, self.magnitude * magnitude)

    @staticmethod
    def _check_factor(factor: float) -> None:
        if not factor > 0 or math.isinf(factor):
            raise SwanError(SWAN_ERR_INVALID_ARG, f"factor {factor} must be finite, > 0")

    def _with(self, freqs, magnitude: float) -> "Rotary":
        return Rotary(dims=self.dims, interleaved=self.interleaved, freqs=freqs,
                      magnitude=magnitude)


def rope(x, pos0: Sequence[int], base, out=None, stream=None):
    """RoPE of rows x [B][H][n][128] (float16 or float32, cuda) at positions pos0[b] + i;
    out=None writes a new tensor, out=x works in place.  base: a number (dims j and j + 64 of
    the whole head, base^(-2j/128)), or a Rotary."""
    import torch

    if isinstance(base, Rotary):
        return _rope_rotary(x, pos0, base, out, stream)
    if out is None:
        out = torch.empty_like(x) if stream is None else _result_like(x, x.shape, stream)
    B, H, n, d = x.shape
    code = SWAN_F16 if x.dtype == torch.float16 else SWAN_F32
    _check(_lib.swan_rope(_ptr(x), _ptr(out), code, B, H, n, d, _i32_array(pos0), float(base),
                          _stream(stream)))
    return out


def _rope_rotary(x, pos0: Sequence[int], rotary: Rotary, out, stream):
    if x.dim() != 4:
        raise SwanError(SWAN_ERR_INVALID_ARG, "x must be [B][H][n][128]")
    code = _storage_code(x.dtype)
    B, H, n, d = x.shape
    _tensor(x, "x", x.dtype, (B, H, n, HEAD_DIM))
    _on_gpu(x=x)
    if out is None:
        out = _result_like(x, x.shape, stream)
    _tensor(out, "out", x.dtype, (B, H, n, HEAD_DIM))
    if out is not x and out.data_ptr() != x.data_ptr() and _share(x, out):
        raise SwanError(SWAN_ERR_INVALID_ARG, "out overlaps x without being it")
    with _CallsOn(_same_gpu(x=x, out=out), stream) as s:
        _check(_lib.swan_rope_rotary(_ptr(x), _ptr(out), code, B, H, n, d,
                                     _per_sequence(pos0, B, "pos0"), ctypes.byref(rotary._desc),
                                     s))
    return out


def _share(a, b) -> bool:
    """Whether two contiguous tensors share a byte."""
    a0, b0 = a.data_ptr(), b.data_ptr()
    return (a0 < b0 + b.numel() * b.element_size() and b0 < a0 + a.numel() * a.element_size())


def _same_gpu(**tensors):
    """The one GPU that all the tensors (None left out) are on."""
    _on_gpu(**tensors)
    device = None
    for name, t in tensors.items():
        if t is None:
            continue
        device = t.device if device is None else device
        if t.device != device:
            raise SwanError(SWAN_ERR_INVALID_ARG, f"{name} is on {t.device}, not on {device}")
    return device


class _CallsOn:
    """Makes `device` current where it is not: a call is enqueued on a stream of the
    current device.  Gives the stream's handle."""

    def __init__(self, device, stream):
        self.index, self.stream, self.guard = device.index, stream, None

    def __enter__(self):
        import torch

        if self.index != torch.cuda.current_device():
            self.guard = torch.cuda.device(self.index)
            self.guard.__enter__()
        return _stream(self.stream, self.index)

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _per_sequence(values: Optional[Sequence[int]], batch: int, name: str):
    if values is not None and len(values) != batch:
        raise SwanError(SWAN_ERR_INVALID_ARG,
                        f"{name} has {len(values)} entries for {batch} sequences")
    return _opt_i32_array(values)


def _storage_code(dtype) -> int:
    import torch

    if dtype not in (torch.float16, torch.float32):
        raise SwanError(SWAN_ERR_UNSUPPORTED, f"dtype {dtype} not supported")
    return SWAN_F16 if dtype == torch.float16 else SWAN_F32


def _workspace(workspace, need: int, device, stream):
    """`workspace`, or `need` bytes of the caching allocator for work on `stream`."""
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise SwanError(SWAN_ERR_WORKSPACE, "workspace must be a contiguous GPU tensor")
        if workspace.device != device:
            raise SwanError(SWAN_ERR_WORKSPACE,
                            f"workspace is on {workspace.device}, not on {device}")
        return workspace
    return _made("empty", (max(need, 16),), "uint8", device, stream)


def _made(how: str, shape, dtype, device, stream):
    """torch.empty or torch.zeros, on the stream that the call is enqueued on (memory of
    another stream's could still be in use there)."""
    import torch

    dtype = getattr(torch, dtype) if isinstance(dtype, str) else dtype
    make = getattr(torch, how)
    if stream is None:
        return make(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return make(shape, dtype=dtype, device=device)


def _result(how: str, shape, dtype, device, stream):
    """_made() for what a call returns: the caller may use it on the current stream and drop
    it, so a block of another stream's is not used again before that work is done."""
    import torch

    t = _made(how, shape, dtype, device, stream)
    if stream is not None and t.is_cuda:
        current = torch.cuda.current_stream(t.device)
        if current != stream:
            t.record_stream(current)
    return t


def _result_like(t, shape, stream):
    """An empty result of t's type beside it."""
    return t.new_empty(shape) if stream is None else _result("empty", shape, t.dtype, t.device, stream)


def qkv_rows(qkv, n_q_heads: int, n_kv_heads: int, pos0: Sequence[int], base,
             q_weight=None, k_weight=None, eps: float = 1e-6, out=None, stream=None):
    """A layer's projections qkv [B][n][(n_q + 2 n_kv) * 128] (float16 or float32, cuda; rows
    may be strided) as q [B][n_q][n][128], k and v [B][n_kv][n][128]: q and k divided by
    their root mean square and weighted (q_weight / k_weight: [128], or [heads][128], of
    qkv's type or float32; None: no norm), then rotated to positions pos0[b] + i as by
    rope() (base: a number or a Rotary); v as it is.  out = (q, k, v) writes existing tensors; n_q_heads = 0 gives
    (None, k, v)."""
    if qkv.dim() != 3:
        raise SwanError(SWAN_ERR_INVALID_ARG, "qkv must be [B][n][(n_q + 2 n_kv) * 128]")
    dtype = qkv.dtype
    code = _storage_code(dtype)
    B, n, width = qkv.shape
    if width != (n_q_heads + 2 * n_kv_heads) * HEAD_DIM or n_q_heads < 0 or n_kv_heads < 0:
        raise SwanError(SWAN_ERR_INVALID_ARG,
                        f"rows of {width} elements for {n_q_heads} + 2 x {n_kv_heads} heads")
    seq, row, last = qkv.stride()
    if last != 1 and width > 1:
        raise SwanError(SWAN_ERR_INVALID_ARG, "qkv's last dimension must be contiguous")
    per_head = w32 = False
    if q_weight is not None or k_weight is not None:
        w32, per_head = _norm_weights(dtype, n_q_heads, n_kv_heads, q_weight, k_weight)
    if not qkv.is_cuda:
        raise SwanError(SWAN_ERR_INVALID_ARG, f"qkv is on {qkv.device}, not on a GPU")
    if out is None:
        q = k = v = None
        if n_q_heads:
            q = _result_like(qkv, (B, n_q_heads, n, HEAD_DIM), stream)
        if n_kv_heads:
            k = _result_like(qkv, (B, n_kv_heads, n, HEAD_DIM), stream)
            v = _result_like(qkv, (B, n_kv_heads, n, HEAD_DIM), stream)
        device = _same_gpu(qkv=qkv, q_weight=q_weight, k_weight=k_weight)
    else:
        q, k, v = out
        for name, t, heads in (("q", q, n_q_heads), ("k", k, n_kv_heads), ("v", v, n_kv_heads)):
            if heads:
                _tensor(t, name, dtype, (B, heads, n, HEAD_DIM))
        device = _same_gpu(qkv=qkv, q=q, k=k, v=v, q_weight=q_weight, k_weight=k_weight)
    # (a dimension of one element has no stride of its own)
    with _CallsOn(device, stream) as s:
        call, how = _lib.swan_qkv_rows, base
        if isinstance(base, Rotary):
            call, how = _lib.swan_qkv_rows_rotary, ctypes.byref(base._desc)
        _check(call(_ptr(qkv), seq if B > 1 else 0, row if n > 1 else width, code, B, n_q_heads,
                    n_kv_heads, n, HEAD_DIM, _per_sequence(pos0, B, "pos0"), how, _ptr(q_weight),
                    _ptr(k_weight), per_head, w32, eps, _ptr(q), _ptr(k), _ptr(v), s))
    return q, k, v


def _norm_weights(dtype, n_q_heads: int, n_kv_heads: int, q_weight, k_weight):
    """(float32 weights, weights per head) of the norm weights given, checked."""
    import torch

    form = None
    for name, w, heads in (("q_weight", q_weight, n_q_heads), ("k_weight", k_weight, n_kv_heads)):
        if w is None:
            continue
        if w.dtype != dtype and w.dtype != torch.float32:
            raise SwanError(SWAN_ERR_INVALID_ARG,
                            f"{name} has dtype {w.dtype}, expected {dtype} or float32")
        two = w.dim() == 2
        _tensor(w, name, w.dtype, (heads, HEAD_DIM) if two else (HEAD_DIM,))
        if form is not None and form != (w.dtype == torch.float32, two):
            raise SwanError(SWAN_ERR_INVALID_ARG, "q_weight and k_weight differ in form")
        form = (w.dtype == torch.float32, two)
    return form


def prompt_attention(q, k, v, causal: bool = True, n: Optional[Sequence[int]] = None,
                     m: Optional[Sequence[int]] = None, scale: float = 0.0, state=None, out=None,
                     workspace=None, stream=None, window: Optional[int] = None, sinks=0):
    """Dense attention of rows q [B][H_q][n][128] over k, v [B][H_kv][m][128] (float16 or
    float32, cuda): a prompt's (causal: row i sees keys j <= i + m_b - n_b) or rows over
    another sequence's keys and values (causal=False).  n / m: the rows used of each
    sequence (None: all); the others are not read, and out's rows past n_b not written
    (zeros where out is None).  state: what SwanCache.attend or attend returned for these
    rows, to continue from.  window (causal only): a row sees the last `window` keys up to
    itself, and the first `sinks` (a number, or one per sequence; behind cached tokens what
    those leave of them: max(0, sinks - cached tokens))."""
    _window(window, sinks)
    if window is not None and not causal:
        raise SwanError(SWAN_ERR_INVALID_ARG, "a window needs causal=True")
    if q.dim() != 4 or k.dim() != 4:
        raise SwanError(SWAN_ERR_INVALID_ARG, "q, k and v must be [B][heads][rows][128]")
    code = _storage_code(q.dtype)
    B, hq, nq, d = q.shape
    hkv, nk = int(k.shape[1]), int(k.shape[2])
    _tensor(q, "q", q.dtype, (B, hq, nq, HEAD_DIM))
    _tensor(k, "k", q.dtype, (B, hkv, nk, HEAD_DIM))
    _tensor(v, "v", q.dtype, (B, hkv, nk, HEAD_DIM))
    o0, lse0 = _state(state, B, hq, nq)
    if out is None:
        _same_gpu(q=q)
        out = _result("empty" if n is None else "zeros", q.shape, q.dtype, q.device, stream)
    _tensor(out, "out", q.dtype, (B, hq, nq, HEAD_DIM))
    device = _same_gpu(q=q, k=k, v=v, out=out, o=o0, lse=lse0)
    ns, ms = _per_sequence(n, B, "n"), _per_sequence(m, B, "m")
    need = ctypes.c_size_t()
    bytes_of, call, how = _lib.swan_prompt_workspace_bytes, _lib.swan_prompt_attention, ()
    if window is None:
        how = (int(causal),)
    else:
        bytes_of = _lib.swan_prompt_window_workspace_bytes
        call = _lib.swan_prompt_attention_window
        first = [sinks] * B if isinstance(sinks, int) else sinks
        how = (window, _per_sequence(first, B, "sinks"))
    _check(bytes_of(code, B, hq, hkv, nq, nk, d, ns, ms, *how, ctypes.byref(need)))
    ws = None
    if need.value:
        ws = _workspace(workspace, need.value, device, stream)
    with _CallsOn(device, stream) as s:
        _check(call(_ptr(q), _ptr(k), _ptr(v), code, B, hq, hkv, nq, nk, d, ns, ms, *how,
                    float(scale), _ptr(o0), _ptr(lse0), _ptr(out), _ptr(ws),
                    0 if ws is None else ws.numel() * ws.element_size(), s))
    return out


def _window(window, sinks, one: bool = False) -> None:
    """Checks of a window and its first keys (one: a number of them, for all sequences)."""
    if one and not isinstance(sinks, int):
        raise SwanError(SWAN_ERR_INVALID_ARG, f"sinks must be one number here, not {sinks}")
    if window is None and (not isinstance(sinks, int) or sinks != 0):
        raise SwanError(SWAN_ERR_INVALID_ARG, "sinks without a window")
    for x in (window, sinks):
        if isinstance(x, (bool, float)):
            raise SwanError(SWAN_ERR_INVALID_ARG, f"window and sinks are whole numbers, not {x}")
    # (ctypes would take the low 32 bits of numbers outside)
    first = [sinks] if isinstance(sinks, int) else sinks
    if window is not None and not 1 <= window < 2**31 or any(not 0 <= x < 2**31 for x in first):
        raise SwanError(SWAN_ERR_INVALID_ARG, f"window {window} or sinks {sinks} out of range")


def _state(state, B: int, heads: int, n: int):
    import torch

    if state is None:
        return None, None
    o, lse = state
    _tensor(o, "state o", torch.float32, (B, heads, n, HEAD_DIM))
    _tensor(lse, "state lse", torch.float32, (B, heads, n))
    return o, lse


class Prefix:
    """Cached tokens that the sequences of a batch share: query sequence b attends to the
    tokens of sequence of[b] of `cache` (-1: none; of=None: sequence 0, for all) before its
    own.  It only refers to the cache: tokens appended to that later belong to the prefix."""

    def __init__(self, cache: "SwanCache", of: Optional[Sequence[int]] = None):
        self.cache = cache
        self.of = None if of is None else [int(x) for x in of]

    def _desc(self, batch: int):
        c = self.cache
        of = [0] * batch if self.of is None else self.of
        if len(of) != batch:
            raise SwanError(SWAN_ERR_INVALID_ARG,
                            f"the prefix is for {len(of)} sequences, not {batch}")
        return PrefixDesc(ctypes.pointer(c.desc), _i32_array(c.seq_len), _i32_array(c.k_active),
                          _opt_i32_array(c.k_value), _i32_array(of))


def attend(sources, q, P_qk, P_vo, n: Optional[Sequence[int]] = None, scale: float = 0.0,
           out=None, workspace=None, stream=None, window: Optional[int] = None, sinks: int = 0):
    """Rows q [B][H_q][n][128] over all cached tokens of one or two sources (Prefix objects:
    a shared prefix, the sequences' own caches), none masked: the state (o [B][H_q][n][128],
    lse [B][H_q][n]) in float32 that prompt_attention continues from.  n: the rows used of
    each sequence (None: all); the others are not read, and not written (zeros where out
    is None).  P_vo None leaves o rotated.  window: row i, standing i positions behind the
    cached tokens, sees those of the last `window` positions up to itself, and the first
    `sinks`."""
    _window(window, sinks, True)
    sources = list(sources)
    if not sources:
        raise SwanError(SWAN_ERR_INVALID_ARG, "no sources")
    c = sources[0].cache
    if q.dim() != 4:
        raise SwanError(SWAN_ERR_INVALID_ARG, "q must be [B][H_q][n][128]")
    B, nq = int(q.shape[0]), int(q.shape[2])
    hq = c.desc.n_q_heads
    _tensor(q, "q", _elem_torch_dtype(c.desc.dtype), (B, hq, nq, HEAD_DIM))
    _rotations(c.desc, P_qk, P_vo)
    if out is None:
        _same_gpu(q=q)
        how = "empty" if n is None else "zeros"
        out = (_result(how, (B, hq, nq, HEAD_DIM), "float32", q.device, stream),
               _result(how, (B, hq, nq), "float32", q.device, stream))
    o, lse = _state(out, B, hq, nq)
    pages = {f"source {i}": s.cache.k_pages for i, s in enumerate(sources)}
    device = _same_gpu(q=q, P_qk=P_qk, P_vo=P_vo, o=o, lse=lse, **pages)
    descs = (PrefixDesc * len(sources))(*[s._desc(B) for s in sources])
    ns = _per_sequence(n, B, "n")
    need = ctypes.c_size_t()
    bytes_of, call, how = _lib.swan_attend_workspace_bytes, _lib.swan_attend, ()
    if window is not None:
        bytes_of, call = _lib.swan_attend_window_workspace_bytes, _lib.swan_attend_window
        how = (window, sinks)
    _check(bytes_of(descs, len(sources), B, nq, ns, *how, ctypes.byref(need)))
    ws = _workspace(workspace, need.value, device, stream)
    with _CallsOn(device, stream) as s:
        _check(call(descs, len(sources), B, nq, ns, *how, _ptr(q), _ptr(P_qk), _ptr(P_vo),
                    float(scale), _ptr(o), _ptr(lse), _ptr(ws), ws.numel() * ws.element_size(), s))
    return o, lse


def decode_attention_prefix(prefix: Prefix, desc: CacheDesc, seq_len: Sequence[int],
                            k_active: Sequence[int], q, P_qk, P_vo, out, workspace,
                            scale: float = 0.0, stream=None,
                            k_value: Optional[Sequence[int]] = None) -> None:
    """swan_decode_attention_prefix: decode_attention with a prefix before each sequence's
    own tokens."""
    _decode_tensors(desc, q, P_qk, P_vo, out)
    device = _same_gpu(q=q, out=out, P_qk=P_qk, P_vo=P_vo, workspace=workspace,
                       prefix=prefix.cache.k_pages)
    if workspace is None or not workspace.is_contiguous():
        raise SwanError(SWAN_ERR_WORKSPACE, "workspace must be a contiguous GPU tensor")
    p = prefix._desc(desc.batch)
    with _CallsOn(device, stream) as s:
        _check(_lib.swan_decode_attention_prefix(
            ctypes.byref(p), ctypes.byref(desc), _i32_array(seq_len), _i32_array(k_active),
            _opt_i32_array(k_value), _ptr(q), _ptr(P_qk), _ptr(P_vo), float(scale), _ptr(out),
            _ptr(workspace), workspace.numel() * workspace.element_size(),
            s))


def decode_step_prefix(prefix: Prefix, desc: CacheDesc, seq_len: Sequence[int],
                       k_active: Sequence[int], k_new, v_new, q, P_qk, P_vo, out, workspace,
                       scale: float = 0.0, stream=None,
                       k_value: Optional[Sequence[int]] = None) -> None:
    """swan_decode_step_prefix: decode_step with a prefix before each sequence's own tokens."""
    et = _elem_torch_dtype(desc.dtype)
    shape = (desc.batch, desc.n_kv_heads, 1, desc.head_dim)
    _tensor(k_new, "k_new", et, shape)
    _tensor(v_new, "v_new", et, shape)
    _decode_tensors(desc, q, P_qk, P_vo, out)
    device = _same_gpu(q=q, k_new=k_new, v_new=v_new, out=out, P_qk=P_qk, P_vo=P_vo,
                       workspace=workspace, prefix=prefix.cache.k_pages)
    if workspace is None or not workspace.is_contiguous():
        raise SwanError(SWAN_ERR_WORKSPACE, "workspace must be a contiguous GPU tensor")
    p = prefix._desc(desc.batch)
    with _CallsOn(device, stream) as s:
        _check(_lib.swan_decode_step_prefix(
            ctypes.byref(p), ctypes.byref(desc), _i32_array(seq_len), _i32_array(k_active),
            _opt_i32_array(k_value), _ptr(k_new), _ptr(v_new), _ptr(q), _ptr(P_qk), _ptr(P_vo),
            float(scale), _ptr(out), _ptr(workspace),
            workspace.numel() * workspace.element_size(), s))


def prefix_workspace_bytes(prefix: Prefix, desc: CacheDesc, seq_len: Sequence[int],
                           k_active: Sequence[int],
                           k_value: Optional[Sequence[int]] = None) -> int:
    out = ctypes.c_size_t()
    p = prefix._desc(desc.batch)
    _check(_lib.swan_prefix_workspace_bytes(ctypes.byref(p), ctypes.byref(desc),
                                            _i32_array(seq_len), _i32_array(k_active),
                                            _opt_i32_array(k_value), ctypes.byref(out)))
    return out.value


def _window_head(desc: CacheDesc, seq_len, k_active, k_value, prefix, window, sinks):
    """The arguments that a windowed decode call and its workspace query share."""
    _window(window, sinks, True)
    if window is None:
        raise SwanError(SWAN_ERR_INVALID_ARG, "window is None")
    B = desc.batch
    return (None if prefix is None else ctypes.byref(prefix._desc(B)), ctypes.byref(desc),
            _per_sequence(seq_len, B, "seq_len"), _per_sequence(k_active, B, "k_active"),
            _per_sequence(k_value, B, "k_value"), window, sinks)


def decode_window_workspace_bytes(desc: CacheDesc, seq_len: Sequence[int],
                                  k_active: Sequence[int], window: int, sinks: int = 0,
                                  k_value: Optional[Sequence[int]] = None,
                                  prefix: Optional[Prefix] = None) -> int:
    out = ctypes.c_size_t()
    _check(_lib.swan_decode_window_workspace_bytes(
        *_window_head(desc, seq_len, k_active, k_value, prefix, window, sinks),
        ctypes.byref(out)))
    return out.value


def decode_window(desc: CacheDesc, seq_len: Sequence[int], k_active: Sequence[int], q, P_qk, P_vo,
                  out, workspace, window: int, sinks: int = 0, scale: float = 0.0, stream=None,
                  k_value: Optional[Sequence[int]] = None, prefix: Optional[Prefix] = None,
                  new=None) -> None:
    """swan_decode_attention_window, or with new = (k_new, v_new) swan_decode_step_window
    (seq_len: lengths before it), behind a prefix where one is given.  workspace None: the
    caching allocator's memory for this call."""
    head = _window_head(desc, seq_len, k_active, k_value, prefix, window, sinks)
    _decode_tensors(desc, q, P_qk, P_vo, out)
    k_new, v_new = new or (None, None)
    if new is not None:
        et = _elem_torch_dtype(desc.dtype)
        shape = (desc.batch, desc.n_kv_heads, 1, desc.head_dim)
        _tensor(k_new, "k_new", et, shape)
        _tensor(v_new, "v_new", et, shape)
    device = _same_gpu(q=q, out=out, P_qk=P_qk, P_vo=P_vo, k_new=k_new, v_new=v_new,
                       prefix=None if prefix is None else prefix.cache.k_pages)
    if workspace is None:
        need = ctypes.c_size_t()
        ask = head
        if new is not None:  # for the lengths after the step
            ask = head[:2] + (_i32_array([L + 1 for L in seq_len]),) + head[3:]
        _check(_lib.swan_decode_window_workspace_bytes(*ask, ctypes.byref(need)))
        workspace = _made("empty", (need.value,), "uint8", device, stream)
    else:
        workspace = _workspace(workspace, 0, device, stream)
    tail = (_ptr(q), _ptr(P_qk), _ptr(P_vo), scale, _ptr(out), workspace.data_ptr(),
            workspace.numel() * workspace.element_size())
    with _CallsOn(device, stream) as s:
        if new is None:
            _check(_lib.swan_decode_attention_window(*head, *tail, s))
        else:
            _check(_lib.swan_decode_step_window(*head, _ptr(k_new), _ptr(v_new), *tail, s))


def copy_sequences(src: CacheDesc, src_len: Sequence[int], k_active_src: Sequence[int],
                   k_value_src: Optional[Sequence[int]], dst: CacheDesc,
                   k_active_dst: Sequence[int], k_value_dst: Optional[Sequence[int]],
                   of: Sequence[int], first: Optional[Sequence[int]] = None,
                   drop: Optional[Sequence[int]] = None, stream=None) -> None:
    """Sequences of src to places of dst (see swan_copy_sequences)."""
    _check(_lib.swan_copy_sequences(
        ctypes.byref(src), _per_sequence(src_len, src.batch, "src_len"),
        _per_sequence(k_active_src, src.batch, "k_active_src"),
        _per_sequence(k_value_src, src.batch, "k_value_src"), ctypes.byref(dst),
        _per_sequence(k_active_dst, dst.batch, "k_active_dst"),
        _per_sequence(k_value_dst, dst.batch, "k_value_dst"),
        _per_sequence(of, dst.batch, "of"), _per_sequence(first, dst.batch, "first"),
        _per_sequence(drop, dst.batch, "drop"), _stream(stream)))


def set_decode_tuning(target_waves: int = 0, short_split_pages: int = 0, merge_pct: int = 0,
                      side_streams: int = 0) -> None:
    """Split plan and launch grouping of the decode calls without a window on this thread
    (swan_set_decode_tuning; 0 = the default, -1 = off where the header allows it).
    With every argument 0 the defaults are restored."""
    t = DecodeTuning(target_waves, short_split_pages, merge_pct, side_streams)
    _check(_lib.swan_set_decode_tuning(ctypes.byref(t)))


def set_profile_events(start=None, stop=None) -> None:
    """Record start/stop (events with a .cuda_event HIP handle: torch.cuda.Event, or one
    made for timing only) around the attention kernels of the next decode calls without a
    window on this thread (None, None disables)."""
    _check(_lib.swan_set_profile_events(None if start is None else start.cuda_event,
                                        None if stop is None else stop.cuda_event))


class SwanCache:
    """Owns the device arrays of one layer's hybrid cache and the host-side lengths.

    The arrays are plain torch tensors (uint8 pages, storage-typed ring); the
    library only ever receives their device pointers.  sparse_values="e4m3"
    (float16 only) stores the pruned values as one-byte E4M3 codes.  k_value
    (one per sequence) prunes the values to other k than the keys (k_active);
    None keeps both at k_active.
    """

    def __init__(self, batch: int, n_q_heads: int, n_kv_heads: int, buffer_tokens: int,
                 sparse_capacity: int, k_active: Sequence[int], dtype, device,
                 head_dim: int = HEAD_DIM, sparse_values: str = "same",
                 k_value: Optional[Sequence[int]] = None):
        import torch

        self.dtype = dtype
        self.sparse_values = sparse_values
        self.device = torch.device(device)
        self.k_active = [int(k) for k in k_active]
        if len(self.k_active) != batch:
            raise ValueError("k_active needs one entry per sequence")
        self.k_value = None if k_value is None else [int(k) for k in k_value]
        if self.k_value is not None and len(self.k_value) != batch:
            raise ValueError("k_value needs one entry per sequence")
        self.seq_len = [0] * batch
        # sequences copied with tokens left out: their length then, and the first token behind the gap
        self._cuts = {}
        self.desc = CacheDesc(batch, n_q_heads, n_kv_heads, head_dim, buffer_tokens,
                              sparse_capacity, dtype_code(dtype, sparse_values), 0, None, None,
                              None, None)
        self._allocate(None)

    def _allocate(self, stream) -> None:
        """The arrays that desc describes, zeroed, for work on `stream`."""
        d = self.desc
        kb, vb, rb = cache_bytes(d, self.k_active, self.k_value)
        # torch's caching allocator returns 256-byte aligned blocks
        self.k_pages = _result("zeros", max(kb, 16), "uint8", self.device, stream)
        self.v_pages = _result("zeros", max(vb, 16), "uint8", self.device, stream)
        shape = (d.batch, d.n_kv_heads, d.buffer_tokens, d.head_dim)
        self.k_ring = _result("zeros", shape, self.dtype, self.device, stream)
        self.v_ring = _result("zeros", shape, self.dtype, self.device, stream)
        d.k_pages = self.k_pages.data_ptr()
        d.v_pages = self.v_pages.data_ptr()
        d.k_ring = self.k_ring.data_ptr() if d.buffer_tokens > 0 else None
        d.v_ring = self.v_ring.data_ptr() if d.buffer_tokens > 0 else None

    @property
    def batch(self) -> int:
        return self.desc.batch

    def append(self, k_new, v_new, P_qk, P_vo, n_new_per_seq=None, stream=None) -> None:
        """Compress-append k_new / v_new ([B][H_kv][n][d]) and advance the lengths.

        n_new_per_seq optionally appends only the first n_b rows of sequence b.
        """
        compress_append(self.desc, self.seq_len, self.k_active, k_new, v_new, P_qk, P_vo,
                        n_new_per_seq, stream, self.k_value)
        n = int(k_new.shape[2])
        per = [n] * self.batch if n_new_per_seq is None else [int(x) for x in n_new_per_seq]
        self._grow([L + m for L, m in zip(self.seq_len, per)])

    def _grow(self, seq_len) -> None:
        """The lengths after an append.  A sequence that grows forgets how it was cut."""
        if self._cuts:
            self._cuts = {b: cut for b, cut in self._cuts.items()
                          if cut[0] == self.seq_len[b] == seq_len[b]}
        self.seq_len = seq_len

    def change_k(self, k_active: Sequence[int], k_value: Optional[Sequence[int]] = None,
                 stream=None) -> None:
        """Change k of the running sequences (swan_change_k): new page arrays for the new
        k, the stored tokens converted into them, the dense buffer kept.  Tokens that
        leave the buffer from now on are pruned with the new k."""
        import torch

        k_active = [int(k) for k in k_active]
        k_value = None if k_value is None else [int(k) for k in k_value]
        dst = CacheDesc(*[getattr(self.desc, f) for f, _ in CacheDesc._fields_])
        kb, vb, _ = cache_bytes(dst, k_active, k_value)
        k_pages, v_pages = (_result("zeros", (max(n, 16),), "uint8", self.k_pages.device, stream)
                            for n in (kb, vb))
        dst.k_pages = k_pages.data_ptr()
        dst.v_pages = v_pages.data_ptr()
        change_k(self.desc, self.k_active, self.k_value, dst, k_active, k_value, self.seq_len,
                 stream)
        # the old pages stay alive until the conversion on the stream has read them
        (stream or torch.cuda.current_stream()).synchronize()
        self.desc, self.k_pages, self.v_pages = dst, k_pages, v_pages
        self.k_active, self.k_value = k_active, k_value

    def outside(self, window: int, sinks=0, decode: bool = False):
        """Per sequence, how many pruned tokens after the first `sinks` (a number, or one per
        sequence) no later row with this window sees: the `drop` that copy_from and select can
        leave out from first=sinks on.  Later rows are those of step() and attend(), and of
        decode() after an append; decode() before it stands at the last cached token, one row
        earlier: decode=True keeps what that sees too (without, decode() with this window
        refuses the copy until a token is appended)."""
        if window is None:
            raise SwanError(SWAN_ERR_INVALID_ARG, "window is None")
        _window(window, sinks)
        b = self.desc.buffer_tokens
        first = [sinks] * self.batch if isinstance(sinks, int) else list(sinks)
        if len(first) != self.batch:
            raise SwanError(SWAN_ERR_INVALID_ARG,
                            f"sinks has {len(first)} entries for {self.batch} sequences")
        hidden = [L - window + (0 if decode else 1) for L in self.seq_len]
        return [max(0, min(x, L - b) - f) for x, L, f in zip(hidden, self.seq_len, first)]

    def _check_last_row(self, window: int, sinks: int, prefix: Optional[Prefix]) -> None:
        """Refuses a decode call whose window shows one more token than the copies that cut its
        sequences kept: its row stands one before the rows that outside() speaks of."""
        _window(window, sinks, True)
        of = None if prefix is None else prefix.of or [0] * self.batch
        for b in range(self.batch):
            held = [(self, b)]
            if not self.seq_len[b] and of is not None and len(of) == self.batch and \
                    0 <= of[b] < prefix.cache.batch:
                held.append((prefix.cache, of[b]))
            for cache, p in held:
                length, first = cache._cuts.get(p, (-1, 0))
                if length == cache.seq_len[p] and length - window == first - 1:
                    raise SwanError(SWAN_ERR_INVALID_ARG,
                                    f"decode: the token before the last {window - 1} of sequence "
                                    f"{b} was left out of a copy (outside(..., decode=True) keeps "
                                    "it)")

    def copy_from(self, src: "SwanCache", of: Sequence[int], first=0,
                  drop: Optional[Sequence[int]] = None, stream=None) -> None:
        """Sequence b becomes sequence of[b] of another cache `src` (-1: it stays as it is; one
        may be taken several times), without its tokens first .. first + drop[b] - 1 (pruned
        ones; first: a number, or one per sequence).  The tokens behind move up: keys keep the
        positions they were turned to, so a caller that counts positions adds drop[b]."""
        import torch

        of = [int(p) for p in of]
        first = [first] * self.batch if isinstance(first, int) else list(first)
        for x in (of, first, [] if drop is None else drop):  # (ctypes would take their low 32 bits)
            if any(not -1 <= v < 2**31 for v in x):
                raise SwanError(SWAN_ERR_INVALID_ARG, f"of, first or drop out of range: {x}")
        device = _same_gpu(src=src.k_pages, dst=self.k_pages)
        with _CallsOn(device, stream):
            copy_sequences(src.desc, src.seq_len, src.k_active, src.k_value, self.desc,
                           self.k_active, self.k_value, of, first, drop,
                           stream)
            # src may be dropped before the copy has read it
            at = stream or torch.cuda.current_stream(device)
            for t in (src.k_pages, src.v_pages, src.k_ring, src.v_ring):
                t.record_stream(at)
        for b, p in enumerate(of):
            if p < 0:
                continue
            left_out = 0 if drop is None else int(drop[b])
            self.seq_len[b] = src.seq_len[p] - left_out
            self._cuts.pop(b, None)
            if left_out:
                self._cuts[b] = (self.seq_len[b], first[b])
            elif p in src._cuts:
                self._cuts[b] = src._cuts[p]

    def select(self, of: Sequence[int], first=0, drop: Optional[Sequence[int]] = None,
               sparse_capacity: Optional[int] = None, stream=None) -> "SwanCache":
        """A new cache of len(of) sequences, sequence b a copy of sequence of[b] (-1: empty):
        forks, a new order, without finished sequences, with another capacity, or (first, drop
        as in copy_from) without tokens that are not needed any more.  (Graphs captured with this
        cache go on with this one.)"""
        of = [int(p) for p in of]
        if any(not -1 <= p < self.batch for p in of):
            raise ValueError(f"of must be sequences of this cache, -1..{self.batch - 1}")
        new = copy.copy(self)
        new.k_active = [self.k_active[max(p, 0)] for p in of]
        new.k_value = None if self.k_value is None else [self.k_value[max(p, 0)] for p in of]
        new.seq_len, new._cuts = [0] * len(of), {}
        d = self.desc
        new.desc = CacheDesc(len(of), d.n_q_heads, d.n_kv_heads, d.head_dim, d.buffer_tokens,
                             d.sparse_capacity if sparse_capacity is None else sparse_capacity,
                             d.dtype, 0, None, None, None, None)
        new._allocate(stream)
        new.copy_from(self, of, first, drop, stream)
        return new

    def workspace(self, seq_len: Optional[Sequence[int]] = None, prefix: Optional[Prefix] = None,
                  stream=None, window: Optional[int] = None, sinks: int = 0):
        """A decode workspace for these lengths (default: the present ones), of the caching
        allocator's memory for `stream` (or, captured, for its graph).  decode() and step()
        take one for each call, so calls on several streams, and graphs that are replayed
        beside them, share none."""
        lens = self.seq_len if seq_len is None else seq_len
        if window is not None:
            need = decode_window_workspace_bytes(self.desc, lens, self.k_active, window, sinks,
                                                 self.k_value, prefix)
        elif prefix is None:
            need = decode_workspace_bytes(self.desc, lens, self.k_active, self.k_value)
        else:
            need = prefix_workspace_bytes(prefix, self.desc, lens, self.k_active, self.k_value)
        return _made("empty", (need,), "uint8", self.k_pages.device, stream)

    def attend(self, q, P_qk, P_vo, of: Optional[Sequence[int]] = None,
               n: Optional[Sequence[int]] = None, scale: float = 0.0,
               prefix: Optional[Prefix] = None, out=None, workspace=None, stream=None,
               window: Optional[int] = None, sinks: int = 0):
        """Rows q [B][H_q][n][128] over all tokens of this cache, of sequence of[b] for query
        sequence b (-1: none; None: its own, b), and of a prefix, or over those that a window
        shows: see attend()."""
        own = Prefix(self, range(self.batch) if of is None else of)
        return attend([own] if prefix is None else [prefix, own], q, P_qk, P_vo, n, scale, out,
                      workspace, stream, window, sinks)

    def decode(self, q, P_qk, P_vo, out=None, scale: float = 0.0, stream=None,
               prefix: Optional[Prefix] = None, window: Optional[int] = None, sinks: int = 0):
        """Attention of q ([B][H_q][d]) over the cache, behind a prefix where one is given.
        window: over the last `window` tokens and the first `sinks` alone (an error where a copy
        cut for later rows, see outside(), left out the first of these `window`)."""
        if out is None:
            out = _result_like(q, q.shape, stream)
        if window is not None or sinks:
            if self._cuts or prefix is not None and prefix.cache._cuts:
                self._check_last_row(window, sinks, prefix)
            decode_window(self.desc, self.seq_len, self.k_active, q, P_qk, P_vo, out, None, window,
                          sinks, scale, stream, self.k_value, prefix)
        elif prefix is None:
            decode_attention(self.desc, self.seq_len, self.k_active, q, P_qk, P_vo, out,
                             self.workspace(None, None, stream), scale, stream, self.k_value)
        else:
            decode_attention_prefix(prefix, self.desc, self.seq_len, self.k_active, q, P_qk, P_vo,
                                    out, self.workspace(None, prefix, stream), scale, stream,
                                    self.k_value)
        return out

    def step(self, k_new, v_new, q, P_qk, P_vo, out=None, scale: float = 0.0, stream=None,
             prefix: Optional[Prefix] = None, window: Optional[int] = None, sinks: int = 0):
        """One decode step (swan_decode_step): append k_new / v_new ([B][H_kv][1][d]),
        advance the lengths, and return the attention of q ([B][H_q][d]) over the cache,
        behind a prefix where one is given; window, sinks as in decode()."""
        if out is None:
            out = _result_like(q, q.shape, stream)
        after = [L + 1 for L in self.seq_len]
        if window is not None or sinks:
            decode_window(self.desc, self.seq_len, self.k_active, q, P_qk, P_vo, out, None, window,
                          sinks, scale, stream, self.k_value, prefix, (k_new, v_new))
            self._grow(after)
            return out
        ws = self.workspace(after, prefix, stream)
        if prefix is None:
            decode_step(self.desc, self.seq_len, self.k_active, k_new, v_new, q, P_qk, P_vo, out,
                        ws, scale, stream, self.k_value)
        else:
            decode_step_prefix(prefix, self.desc, self.seq_len, self.k_active, k_new, v_new, q,
                               P_qk, P_vo, out, ws, scale, stream, self.k_value)
        self._grow(after)
        return out
