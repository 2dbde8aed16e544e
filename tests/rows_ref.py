"""Plain float64 forms of the several-row operators, and bounds on a kernel's error that
follow from its arithmetic, for the GPU tests (torch, on whatever device the inputs are)."""
import math

import numpy as np

from tests import swan_cases as C

D = 128
HALF = {"f16": 2.0 ** -11, "f32": 2.0 ** -24}  # half a step of a rounding


def softmax_rows(q, k, v, seen=None, state=None):
    """softmax(q k^T / sqrt(D)) v over the pairs of `seen` ([rows][keys] or None), continued
    from state (o, lse): o [rows][D] and lse [rows], float64; rows with nothing give 0, -inf."""
    import torch

    q, k, v = q.double(), k.double(), v.double()
    s = (q @ k.T) / math.sqrt(D)
    if seen is not None:
        s = s.masked_fill(~seen, -math.inf)
    o0 = torch.zeros(q.shape[0], D, dtype=torch.float64, device=q.device)
    lse0 = torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device)
    if state is not None:
        o0, lse0 = state[0].double(), state[1].double()
    top = lse0 if k.shape[0] == 0 else torch.maximum(s.amax(1), lse0)
    safe = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p, w0 = torch.exp(s - safe[:, None]), torch.exp(lse0 - safe)
    total = p.sum(1) + w0
    o = torch.where(w0[:, None] > 0, w0[:, None] * o0, torch.zeros_like(o0))
    if seen is None:
        o = o + p @ v
    else:  # a value that a row does not see does not reach it
        for j in range(v.shape[0]):
            o = o + torch.where(seen[:, j, None], p[:, j, None] * v[j], torch.zeros_like(o))
    o = o / torch.where(total > 0, total, torch.ones_like(total))[:, None]
    return o, safe + torch.log(total)


def bound(dtype, q, k, v, o, keys, out_dtype=None, turned=False):
    """A bound on |kernel - o|, elementwise for o [rows][D]: the output's rounding; p's
    rounding, which moves weights that sum to one by a factor within 2 u each; a score's
    error, 2^-16 of |q| |k| / sqrt(D) (128 terms summed in float32, twice: the rotation's and
    the product's), in the exponent; the accumulation of `keys` terms in float32, which
    counts in full for float32 storage and is far below p's rounding for binary16.  The
    weights' errors multiply the values: an element's are at most the largest |v|, and after
    a rotation (turned) the largest norm of a row of v."""
    norm = lambda x: x.double().norm(dim=-1).max().item() if x.numel() else 0.0  # noqa: E731
    biggest = v.double().abs().max().item() if v.numel() else 0.0
    if turned:
        biggest = norm(v)
    score = norm(q) * norm(k) / math.sqrt(D) * 2.0 ** -16
    u = HALF[dtype] if dtype == "f16" else 2.0 ** -22  # (float32: exp2 within 2 ulp)
    rel = 2 * u + 2 * score + (keys + 16) * 2.0 ** -24
    if turned:  # and the turn's own sum of 128 products in float32
        rel += 128 * 2.0 ** -24
    return HALF[out_dtype or dtype] * o.abs() + biggest * rel + 2.0 ** -24


def close(got, want, tol, what=""):
    import torch

    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaNs elsewhere"
    same = (got == want) | torch.isnan(want)
    err = torch.where(same, torch.zeros_like(want), (got - want).abs())
    worst = (err / tol).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} of the bound, error {err.max().item():.3g}"
    return worst


def cached_rows(cache, b, h, role):
    """[L][D] float64: the rows that the cache holds of a (sequence, kv head), pruned
    components zero, then the buffer's, read back through the documented layout."""
    import torch

    L, bb = cache.seq_len[b], cache.desc.buffer_tokens
    S = max(0, L - bb)
    rows = np.zeros((L, D))
    if S:
        code = cache.sparse_values == "e4m3"
        esize = np.float32 if cache.dtype == torch.float32 else np.float16
        idx, val, _, _ = C.unit_pages(cache, b, h, role, S, np.uint8 if code else esize)
        if code:
            val = torch.tensor(np.ascontiguousarray(val)).view(torch.float8_e4m3fn).double()
            val = val.numpy()
        np.put_along_axis(rows[:S], idx, np.asarray(val, dtype=np.float64), axis=1)
    if L > S:
        rows[S:] = C.ring_rows(cache, b, h, role, L)
    return torch.tensor(rows, device=cache.device)


def rotations(heads, seed, device):
    import torch

    g = torch.Generator().manual_seed(seed)
    q, _ = torch.linalg.qr(torch.randn(heads, D, D, dtype=torch.float64, generator=g))
    return q.to(torch.float32).contiguous().to(device)


def filled_cache(swan, device, lengths, hq, hkv, buffer, k, dtype, seed, values="same",
                 k_value=None, spare=8, P=None):
    """A SwanCache with random rows of the given lengths appended (P: (P_qk, P_vo))."""
    import torch

    td = C.torch_dtype(dtype)
    g = torch.Generator().manual_seed(seed)
    n = max(lengths)
    cache = swan.SwanCache(len(lengths), hq, hkv, buffer, max(0, n + spare - buffer), k, td, device,
                           sparse_values=values, k_value=k_value)
    P_qk, P_vo = P or (rotations(hkv, seed + 1, device), rotations(hkv, seed + 2, device))
    if n:
        spectrum = torch.exp(-torch.arange(D) / 16.0)
        kv = [torch.matmul(torch.randn(len(lengths), hkv, n, D, generator=g).to(device) *
                           spectrum.to(device), R.transpose(1, 2)).to(td).contiguous()
              for R in (P_qk, P_vo)]
        cache.append(kv[0], kv[1], P_qk, P_vo, n_new_per_seq=list(lengths))
    return cache, P_qk, P_vo
