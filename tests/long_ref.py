"""Plain float64 forms of what long-running sequences take (sliding windows, rotary positions),
for the tests (torch, on whatever device the inputs are)."""
import math

from tests import rows_ref as R

D = 128


def seen_mask(p, j, window, sinks):
    """Rows at positions p against keys at positions j: [rows][keys]."""
    p, j = p[:, None], j[None]
    return (j <= p) & ((j > p - window) | (j < sinks))


def rotate(x, pos, rotary):
    """x [..., n][128] float64 at positions pos [n] (float64), as swan.Rotary says."""
    import torch

    half = rotary.dims // 2
    t = pos[:, None] * torch.tensor(rotary.freqs, dtype=torch.float64, device=x.device)
    c, s = rotary.magnitude * torch.cos(t), rotary.magnitude * torch.sin(t)
    y = x.clone()
    if rotary.interleaved:
        a, b = slice(0, rotary.dims, 2), slice(1, rotary.dims, 2)
    else:
        a, b = slice(0, half), slice(half, rotary.dims)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def cached_attention(cache, b, h, q, P_qk, P_vo, p, window, sinks, before=None, chunk=None):
    """Rows q [rows][128] (un-rotated) at positions p over what `cache` holds of (sequence b, kv
    head h), behind the rows `before` = (K, V) of a prefix, and with chunk = (k, v) rows behind
    the cached tokens (v rotated): (o, lse) in the basis that P_vo gives (None: rotated), and the
    turned queries, keys and values for a bound."""
    import torch

    K, V = R.cached_rows(cache, b, h, 0), R.cached_rows(cache, b, h, 1)
    if before is not None:
        K, V = torch.cat([before[0], K]), torch.cat([before[1], V])
    turned = q.double() @ P_qk[h].double()
    if chunk is not None:
        K = torch.cat([K, chunk[0].double() @ P_qk[h].double()])
        V = torch.cat([V, chunk[1].double()])
    j = torch.arange(K.shape[0], device=q.device)
    o, lse = R.softmax_rows(turned, K, V, seen_mask(p, j, window, sinks))
    if P_vo is not None:
        o = o @ P_vo[h].double().T
    return o, lse, (turned, K, V)


def lse_bound(q, k):
    """A bound on the error of lse: a score's (rows_ref.bound), its own rounding and the
    sum's."""
    if not k.numel():
        return 2.0 ** -20
    top = q.norm(dim=-1).max().item() * k.norm(dim=-1).max().item() / math.sqrt(D)
    return top * 2.0 ** -15 + (k.shape[0] + 32) * 2.0 ** -23
