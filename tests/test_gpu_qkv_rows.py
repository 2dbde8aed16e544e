"""swan_qkv_rows: heads split, norms and rotation against the formula in float64."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
D = 128


def _formula(x, hq, hkv, pos0, base, wq, wk, eps):
    """q, k, v float64 numpy [B][heads][n][D] of qkv rows x [B][n][width]."""
    B, n, _ = x.shape
    rows = x.astype(np.float64).reshape(B, n, hq + 2 * hkv, D).transpose(0, 2, 1, 3)
    angle = (np.asarray(pos0, dtype=np.float64)[:, None] + np.arange(n))[..., None] * \
        np.float64(base) ** (-2.0 * np.arange(D // 2) / D)
    turn = np.exp(1j * angle)[:, None]  # [B][1][n][64]

    def head(part, w):
        if w is not None:
            r = 1 / np.sqrt(np.mean(part * part, axis=-1, keepdims=True) + eps)
            w = w.astype(np.float64)
            part = part * r * (w if w.ndim == 1 else w[None, :, None, :])
        z = (part[..., :64] + 1j * part[..., 64:]) * turn
        return np.concatenate([z.real, z.imag], axis=-1)

    return head(rows[:, :hq], wq), head(rows[:, hq:hq + hkv], wk), rows[:, hq + hkv:]


def _make(torch, device, B, n, hq, hkv, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(B, n, (hq + 2 * hkv) * D, generator=g) * 2).to(dtype).to(device)


def _close(got, want, dtype):
    """A rounding is off by half a step, where the float64 value may be off by its own
    (angles to 1e5 with 2^-52 each: 2^-35 at most, far below half a step of either type)."""
    import torch

    got = got.double().cpu().numpy()
    u = 2.0 ** -11 if dtype == torch.float16 else 2.0 ** -24
    tiny = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -140
    tol = np.abs(want) * u * (1 + 2.0 ** -8) + np.abs(want).max() * 2.0 ** -34 + tiny
    assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / tol)


# few rows (one wave each), and several (4 positions a workgroup): both sides of 4096 rows
SHAPES = [(1, 1, 1, 1), (1, 1, 32, 8), (4, 1, 32, 8), (3, 5, 12, 4), (2, 31, 16, 1), (1, 85, 32, 8),
          (1, 86, 32, 8), (2, 129, 20, 4), (5, 203, 4, 4), (64, 3, 6, 2), (3, 401, 7, 7)]


@pytest.mark.parametrize("norms", ["none", "shared", "heads", "q only"])
@pytest.mark.parametrize("name", ["float16", "float32"])
@pytest.mark.parametrize("B,n,hq,hkv", SHAPES)
def test_rows_are_the_formula(gpu_device, swan_mod, torch_mod, B, n, hq, hkv, name, norms):
    torch = torch_mod
    dtype = getattr(torch, name)
    x = _make(torch, gpu_device, B, n, hq, hkv, dtype, B + n)
    g = torch.Generator().manual_seed(9)
    wq = wk = None
    if norms != "none":
        shape = (lambda h: (h, D)) if norms == "heads" else (lambda h: (D,))
        # float32 weights for binary16 rows in one form, the rows' own type in the others
        wt = torch.float32 if norms == "shared" else dtype
        wq = (1 + 0.3 * torch.randn(shape(hq), generator=g)).to(wt).to(gpu_device)
        if norms != "q only":
            wk = (1 + 0.3 * torch.randn(shape(hkv), generator=g)).to(wt).to(gpu_device)
    pos0 = [(7919 * b) % 100000 for b in range(B)]
    q, k, v = swan_mod.qkv_rows(x, hq, hkv, pos0, 10000.0, wq, wk, eps=1e-5)
    torch.cuda.synchronize()
    host = [None if w is None else w.double().cpu().numpy() for w in (wq, wk)]
    eq, ek, ev = _formula(x.double().cpu().numpy(), hq, hkv, pos0, 10000.0, *host, 1e-5)
    _close(q, eq, dtype)
    _close(k, ek, dtype)
    assert np.array_equal(v.double().cpu().numpy(), ev)


@pytest.mark.parametrize("name", ["float16", "float32"])
@pytest.mark.parametrize("B,n", [(2, 9), (3, 700)])
def test_without_norms_it_is_rope(gpu_device, swan_mod, torch_mod, B, n, name):
    torch = torch_mod
    x = _make(torch, gpu_device, B, n, 8, 4, getattr(torch, name), 5)
    pos0 = [100, 65000, 3][:B]
    q, k, v = swan_mod.qkv_rows(x, 8, 4, pos0, 500000.0)
    heads = x.view(B, n, 16, D).transpose(1, 2).contiguous()
    assert torch.equal(q, swan_mod.rope(heads[:, :8].contiguous(), pos0, 500000.0))
    assert torch.equal(k, swan_mod.rope(heads[:, 8:12].contiguous(), pos0, 500000.0))
    assert torch.equal(v, heads[:, 12:])


@pytest.mark.parametrize("n", [3, 300])
def test_strided_rows_and_single_parts(gpu_device, swan_mod, torch_mod, n):
    """Rows inside wider ones, sequences further apart than their rows; keys and values or
    queries alone; outputs given."""
    torch = torch_mod
    B, hq, hkv = 2, 6, 2
    wide = _make(torch, gpu_device, B, n + 2, hq + 6, hkv, torch.float16, 3)
    x = wide[:, 1:n + 1, 2 * D:(2 + hq + 2 * hkv) * D]
    want = swan_mod.qkv_rows(x.contiguous(), hq, hkv, [5, 6], 10000.0)
    got = swan_mod.qkv_rows(x, hq, hkv, [5, 6], 10000.0)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    out = [torch.full_like(t, 7.0) for t in want]
    swan_mod.qkv_rows(x, hq, hkv, [5, 6], 10000.0, out=out)
    for a, b in zip(out, want):
        assert torch.equal(a, b)
    none, k, v = swan_mod.qkv_rows(x[..., hq * D:], 0, hkv, [5, 6], 10000.0)
    assert none is None and torch.equal(k, want[1]) and torch.equal(v, want[2])
    q, none, _ = swan_mod.qkv_rows(x[..., :hq * D], hq, 0, [5, 6], 10000.0)
    assert none is None and torch.equal(q, want[0])


@pytest.mark.parametrize("n", [2, 300])
@pytest.mark.parametrize("name", ["float16", "float32"])
def test_rows_of_zeros_infinities_and_nans(gpu_device, swan_mod, torch_mod, name, n):
    """A row of zeros stays zeros under a norm; an infinity makes itself NaN and the rest of
    its row 0, as x / sqrt(inf); a NaN its row; other rows are as they were."""
    torch = torch_mod
    x = _make(torch, gpu_device, 1, n, 8, 4, getattr(torch, name), 11)
    w = torch.ones(D, device=gpu_device, dtype=x.dtype)
    good = swan_mod.qkv_rows(x, 8, 4, [3], 10000.0, w, w)
    x[0, 0, :D] = 0
    x[0, 0, D + 5] = math.inf
    x[0, 1, 2 * D + 70] = math.nan
    x[0, 1, 12 * D + 1] = math.nan  # a value
    q, k, v = swan_mod.qkv_rows(x, 8, 4, [3], 10000.0, w, w)
    assert torch.all(q[0, 0, 0] == 0)
    row = q[0, 1, 0]
    assert torch.isnan(row[[5, 69]]).all()
    rest = [j for j in range(D) if j not in (5, 69)]
    assert torch.all(row[rest] == 0)
    assert torch.isnan(q[0, 2, 1]).all()
    assert torch.isnan(v[0, 0, 1, 1]) and torch.equal(v[0, 0, 1, 2:], good[2][0, 0, 1, 2:])
    assert torch.equal(q[0, 3:], good[0][0, 3:]) and torch.equal(k, good[1])


def test_no_rows(gpu_device, swan_mod, torch_mod):
    torch = torch_mod
    x = torch.empty(2, 0, 12 * D, dtype=torch.float16, device=gpu_device)
    q, k, v = swan_mod.qkv_rows(x, 8, 2, [0, 0], 10000.0)
    assert q.shape == (2, 8, 0, D) and k.shape == v.shape == (2, 2, 0, D)


def test_on_another_stream_and_captured(gpu_device, swan_mod, torch_mod):
    torch = torch_mod
    x = _make(torch, gpu_device, 2, 40, 8, 2, torch.float16, 1)
    want = swan_mod.qkv_rows(x, 8, 2, [1, 2], 10000.0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = swan_mod.qkv_rows(x, 8, 2, [1, 2], 10000.0, stream=side)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    out = [torch.zeros_like(t) for t in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        swan_mod.qkv_rows(x, 8, 2, [1, 2], 10000.0, out=out)
    for turn in range(3):
        x.add_(0.5)
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, swan_mod.qkv_rows(x, 8, 2, [1, 2], 10000.0)):
            assert torch.equal(a, b), turn
