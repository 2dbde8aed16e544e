"""swan_rope_rotary and swan_qkv_rows_rotary against the formula in float64, rounded once."""
import math

import pytest

from tests import long_ref as LR
from tests import rows_ref as R

pytestmark = pytest.mark.gpu
D = 128


def _forms(swan):
    return [swan.Rotary(10000.0, dims=128), swan.Rotary(10000.0, dims=64),
            swan.Rotary(500000.0, dims=128, interleaved=True),
            swan.Rotary(10000.0, dims=96, interleaved=True), swan.Rotary(10000.0, dims=8),
            swan.Rotary(10000.0, dims=24), swan.Rotary(100.0, dims=8, interleaved=True),
            swan.Rotary(500000.0).by_parts(8.0, 8192),
            swan.Rotary(10000.0, dims=64, interleaved=True).stretched(4.0),
            swan.Rotary(10000.0, dims=120, magnitude=1.25)]


def _bound(torch, want, dtype, rows):
    """One rounding (half a step, and half the smallest step of binary16's subnormals), and the
    float64 steps before it, far below: 2^-40 of the row."""
    half = R.HALF["f32" if dtype == torch.float32 else "f16"]
    tiny = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -150
    return half * want.abs() + tiny + rows.double().abs().max().item() * 2.0 ** -36


SHAPES = [(1, 1, 1, [0]), (3, 5, 1, [7, 0, 120000]), (1, 32, 1, [4095]), (2, 7, 130, [1000, 2**30]),
          (1, 40, 700, [0]), (8, 2, 40, [5] * 8), (2, 33, 300, [3, 9])]


@pytest.mark.parametrize("name", ["float16", "float32"])
@pytest.mark.parametrize("B,H,n,pos0", SHAPES)
def test_rope_is_the_formula(gpu_device, swan_mod, torch_mod, B, H, n, pos0, name):
    torch = torch_mod
    dtype = getattr(torch, name)
    g = torch.Generator().manual_seed(n)
    x = torch.randn(B, H, n, D, generator=g).to(dtype).to(gpu_device)
    for r in _forms(swan_mod):
        y = swan_mod.rope(x, pos0, r)
        in_place = x.clone()
        assert swan_mod.rope(in_place, pos0, r, out=in_place) is in_place
        torch.cuda.synchronize()
        assert torch.equal(in_place, y)
        assert torch.equal(y[..., r.dims:], x[..., r.dims:])
        for b in range(B):
            pos = torch.arange(n, device=gpu_device, dtype=torch.float64) + pos0[b]
            want = LR.rotate(x[b].double(), pos, r)
            R.close(y[b], want, _bound(torch, want, dtype, x), f"{r.dims} {r.interleaved} {b}")


def test_the_whole_head_is_the_base(gpu_device, swan_mod, torch_mod):
    """A Rotary of a base gives the base's rows but for a last bit (its frequencies are the
    host's)."""
    torch = torch_mod
    g = torch.Generator().manual_seed(1)
    x = torch.randn(2, 6, 50, D, generator=g).to(gpu_device)
    a, b = swan_mod.rope(x, [3, 4000], 10000.0), swan_mod.rope(x, [3, 4000], swan_mod.Rotary(10000.0))
    assert (a - b).abs().max().item() <= 2.0 ** -23 * x.abs().max().item() * 2


@pytest.mark.parametrize("name", ["float16", "float32"])
@pytest.mark.parametrize("B,n,hq,hkv", [(1, 1, 2, 1), (3, 1, 8, 2), (2, 65, 7, 3), (1, 500, 12, 4),
                                        (2, 300, 0, 8), (4, 33, 32, 8)])
def test_qkv_rows_are_the_formula(gpu_device, swan_mod, torch_mod, B, n, hq, hkv, name):
    torch = torch_mod
    dtype = getattr(torch, name)
    g = torch.Generator().manual_seed(n)
    wide = torch.randn(B, n + 1, (hq + 2 * hkv) * D + 8, generator=g).to(dtype).to(gpu_device)
    x = wide[:, :n, :(hq + 2 * hkv) * D]  # rows with a stride
    pos0 = [11 * b + 900 for b in range(B)]
    for form, r in enumerate(_forms(swan_mod)):
        per_head, w_dtype = form % 2, dtype if form % 3 else torch.float32
        shape = lambda h: (h, D) if per_head else (D,)  # noqa: E731
        ws = [None, None]
        if form != 4:
            ws = [(1 + 0.2 * torch.randn(*shape(h), generator=g)).to(w_dtype).to(gpu_device)
                  for h in (hq, hkv)]
            if hq == 0:
                ws[0] = None
        q, k, v = swan_mod.qkv_rows(x, hq, hkv, pos0, r, *ws, eps=1e-5)
        torch.cuda.synchronize()
        rows = x.double().view(B, n, hq + 2 * hkv, D).transpose(1, 2)
        assert torch.equal(v.double(), rows[:, hq + hkv:])
        for got, h0, h1, w in ((q, 0, hq, ws[0]), (k, hq, hq + hkv, ws[1])):
            if h0 == h1:
                assert got is None
                continue
            want = rows[:, h0:h1]
            if w is not None:
                want = want / torch.sqrt(want.square().mean(-1, keepdim=True) + 1e-5)
                want = want * (w.double()[None, :, None] if per_head else w.double())
            pos = torch.arange(n, device=gpu_device, dtype=torch.float64)
            want = torch.stack([LR.rotate(want[b], pos + pos0[b], r) for b in range(B)])
            R.close(got, want, _bound(torch, want, dtype, want), f"form {form}")


def test_dims_that_are_not_turned_keep_their_bits(gpu_device, swan_mod, torch_mod):
    """Infinities and NaNs past the turned dims stay where they are, and reach no other; NaN
    bits stay as they are."""
    torch = torch_mod
    for shape in ((1, 2, 3, D), (1, 40, 500, D)):
        x = torch.randn(*shape, generator=torch.Generator().manual_seed(2)).half().to(gpu_device)
        x[0, 1, 1, 64] = math.inf
        x[0, 1, 1, 127] = math.nan
        x[0, 0, 2, 100] = -math.inf
        bits = x.view(torch.int16)
        bits[0, 1, 2, 90] = 0x7D55
        for inter in (False, True):
            r = swan_mod.Rotary(dims=64, interleaved=inter)
            y = swan_mod.rope(x, [5], r)
            assert torch.equal(y.view(torch.int16)[..., 64:], bits[..., 64:])
            assert torch.isfinite(y[..., :64].float()).all()
            rows = x.transpose(1, 2).reshape(shape[0], shape[2], -1).contiguous()
            q, _, _ = swan_mod.qkv_rows(rows, shape[1], 0, [5], r)
            assert torch.equal(q.view(torch.int16), y.view(torch.int16))


def test_on_another_stream_and_captured(gpu_device, swan_mod, torch_mod):
    torch = torch_mod
    x = torch.randn(2, 40, 300, D, generator=torch.Generator().manual_seed(2)).half().to(gpu_device)
    r = swan_mod.Rotary(dims=64, interleaved=True)
    want = swan_mod.rope(x, [1, 2], r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = swan_mod.rope(x, [1, 2], r, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graph, y = torch.cuda.CUDAGraph(), torch.zeros_like(x)
    with torch.cuda.graph(graph, stream=side):
        swan_mod.rope(x, [1, 2], r, out=y)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@pytest.mark.parametrize("name,H", [("float16", 130), ("float32", 66)])
def test_outputs_larger_than_the_caches(gpu_device, swan_mod, torch_mod, name, H):
    """More than 128 MiB of outputs, in one call and in parts of it: bit for bit the same."""
    torch = torch_mod
    n = 4099
    dtype = getattr(torch, name)
    g = torch.Generator().manual_seed(H)
    part = torch.randn(1, 7, n, D, generator=g).to(dtype).to(gpu_device)
    x = part.repeat(1, (H + 6) // 7, 1, 1)[:, :H].contiguous()
    r = swan_mod.Rotary(500000.0, dims=96, interleaved=True)
    y = swan_mod.rope(x, [11], r)
    few = swan_mod.rope(part, [11], r)
    for h in range(0, H, 7):
        assert torch.equal(y[:, h:h + 7], few[:, :min(7, H - h)])
    in_place = x.clone()
    swan_mod.rope(in_place, [11], r, out=in_place)
    assert torch.equal(in_place, y)
