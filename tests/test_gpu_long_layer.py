"""The layer with a window, another rotary form, copies and compaction, used together as a
long-running sequence uses them, against the formula in float64 over all its tokens."""
import math

import pytest

from tests import long_ref as LR
from tests import rows_ref as R
from tests.test_gpu_layer_rows import HIDDEN, TOL, _err, _layer, _x

pytestmark = pytest.mark.gpu
D = 128


class Told:
    """A layer, and what its rows should be: q, k (turned to absolute positions) and v of every
    token from the projections, in float64.  k = 128 kept components: nothing is pruned."""

    def __init__(self, torch, layer):
        self.torch, self.layer, self.k, self.v = torch, layer, [], []
        self.at = 0

    def rows(self, x):
        layer, torch = self.layer, self.torch
        B, n = x.shape[:2]
        rows = (x @ layer.W_qkv).double()
        q, k, v = rows.split([layer.n_heads * D, layer.n_kv_heads * D, layer.n_kv_heads * D], -1)
        out = []
        for t, w in ((q, layer.q_norm), (k, layer.k_norm), (v, None)):
            t = t.reshape(B, n, -1, D).transpose(1, 2)
            if w is not None:
                t = t / torch.sqrt(t.square().mean(-1, keepdim=True) + layer.norm_eps) * w.double()
            out.append(t)
        pos = torch.arange(n, device=x.device, dtype=torch.float64) + self.at
        q, k = (LR.rotate(t, pos, layer.rope_base) for t in out[:2])
        self.k.append(k)
        self.v.append(out[2])
        self.at += n
        return q

    def want(self, x):
        layer, torch = self.layer, self.torch
        q = self.rows(x)
        k, v = torch.cat(self.k, 2), torch.cat(self.v, 2)
        B, n, G = x.shape[0], x.shape[1], layer.n_heads // layer.n_kv_heads
        p = torch.arange(n, device=x.device) + self.at - n
        seen = LR.seen_mask(p, torch.arange(self.at, device=x.device), layer.window, layer.sinks)
        out = torch.empty(B, n, layer.n_heads * D, dtype=torch.float64, device=x.device)
        for b in range(B):
            for h in range(layer.n_heads):
                o, _ = R.softmax_rows(q[b, h], k[b, h // G], v[b, h // G], seen)
                out[b, :, h * D:(h + 1) * D] = o
        return out @ layer.W_o_hat.double()


@pytest.mark.parametrize("name", ["float16", "float32"])
def test_a_long_sequence(gpu_device, swan_mod, torch_mod, name):
    """A prompt, chunks, steps, compaction in between, a copy in another order, and on."""
    torch = torch_mod
    dtype = getattr(torch, name)
    rotary = swan_mod.Rotary(10000.0, dims=64, interleaved=True).by_parts(4.0, 256)
    layer = _layer(torch, gpu_device, hq=4, hkv=2, batch=2, buffer=16, capacity=500, k=128,
                   window=60, sinks=5, dtype=dtype)
    layer.rope_base = rotary
    told = Told(torch, layer)
    seed = 0

    def go(n):
        nonlocal seed
        seed += 1
        x = _x(torch, gpu_device, 2, n, seed, dtype)
        y = layer(x, attend=True).reshape(2, n, HIDDEN)
        torch.cuda.synchronize()
        assert _err(y, told.want(x)) < TOL, (n, told.at)

    go(3)
    go(150)
    go(40)
    for _ in range(3):
        go(1)
    drop = layer.compact(capacity=300)
    assert drop == [196 - 59 - 5] * 2 and layer.positions() == [196, 196]
    assert layer.cache.seq_len == [64, 64]
    for _ in range(3):
        go(1)
    go(33)
    go(100)
    layer.compact()
    assert layer.positions() == [told.at] * 2
    swapped = layer.select([1, 0])
    told2 = Told(torch, swapped)
    told2.k, told2.v = [t.flip(0) for t in told.k], [t.flip(0) for t in told.v]
    told2.at = told.at
    x = _x(torch, gpu_device, 2, 1, 99, dtype)
    y = layer(x)
    z = swapped(x.flip(0).contiguous())
    assert _err(z.flip(0), y.double()) < TOL
    told.rows(x)
    told2.rows(x.flip(0).contiguous())
    layer, told = swapped, told2
    go(20)
    go(1)


def test_a_fork_of_a_compacted_layer(gpu_device, swan_mod, torch_mod):
    """Users behind a shared prompt, part of which their windows leave."""
    torch = torch_mod
    base = _layer(torch, gpu_device, hq=4, hkv=2, batch=1, buffer=16, capacity=500, k=128, window=50,
                  sinks=3)
    base.rope_base = swan_mod.Rotary(10000.0)
    told = Told(torch, base)
    x = _x(torch, gpu_device, 1, 200, 1)
    assert _err(base(x, attend=True), told.want(x)) < TOL
    base.compact()
    users = base.fork([0, 0, 0], buffer_tokens=16, capacity=300, k_active=[128] * 3)
    assert users.positions() == [200] * 3
    mine = Told(torch, users)
    mine.k, mine.v = [told.k[0].expand(3, -1, -1, -1)], [told.v[0].expand(3, -1, -1, -1)]
    mine.at = 200
    for seed, n in ((2, 7), (3, 1), (4, 60), (5, 1), (6, 30)):
        x = _x(torch, gpu_device, 3, n, seed)
        y = users(x, attend=True).reshape(3, n, HIDDEN)
        assert _err(y, mine.want(x)) < TOL, n
    assert users.compact() == [99 - 49 - 0] * 3
    assert users.positions() == [299] * 3
    two = users.select([2, 0])
    assert two.positions() == [299] * 2
    mine.k, mine.v = [t[[2, 0]] for t in mine.k], [t[[2, 0]] for t in mine.v]
    mine.layer = two
    for seed, n in ((7, 1), (8, 5)):
        x = _x(torch, gpu_device, 2, n, seed)
        y = two(x, attend=True).reshape(2, n, HIDDEN)
        assert _err(y, mine.want(x)) < TOL, n


def test_without_a_window_nothing_changes(gpu_device, swan_mod, torch_mod):
    """A Rotary of the whole head is the base but for a last bit, and a copy goes on as its
    source."""
    torch = torch_mod
    a = _layer(torch, gpu_device)
    b = _layer(torch, gpu_device)
    b.rope_base = swan_mod.Rotary(10000.0)
    for n, seed in ((50, 1), (1, 2), (20, 3)):
        x = _x(torch, gpu_device, 2, n, seed)
        ya, yb = a(x, attend=True), b(x, attend=True)
        assert _err(yb.reshape(2, n, HIDDEN), ya.double().reshape(2, n, HIDDEN)) < TOL
    c = a.select([1, 0])
    x = _x(torch, gpu_device, 2, 1, 9)
    assert _err(c(x.flip(0).contiguous()).flip(0), a(x).double()) < TOL
    with pytest.raises(ValueError):
        a.compact()
    assert math.isfinite(ya.float().abs().max().item())
