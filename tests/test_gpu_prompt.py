"""swan_prompt_attention against the formula in float64: prompts, other keys, lengths and
masks that leave rows empty, states, infinities in places that a row does not see."""
import math

import pytest

from tests import rows_ref as R
from tests import swan_cases as C

pytestmark = pytest.mark.gpu
D = 128


def _inputs(torch, device, B, hq, hkv, n, m, dtype, seed, sharp=1.5):
    g = torch.Generator().manual_seed(seed)
    td = C.torch_dtype(dtype)
    make = lambda h, r, s: (torch.randn(B, h, r, D, generator=g) * s).to(td).to(device)  # noqa: E731
    return make(hq, n, sharp), make(hkv, m, 1.0), make(hkv, m, 1.0)


def _check(torch, got, q, k, v, causal, ns, ms, dtype, state=None):
    B, hq, n, _ = q.shape
    G = hq // k.shape[1]
    for b in range(B):
        nb, mb = ns[b], ms[b]
        i = torch.arange(nb, device=q.device)[:, None]
        j = torch.arange(mb, device=q.device)[None]
        seen = j <= i + mb - nb if causal else None
        for h in range(hq):
            st = None if state is None else (state[0][b, h, :nb], state[1][b, h, :nb])
            kb, vb = k[b, h // G, :mb], v[b, h // G, :mb]
            want, _ = R.softmax_rows(q[b, h, :nb], kb, vb, seen, st)
            fine = vb[torch.isfinite(vb.float())]
            if state is not None:
                fine = torch.cat([fine.reshape(-1).float(), state[0].reshape(-1)])
            tol = R.bound(dtype, q[b, h, :nb], kb, fine.reshape(-1, 1), torch.nan_to_num(want), mb)
            R.close(got[b, h, :nb], want, tol, f"sequence {b}, head {h}")


CASES = [  # B, hq, hkv, n, m, causal
    (1, 1, 1, 1, 1, True), (1, 2, 1, 2, 2, True), (2, 4, 2, 31, 31, True), (1, 3, 1, 63, 63, True),
    (1, 2, 2, 64, 64, True), (1, 8, 2, 65, 65, True), (1, 1, 1, 127, 127, True),
    (1, 4, 4, 128, 128, True), (2, 5, 1, 129, 129, True), (1, 16, 1, 200, 200, True),
    (1, 2, 2, 333, 333, True), (1, 4, 1, 500, 500, True),
    (1, 2, 1, 1, 700, False), (3, 4, 2, 1, 64, False), (2, 6, 2, 7, 65, False),
    (1, 2, 2, 130, 1, False), (2, 2, 1, 33, 129, False), (1, 12, 4, 5, 1000, False),
    (1, 2, 1, 40, 140, True), (1, 2, 1, 140, 40, True), (1, 4, 2, 3, 1025, True),
]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("B,hq,hkv,n,m,causal", CASES)
def test_attention_is_the_formula(gpu_device, swan_mod, torch_mod, B, hq, hkv, n, m, causal, dtype):
    torch = torch_mod
    q, k, v = _inputs(torch, gpu_device, B, hq, hkv, n, m, dtype, n + m)
    got = swan_mod.prompt_attention(q, k, v, causal=causal)
    torch.cuda.synchronize()
    _check(torch, got, q, k, v, causal, [n] * B, [m] * B, dtype)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("split", [False, True])
def test_ragged_batches_with_nans_behind_them(gpu_device, swan_mod, torch_mod, causal, dtype, split):
    """Lengths of zero and one among them; what lies past a sequence's rows is NaN and
    neither read nor written.  split: few rows over long keys (partials, then a join)."""
    torch = torch_mod
    n, m = (3, 900) if split else (150, 210)
    ns = [n, 0, 1, n, 2, n] if split else [150, 0, 1, 64, 65, 130]
    ms = [m, 5, 1, 0, 700, 257] if split else [210, 9, 1, 0, 65, 64]
    q, k, v = _inputs(torch, gpu_device, 6, 4, 2, n, m, dtype, 77)
    for b in range(6):
        q[b, :, ns[b]:] = math.nan
        k[b, :, ms[b]:] = math.nan
        v[b, :, ms[b]:] = math.nan
    out = torch.full_like(q, 5.0)
    swan_mod.prompt_attention(q, k, v, causal=causal, n=ns, m=ms, out=out)
    torch.cuda.synchronize()
    _check(torch, out, q, k, v, causal, ns, ms, dtype)
    for b in range(6):
        assert torch.all(out[b, :, ns[b]:] == 5.0)
    fresh = swan_mod.prompt_attention(q, k, v, causal=causal, n=ns, m=ms)
    for b in range(6):
        assert torch.equal(fresh[b, :, :ns[b]], out[b, :, :ns[b]])
        assert torch.all(fresh[b, :, ns[b]:] == 0)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n,m,causal", [(90, 90, True), (2, 1000, False), (70, 3, True)])
def test_continued_from_a_state(gpu_device, swan_mod, torch_mod, n, m, causal, dtype):
    """Rows with a state far below, beside and far above their scores, and without one."""
    torch = torch_mod
    q, k, v = _inputs(torch, gpu_device, 2, 4, 2, n, m, dtype, 5)
    g = torch.Generator().manual_seed(8)
    o = torch.randn(2, 4, n, D, generator=g).to(gpu_device)
    lse = (torch.randn(2, 4, n, generator=g) * 3).to(gpu_device)
    lse[0, 0] = -60.0
    lse[0, 1] = 60.0
    lse[1, 2] = -math.inf
    o[1, 2] = math.nan  # of no weight
    got = swan_mod.prompt_attention(q, k, v, causal=causal, state=(o, lse))
    o = torch.nan_to_num(o)
    _check(torch, got, q, k, v, causal, [n] * 2, [m] * 2, dtype, (o, lse))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("place", ["value", "key"])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_nothing_comes_from_what_a_row_does_not_see(gpu_device, swan_mod, torch_mod, what, place,
                                                     dtype):
    torch = torch_mod
    n = 150
    q, k, v = _inputs(torch, gpu_device, 1, 2, 1, n, n, dtype, 4)
    good = swan_mod.prompt_attention(q, k, v)
    where = k if place == "key" else v
    where[0, 0, 70, 3] = what
    where[0, 0, 133, 9] = what
    got = swan_mod.prompt_attention(q, k, v)
    torch.cuda.synchronize()
    assert torch.equal(got[:, :, :70], good[:, :, :70])
    if place == "value":
        # its own dimension alone, in the rows that see it
        other = [d for d in range(D) if d not in (3, 9)]
        assert torch.equal(got[..., other], good[..., other])
        assert not torch.isfinite(got[:, :, 70:, 3]).any()
        assert torch.equal(got[:, :, :133, 9], good[:, :, :133, 9])
        assert not torch.isfinite(got[:, :, 133:, 9]).any()
        if not math.isnan(what):
            assert torch.all(got[:, :, 70:, 3] == what)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_sharp_and_flat_softmax(gpu_device, swan_mod, torch_mod, dtype):
    """One key far above 30000 others that together weigh as much: p then lies between 2^-15
    and 2^-16 of the largest, and all of it counts; then keys whose scores grow."""
    torch = torch_mod
    m = 30000
    td = C.torch_dtype(dtype)
    q = torch.zeros(1, 1, 1, D, device=gpu_device, dtype=td)
    k = torch.zeros(1, 1, m, D, device=gpu_device, dtype=td)
    v = torch.ones(1, 1, m, D, device=gpu_device, dtype=td)
    q[..., 0] = 16.0
    k[:, :, 11, 0] = 7.25
    v[:, :, 11] = -1.0
    got = swan_mod.prompt_attention(q, k, v, causal=False)
    want, _ = R.softmax_rows(q[0, 0], k[0, 0], v[0, 0])
    tol = R.bound(dtype, q[0, 0], k[0, 0], v[0, 0], want, m)
    assert abs(want[0, 0].item()) < 0.1
    R.close(got[0, 0], want, tol, "flat tail")
    k[0, 0, :, 0] = torch.linspace(-50, 50, m).to(td)
    v[0, 0] = torch.randn(m, D, generator=torch.Generator().manual_seed(1)).to(td)
    got = swan_mod.prompt_attention(q, k, v, causal=False)
    want, _ = R.softmax_rows(q[0, 0], k[0, 0], v[0, 0])
    R.close(got[0, 0], want, R.bound(dtype, q[0, 0], k[0, 0], v[0, 0], want, m), "growing scores")


def test_scale_and_repeatability(gpu_device, swan_mod, torch_mod):
    torch = torch_mod
    q, k, v = _inputs(torch, gpu_device, 2, 4, 2, 100, 100, "f16", 6)
    a = swan_mod.prompt_attention(q, k, v, scale=0.25)
    b = swan_mod.prompt_attention((q.float() * 0.25 * math.sqrt(D) * 2).half() * 0.5, k, v)
    assert (a - b).abs().max().item() < 0.02
    for _ in range(5):
        assert torch.equal(a, swan_mod.prompt_attention(q, k, v, scale=0.25))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_a_row_has_its_bits_whatever_its_neighbours_are(gpu_device, swan_mod, torch_mod, dtype):
    """Rows beside it that are much larger, no numbers, or infinite."""
    torch = torch_mod
    q, k, v = _inputs(torch, gpu_device, 1, 2, 1, 150, 300, dtype, 12)
    want = swan_mod.prompt_attention(q, k, v)
    for other in (60.0, math.nan, math.inf):
        changed = q.clone()
        changed[:, :, 1::2] = changed[:, :, 1::2] * other
        got = swan_mod.prompt_attention(changed, k, v)
        assert torch.equal(got[:, :, 0::2], want[:, :, 0::2]), other


def test_on_another_stream_and_captured(gpu_device, swan_mod, torch_mod):
    """Single tokens (a workspace) and a prompt (none), captured in two graphs that are
    replayed in turn with eager calls between."""
    torch = torch_mod
    one = _inputs(torch, gpu_device, 2, 4, 2, 1, 900, "f16", 2)
    many = _inputs(torch, gpu_device, 2, 4, 2, 150, 150, "f16", 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = swan_mod.prompt_attention(*one, causal=False, stream=side)
    side.synchronize()
    assert torch.equal(got, swan_mod.prompt_attention(*one, causal=False))
    graphs = []
    for args, causal in ((one, False), (many, True), (one, False)):
        out = torch.zeros_like(args[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            swan_mod.prompt_attention(*args, causal=causal, out=out)
        graphs.append((graph, args, causal, out))
    for turn in range(3):
        one[0].mul_(0.9)
        many[2].add_(0.1)
        for graph, args, causal, out in graphs:
            out.zero_()
            graph.replay()
        for _, args, causal, out in graphs:
            assert torch.equal(out, swan_mod.prompt_attention(*args, causal=causal)), turn
