"""Calls on a stream that is not the current one: whose memory their results and workspaces
are, and when it is used again."""
import pytest

from tests import rows_ref as R

pytestmark = pytest.mark.gpu
D = 128


def _busy(torch, device):
    """Work of some milliseconds on the current stream."""
    a = torch.ones(4096, 4096, device=device)
    for _ in range(20):
        a = a @ a * 2.0 ** -12
    return a


def _caches(swan_mod, gpu_device):
    own, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [300, 40, 500], 8, 2, 16, [64] * 3, "f16",
                                     71)
    past, _, _ = R.filled_cache(swan_mod, gpu_device, [900], 8, 2, 16, [64], "f16", 72,
                                P=(P_qk, P_vo))
    return own, past, P_qk, P_vo


@pytest.mark.parametrize("call", ["decode", "decode prefix", "step", "attend", "prompt", "rows"])
def test_a_result_used_on_the_current_stream_and_dropped(gpu_device, swan_mod, torch_mod, call):
    """Its memory is not given to the call's stream again while the current one reads it."""
    torch = torch_mod
    own, past, P_qk, P_vo = _caches(swan_mod, gpu_device)
    g = torch.Generator().manual_seed(1)
    rows = torch.randn(3, 8, 1, D, generator=g).half().to(gpu_device)
    kv = torch.randn(3, 2, 1, D, generator=g).half().to(gpu_device)
    q = rows[:, :, 0].contiguous()
    qkv = torch.randn(3, 1, 12 * D, generator=g).half().to(gpu_device)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    run = {"decode": lambda: own.decode(q, P_qk, P_vo, stream=side),
           "decode prefix": lambda: own.decode(q, P_qk, P_vo, stream=side,
                                               prefix=swan_mod.Prefix(past)),
           "step": lambda: own.step(kv, kv, q, P_qk, P_vo, stream=side),
           "attend": lambda: own.attend(rows, P_qk, P_vo, stream=side)[0],
           "prompt": lambda: swan_mod.prompt_attention(rows, kv, kv, stream=side),
           "rows": lambda: swan_mod.qkv_rows(qkv, 8, 2, [0] * 3, 10000.0, stream=side)[0]}[call]
    result = run()
    side.synchronize()
    want = result.clone()
    torch.cuda.synchronize()
    keep = _busy(torch, gpu_device)
    kept = result.clone()  # behind the work above
    place, shape = result.data_ptr(), result.shape
    del result
    with torch.cuda.stream(side):
        others = [torch.full(shape, 7.0, dtype=want.dtype, device=gpu_device) for _ in range(50)]
    busy = not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert busy, "the current stream was done too early to show anything"
    assert all(t.data_ptr() != place for t in others)
    assert torch.equal(kept, want)
    del keep


def test_plain_calls_on_two_streams_at_once(gpu_device, swan_mod, torch_mod):
    """Decode calls of one cache, enqueued on two streams without waiting."""
    torch = torch_mod
    own, _, P_qk, P_vo = _caches(swan_mod, gpu_device)
    g = torch.Generator().manual_seed(2)
    qs = [torch.randn(3, 8, D, generator=g).half().to(gpu_device) for _ in range(2)]
    want = [own.decode(q, P_qk, P_vo) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            got[i].append(own.decode(qs[i], P_qk, P_vo, stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i]), i


def test_a_plan_that_grows_on_a_side_stream(gpu_device, swan_mod, torch_mod):
    """Decode calls on a side stream alone, of lengths that need more workspace from call to
    call, while the current stream makes, fills and reads tensors."""
    torch = torch_mod
    cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [6000, 3000], 8, 8, 16, [32] * 2, "f16",
                                       73)
    g = torch.Generator().manual_seed(3)
    q = torch.randn(2, 8, D, generator=g).half().to(gpu_device)
    lengths = [[n, n // 2] for n in (20, 100, 300, 1000, 3000, 6000)]
    want = []
    for cache.seq_len in lengths:
        want.append(cache.decode(q, P_qk, P_vo))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for turn in range(3):
        got, mine = [], []
        for i, cache.seq_len in enumerate(lengths):
            for _ in range(4):
                got.append((i, cache.decode(q, P_qk, P_vo, stream=side)))
                mine.append(torch.full((300, 1000), float(len(mine)), device=gpu_device))
        assert all(bool((t == n).all()) for n, t in enumerate(mine))
        side.synchronize()
        assert all(torch.equal(x, want[i]) for i, x in got), turn


def test_a_graph_beside_a_plan_that_grows(gpu_device, swan_mod, torch_mod):
    """Two captured decode calls of one cache, replayed on two streams at once, with eager
    calls that need more workspace, and other tensors, between."""
    torch = torch_mod
    cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [6000, 3000], 8, 8, 16, [32] * 2, "f16",
                                       74)
    g = torch.Generator().manual_seed(4)
    qs = [torch.randn(2, 8, D, generator=g).half().to(gpu_device) for _ in range(2)]
    cache.seq_len = [300, 200]
    want = [cache.decode(q, P_qk, P_vo) for q in qs]
    torch.cuda.synchronize()
    outs, graphs = [torch.zeros_like(q) for q in qs], []
    for q, out in zip(qs, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.decode(q, P_qk, P_vo, out=out)
        graphs.append(graph)
    cache.seq_len = [6000, 3000]
    longer = cache.decode(qs[0], P_qk, P_vo)
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    for turn in range(4):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        again = cache.decode(qs[0], P_qk, P_vo)
        mine = [torch.full((100, 1000), 3.0, device=gpu_device) for _ in range(8)]
        torch.cuda.synchronize()
        assert torch.equal(again, longer), turn
        assert all(bool((t == 3).all()) for t in mine), turn
        for out, x in zip(outs, want):
            assert torch.equal(out, x), turn


def test_change_k_and_rope_on_a_side_stream(gpu_device, swan_mod, torch_mod):
    """While the current stream is busy: pages cleared and converted on the side stream."""
    torch = torch_mod
    caches = []
    for stream in (None, torch.cuda.Stream()):
        cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [2000, 300], 8, 2, 16, [64] * 2,
                                           "f16", 75)
        x = torch.randn(2, 8, 50, D, generator=torch.Generator().manual_seed(5)).half().to(gpu_device)
        torch.cuda.synchronize()
        keep = _busy(torch, gpu_device)
        turned = swan_mod.rope(x, [3, 900], 10000.0, stream=stream)
        cache.change_k([40, 32], stream=stream)
        torch.cuda.synchronize()
        caches.append((cache, turned))
        del keep
    (a, x), (b, y) = caches
    assert torch.equal(x, y)
    assert torch.equal(a.k_pages, b.k_pages) and torch.equal(a.v_pages, b.v_pages)


def test_captured_on_a_stream_beside_the_capturing_one(gpu_device, swan_mod, torch_mod):
    """Calls on a side stream that joins a capture, results and workspaces of the graph's
    memory; one result is dropped inside the capture."""
    torch = torch_mod
    own, past, P_qk, P_vo = _caches(swan_mod, gpu_device)
    g = torch.Generator().manual_seed(6)
    q = torch.randn(3, 8, D, generator=g).half().to(gpu_device)
    prefix = swan_mod.Prefix(past)
    own.decode(q, P_qk, P_vo), own.decode(q, P_qk, P_vo, prefix=prefix)
    torch.cuda.synchronize()
    out, side, graph = torch.zeros(2, *q.shape, device=gpu_device).half(), torch.cuda.Stream(), \
        torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        current = torch.cuda.current_stream()
        side.wait_stream(current)
        a = own.decode(q, P_qk, P_vo, stream=side)
        b = own.decode(q, P_qk, P_vo, stream=side, prefix=prefix)
        current.wait_stream(side)
        out[0].copy_(a)
        out[1].copy_(b)
        del a
    for turn in range(4):
        q.mul_(0.9)
        out.zero_()
        graph.replay()
        want = own.decode(q, P_qk, P_vo), own.decode(q, P_qk, P_vo, prefix=prefix)
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), turn
