"""swan_copy_sequences: copies, forks, new orders, tokens left out, byte for byte as the
documented layout has them; calls on the copies give what the sources give."""
import pytest

from tests import rows_ref as R
from tests import swan_cases as C

pytestmark = pytest.mark.gpu
D = 128


def _tokens(torch, cache, b):
    """What the cache holds of sequence b: per head and role its rows as stored."""
    return [[R.cached_rows(cache, b, h, r) for r in (0, 1)] for h in range(cache.desc.n_kv_heads)]


def _without(torch, rows, first, drop):
    return torch.cat([rows[:first], rows[first + drop:]])


CASES = [  # lengths, hkv, buffer, k, of, first, drop, values, k_value
    ([200, 64, 0], 2, 16, [48, 48, 48], [2, 0, 0], 0, None, "same", None),
    ([200, 300, 150], 1, 32, [48] * 3, [1, 1, 0], 4, [100, 64, 0], "same", None),
    ([900, 500], 2, 100, [77, 77], [0, 1, 0, -1], 0, [700, 1, 64, 5], "same", [50, 50]),
    ([700, 300], 3, 0, [40, 40], [1, 0], [64, 3], [236, 697], "same", None),
    ([700, 300], 1, 128, [40, 40], [1, 0], [1, 65], [171, 300], "e4m3", None),
    ([20, 5], 2, 30, [40, 40], [1, 0], 0, None, "same", None),
]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("lengths,hkv,buffer,k,of,first,drop,values,k_value", CASES)
def test_copies_hold_the_tokens(gpu_device, swan_mod, torch_mod, lengths, hkv, buffer, k, of, first,
                                drop, values, k_value, dtype):
    torch = torch_mod
    if values == "e4m3" and dtype == "f32":
        return
    src, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, lengths, hkv, hkv, buffer, k, dtype, 7,
                                     values, k_value)
    dst = swan_mod.SwanCache(len(of), hkv, hkv, buffer, max(lengths) + 100, [k[0]] * len(of),
                             C.torch_dtype(dtype), gpu_device, sparse_values=values,
                             k_value=None if k_value is None else [k_value[0]] * len(of))
    for t in (dst.k_pages, dst.v_pages):
        t.fill_(0x55)
    for t in (dst.k_ring, dst.v_ring):
        t.fill_(7.0)
    dst.seq_len = [3] * len(of)
    before = [t.clone() for t in (src.k_pages, src.v_pages, src.k_ring, src.v_ring)]
    old = [t.clone() for t in (dst.k_pages, dst.v_pages, dst.k_ring, dst.v_ring)]
    dst.copy_from(src, of, first, drop)
    torch.cuda.synchronize()
    firsts = [first] * len(of) if isinstance(first, int) else first
    per = dst.k_pages.numel() // len(of), dst.v_pages.numel() // len(of)
    for b, p in enumerate(of):
        if p < 0:
            assert dst.seq_len[b] == 3
            assert torch.equal(dst.k_pages[b * per[0]:(b + 1) * per[0]],
                               old[0][b * per[0]:(b + 1) * per[0]])
            assert torch.equal(dst.v_ring[b], old[3][b])
            continue
        d = 0 if drop is None else drop[b]
        assert dst.seq_len[b] == lengths[p] - d
        got, want = _tokens(torch, dst, b), _tokens(torch, src, p)
        for h in range(hkv):
            for r in (0, 1):
                assert torch.equal(got[h][r], _without(torch, want[h][r], firsts[b], d)), (b, h, r)
        # the slots behind the last token
        S = max(0, dst.seq_len[b] - buffer)
        pages = (S + 63) // 64
        for x, (t, was) in enumerate(((dst.k_pages, old[0]), (dst.v_pages, old[1]))):
            unit = t[b * per[x]:(b + 1) * per[x]].view(hkv, -1)
            each = unit.shape[1] // ((dst.desc.sparse_capacity + 63) // 64)
            assert torch.all(unit[:, pages * each:] == 0x55)
            if S % 64:
                chunk = 8 if values == "e4m3" else 16
                last = unit[:, (pages - 1) * each:pages * each]
                assert torch.all(last[:, S % 64 * chunk:64 * chunk] == 0x55)
        if 0 < dst.seq_len[b] < buffer:
            assert torch.all(dst.k_ring[b, :, dst.seq_len[b]:] == 7.0)
    for t, was in zip((src.k_pages, src.v_pages, src.k_ring, src.v_ring), before):
        assert torch.equal(t, was)


@pytest.mark.parametrize("dtype,hq,hkv", [("f16", 4, 4), ("f16", 8, 2), ("f32", 4, 2)])
def test_copies_go_on_as_their_sources(gpu_device, swan_mod, torch_mod, dtype, hq, hkv):
    """Decode steps of a new order, and of sequences cut to their window, are the sources' bit
    for bit (the window's: the same tokens in other splits, so within two roundings)."""
    torch = torch_mod
    src, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [500, 80, 300], hq, hkv, 32, [48, 64, 48],
                                     dtype, 7, spare=100)
    new = src.select([2, 0, 2, 1])
    assert new.seq_len == [300, 500, 300, 80] and new.k_active == [48, 48, 48, 64]
    window, sinks = 100, 3
    cut = src.select([0, 1, 2], sinks, src.outside(window, sinks), sparse_capacity=300)
    assert cut.seq_len == [3 + 99, 80, 3 + 99]
    g = torch.Generator().manual_seed(1)
    td = C.torch_dtype(dtype)
    for i in range(70):
        k = torch.randn(3, hkv, 1, D, generator=g).to(td).to(gpu_device)
        v = torch.randn(3, hkv, 1, D, generator=g).to(td).to(gpu_device)
        q = torch.randn(3, hq, D, generator=g).to(td).to(gpu_device)
        pick = lambda t: t[[2, 0, 2, 1]].contiguous()  # noqa: E731
        whole = src.step(k, v, q, P_qk, P_vo)
        same = new.step(pick(k), pick(v), pick(q), P_qk, P_vo)
        assert (same.float() - pick(whole).float()).abs().max().item() <= \
            4 * R.HALF[dtype] * whole.float().abs().max().item() + 2.0 ** -18
        a = src.decode(q, P_qk, P_vo, window=window, sinks=sinks)
        b = cut.step(k, v, q, P_qk, P_vo, window=window, sinks=sinks)
        assert (a.float() - b.float()).abs().max().item() <= \
            4 * R.HALF[dtype] * a.float().abs().max().item() + 2.0 ** -18, i
    for x, y in ((0, 2), (1, 0), (3, 1)):
        for p, r in zip(_tokens(torch, new, x), _tokens(torch, src, y)):
            assert torch.equal(p[0], r[0]) and torch.equal(p[1], r[1])


def test_on_another_stream_and_captured(gpu_device, swan_mod, torch_mod):
    torch = torch_mod
    src, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [500, 80], 2, 2, 32, [48, 48], "f16", 7)
    side = torch.cuda.Stream()
    want = src.select([1, 0], 4, [0, 77])
    side.wait_stream(torch.cuda.current_stream())
    got = src.select([1, 0], 4, [0, 77], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for name in ("k_pages", "v_pages", "k_ring", "v_ring"):
        assert torch.equal(getattr(got, name), getattr(want, name))
    other = src.select([0, 1])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        other.copy_from(src, [1, 0], 4, [0, 77])
    for _ in range(3):
        for name in ("k_pages", "v_pages", "k_ring", "v_ring"):
            getattr(other, name).zero_()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("k_pages", "v_pages", "k_ring", "v_ring"):
            assert torch.equal(getattr(other, name), getattr(want, name)), name


def test_offsets_beyond_32_bits(gpu_device, swan_mod, torch_mod):
    """The last head's pages lie past 2^32 bytes in both caches."""
    torch = torch_mod
    hkv, tokens = 64, 700
    src = swan_mod.SwanCache(1, hkv, hkv, 16, 200000, [128], torch.float32, gpu_device)
    assert src.k_pages.numel() > 2**32
    g = torch.Generator().manual_seed(1)
    P = R.rotations(hkv, 3, gpu_device)
    rows = torch.randn(1, hkv, tokens, D, generator=g).to(gpu_device)
    src.append(rows, rows, P, P)
    dst = src.select([0], 3, [133])
    torch.cuda.synchronize()
    for h in (0, hkv - 1):
        for r in (0, 1):
            a, b = R.cached_rows(dst, 0, h, r), R.cached_rows(src, 0, h, r)
            assert torch.equal(a, _without(torch, b, 3, 133))


def test_a_source_dropped_at_once(gpu_device, swan_mod, torch_mod):
    """A copy on another stream than the source's memory, which is dropped while the copy
    waits: new tensors do not take its place before the copy has read it."""
    torch = torch_mod
    side = torch.cuda.Stream()
    src, _, _ = R.filled_cache(swan_mod, gpu_device, [3000, 2500], 8, 8, 64, [48, 48], "f16", 5)
    want = src.select([1, 0], 4, [0, 77])
    torch.cuda.synchronize()
    sizes = [t.numel() * t.element_size() for t in (src.k_pages, src.v_pages, src.k_ring, src.v_ring)]
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        got = src.select([1, 0], 4, [0, 77])
    del src
    others = [torch.full((n,), 0x3C, dtype=torch.uint8, device=gpu_device) for n in sizes * 2]
    torch.cuda.synchronize()
    for name in ("k_pages", "v_pages", "k_ring", "v_ring"):
        assert torch.equal(getattr(got, name), getattr(want, name)), name
    del others
