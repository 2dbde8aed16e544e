"""A sliding window over a cache: swan_attend_window (rows) and swan_decode_attention_window /
swan_decode_step_window (single tokens) against the formula in float64 on what the cache holds,
with and without a prefix."""
import math

import pytest

from tests import long_ref as LR
from tests import rows_ref as R

pytestmark = pytest.mark.gpu
D = 128


def _queries(torch, device, dtype, *shape, seed=0, sharp=3.0):
    g = torch.Generator().manual_seed(seed)
    from tests import swan_cases as C

    return (torch.randn(*shape, generator=g) * sharp).to(C.torch_dtype(dtype)).to(device)


def _prefix_rows(prefix, b, h):
    if prefix is None or prefix.of[b] < 0:
        return None
    return [R.cached_rows(prefix.cache, prefix.of[b], h, r) for r in (0, 1)]


def _check_decode(torch, cache, q, P_qk, P_vo, out, window, sinks, dtype, prefix=None):
    hkv, G = cache.desc.n_kv_heads, cache.desc.n_q_heads // cache.desc.n_kv_heads
    for b in range(cache.batch):
        for h in range(hkv):
            before = _prefix_rows(prefix, b, h)
            L = cache.seq_len[b] + (0 if before is None else before[0].shape[0])
            p = torch.full((G,), L - 1, device=q.device)
            rows = q[b, h * G:(h + 1) * G]
            want, _, (t, K, V) = LR.cached_attention(cache, b, h, rows, P_qk, P_vo, p, window,
                                                     sinks, before)
            tol = R.bound(dtype, t, K, V, want, L, turned=P_vo is not None)
            R.close(out[b, h * G:(h + 1) * G], want, tol, f"sequence {b}, kv head {h}")


DECODE = [  # lengths, hq, hkv, buffer, k, window, sinks, values, k_value
    ([1], 1, 1, 16, [64], 1, 0, "same", None),
    ([5, 20], 4, 4, 8, [48, 48], 3, 1, "same", None),
    ([300, 17], 4, 4, 16, [64, 64], 100, 4, "same", None),
    ([700], 8, 2, 64, [64], 200, 70, "same", None),
    ([700, 64, 129], 8, 2, 0, [40, 40, 40], 129, 4, "same", None),
    ([600, 601, 3], 16, 2, 128, [50, 20, 128], 64, 3, "same", None),
    ([520, 130], 6, 3, 100, [77, 30], 300, 0, "same", [51, 90]),
    ([520, 333], 5, 5, 30, [16, 120], 77, 130, "same", None),
    ([900], 8, 1, 64, [64], 10**9, 5, "same", None),
    ([900, 257], 8, 2, 64, [64, 96], 256, 64, "e4m3", None),
    ([450, 257], 3, 3, 16, [33, 8], 100, 1, "e4m3", [8, 40]),
    ([130], 2, 1, 200, [64], 40, 3, "same", None),
    ([1000], 2, 1, 300, [64], 40, 320, "same", None),
]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("lengths,hq,hkv,buffer,k,window,sinks,values,k_value", DECODE)
def test_decode_is_the_formula(gpu_device, swan_mod, torch_mod, lengths, hq, hkv, buffer, k, window,
                               sinks, values, k_value, dtype):
    torch = torch_mod
    if values == "e4m3" and dtype == "f32":
        return
    cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, lengths, hq, hkv, buffer, k, dtype, 7,
                                       values, k_value)
    q = _queries(torch, gpu_device, dtype, len(lengths), hq, D, seed=3)
    for P in (P_vo, None):
        out = cache.decode(q, P_qk, P, window=window, sinks=sinks)
        torch.cuda.synchronize()
        _check_decode(torch, cache, q, P_qk, P, out, window, sinks, dtype)


@pytest.mark.parametrize("dtype,hq,hkv", [("f16", 4, 4), ("f16", 8, 2), ("f16", 24, 2), ("f32", 4, 2)])
def test_a_step_is_append_and_decode(gpu_device, swan_mod, torch_mod, dtype, hq, hkv):
    """Bit for bit, from an empty cache over the end of the window and the first keys."""
    torch = torch_mod
    a, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [0, 0], hq, hkv, 8, [48, 24], dtype, 7,
                                   spare=200)
    b, _, _ = R.filled_cache(swan_mod, gpu_device, [0, 0], hq, hkv, 8, [48, 24], dtype, 7, spare=200)
    for i in range(100):
        k = _queries(torch, gpu_device, dtype, 2, hkv, 1, D, seed=3 * i, sharp=1)
        v = _queries(torch, gpu_device, dtype, 2, hkv, 1, D, seed=3 * i + 1, sharp=1)
        q = _queries(torch, gpu_device, dtype, 2, hq, D, seed=3 * i + 2)
        got = a.step(k, v, q, P_qk, P_vo, window=30, sinks=3)
        b.append(k, v, P_qk, P_vo)
        want = b.decode(q, P_qk, P_vo, window=30, sinks=3)
        assert torch.equal(got, want), i
        if i in (0, 7, 8, 29, 30, 40, 72, 99):
            _check_decode(torch, a, q, P_qk, P_vo, got, 30, 3, dtype)
    assert a.seq_len == b.seq_len == [100, 100]
    assert torch.equal(a.k_pages, b.k_pages) and torch.equal(a.v_ring, b.v_ring)


@pytest.mark.parametrize("dtype,hq,hkv", [("f16", 4, 4), ("f16", 8, 2), ("f32", 4, 2)])
@pytest.mark.parametrize("window,sinks", [(40, 4), (300, 0), (700, 200), (1, 0), (10**6, 9)])
def test_decode_behind_a_prefix(gpu_device, swan_mod, torch_mod, dtype, hq, hkv, window, sinks):
    torch = torch_mod
    base, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [300, 150], hq, hkv, 32, [64, 40], dtype,
                                      7)
    own, _, _ = R.filled_cache(swan_mod, gpu_device, [200, 17, 5, 0], hq, hkv, 16, [64] * 4, dtype, 9,
                               P=(P_qk, P_vo))
    prefix = swan_mod.Prefix(base, [0, 1, -1, 0])
    q = _queries(torch, gpu_device, dtype, 4, hq, D, seed=3)
    out = own.decode(q, P_qk, P_vo, prefix=prefix, window=window, sinks=sinks)
    torch.cuda.synchronize()
    _check_decode(torch, own, q, P_qk, P_vo, out, window, sinks, dtype, prefix)
    k = _queries(torch, gpu_device, dtype, 4, hkv, 1, D, seed=5, sharp=1)
    out = own.step(k, k, q, P_qk, P_vo, prefix=prefix, window=window, sinks=sinks)
    torch.cuda.synchronize()
    assert own.seq_len == [201, 18, 6, 1]
    _check_decode(torch, own, q, P_qk, P_vo, out, window, sinks, dtype, prefix)


ROWS = [  # lengths, hq, hkv, n, buffer, k, window, sinks, values
    ([1], 1, 1, 1, 16, [64], 1, 0, "same"),
    ([200, 50], 4, 2, 7, 16, [64, 40], 30, 4, "same"),
    ([700, 3], 8, 2, 70, 64, [64, 64], 200, 70, "same"),
    ([400], 4, 4, 150, 0, [50], 64, 64, "same"),
    ([500, 130, 64], 8, 1, 33, 100, [64, 16, 128], 90, 130, "same"),
    ([900, 300], 4, 1, 100, 128, [64, 64], 500, 3, "e4m3"),
    ([640], 2, 2, 300, 64, [64], 100, 0, "same"),
    ([640], 8, 1, 64, 300, [64], 100, 330, "same"),
    ([300], 2, 1, 20, 16, [64], 10**9, 0, "same"),
]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("lengths,hq,hkv,n,buffer,k,window,sinks,values", ROWS)
def test_rows_over_a_cache_are_the_formula(gpu_device, swan_mod, torch_mod, lengths, hq, hkv, n,
                                           buffer, k, window, sinks, values, dtype):
    """The states, and a chunk that goes on from them."""
    torch = torch_mod
    if values == "e4m3" and dtype == "f32":
        return
    cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, lengths, hq, hkv, buffer, k, dtype, 7,
                                       values)
    B, G = len(lengths), hq // hkv
    q = _queries(torch, gpu_device, dtype, B, hq, n, D, seed=3)
    kn = _queries(torch, gpu_device, dtype, B, hkv, n, D, seed=4, sharp=1)
    vn = _queries(torch, gpu_device, dtype, B, hkv, n, D, seed=5, sharp=1)
    ns = [n if b != 1 else (n + 1) // 2 for b in range(B)]
    o, lse = cache.attend(q, P_qk, None, n=ns, window=window, sinks=sinks)
    both = swan_mod.prompt_attention(q, kn, vn, n=ns, m=ns, state=(o, lse), window=window,
                                     sinks=[max(0, sinks - L) for L in lengths])
    torch.cuda.synchronize()
    for b in range(B):
        p = torch.arange(ns[b], device=gpu_device) + lengths[b]
        for h in range(hkv):
            for x in range(h * G, (h + 1) * G):
                rows = q[b, x, :ns[b]]
                want, wl, (t, K, V) = LR.cached_attention(cache, b, h, rows, P_qk, None, p, window,
                                                          sinks)
                tol = R.bound(dtype, t, K, V, want, lengths[b], "f32")
                R.close(o[b, x, :ns[b]], want, tol, f"sequence {b}, head {x}")
                none = torch.isinf(wl)
                assert torch.equal(torch.isinf(lse[b, x, :ns[b]]), none)
                d = (lse[b, x, :ns[b]].double() - wl)[~none].abs()
                assert not d.numel() or d.max().item() <= LR.lse_bound(t, K)
                chunk = (kn[b, h, :ns[b]], vn[b, h, :ns[b]])
                want, _, (t, K, V) = LR.cached_attention(cache, b, h, rows, P_qk, None, p, window,
                                                         sinks, None, chunk)
                tol = R.bound(dtype, t, K, V, want, K.shape[0])
                tol = tol + R.bound(dtype, t, K, V, want, K.shape[0], "f32")  # (two parts joined)
                R.close(both[b, x, :ns[b]], want, tol, f"chunk, sequence {b}, head {x}")
        assert torch.all(o[b, :, ns[b]:] == 0)


@pytest.mark.parametrize("dtype,hq,hkv", [("f16", 4, 4), ("f16", 16, 2), ("f32", 4, 2)])
@pytest.mark.parametrize("window,sinks", [(40, 4), (300, 0), (260, 170), (700, 1000)])
def test_rows_behind_a_prefix(gpu_device, swan_mod, torch_mod, dtype, hq, hkv, window, sinks):
    """Sequences of other lengths behind one prefix, whose rows share its tiles; one sequence
    behind none; two over one cache."""
    torch = torch_mod
    base, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [300, 150], hq, hkv, 32, [64, 40], dtype,
                                      7)
    own, _, _ = R.filled_cache(swan_mod, gpu_device, [200, 17, 0], hq, hkv, 16, [64] * 3, dtype, 9,
                               P=(P_qk, P_vo))
    prefix, of = swan_mod.Prefix(base, [0, 0, -1, 1, 0]), [0, 1, 0, 2, 0]
    n, G = 21, hq // hkv
    q = _queries(torch, gpu_device, dtype, 5, hq, n, D, seed=3)
    o, lse = own.attend(q, P_qk, P_vo, of=of, prefix=prefix, window=window, sinks=sinks)
    torch.cuda.synchronize()
    for b in range(5):
        for h in range(hkv):
            before = _prefix_rows(prefix, b, h)
            L = own.seq_len[of[b]] + (0 if before is None else before[0].shape[0])
            p = torch.arange(n, device=gpu_device) + L
            for x in range(h * G, (h + 1) * G):
                want, _, (t, K, V) = LR.cached_attention(own, of[b], h, q[b, x], P_qk, P_vo, p,
                                                         window, sinks, before)
                R.close(o[b, x], want, R.bound(dtype, t, K, V, want, L, "f32", turned=True),
                        f"sequence {b}, head {x}")


def _poison(torch, cache, b, tokens, what):
    """Every value byte pair of these pruned tokens becomes `what` in both roles."""
    kp = [(k + 7) // 8 * 8 for k in (cache.k_active[b], (cache.k_value or cache.k_active)[b])]
    npc = (cache.desc.sparse_capacity + 63) // 64
    size = 4 if cache.dtype == torch.float32 else 2
    for pages, k, ks in ((cache.k_pages, kp[0], cache.k_active),
                         (cache.v_pages, kp[1], cache.k_value or cache.k_active)):
        first = sum((x + 7) // 8 * 8 * 64 * (size + 1) * npc * cache.desc.n_kv_heads for x in ks[:b])
        unit = pages[first:first + cache.desc.n_kv_heads * npc * k * 64 * (size + 1)]
        unit = unit.view(cache.desc.n_kv_heads, npc, -1)
        vals = unit[..., :64 * k * size].view(cache.desc.n_kv_heads, npc, k * size // 16, 64, 16)
        for t in tokens:
            row = torch.full((16 // size,), what, dtype=cache.dtype, device=pages.device)
            vals[:, t // 64, :, t % 64] = row.view(torch.uint8)


@pytest.mark.parametrize("dtype,hq,hkv", [("f16", 4, 4), ("f16", 8, 2), ("f32", 4, 2)])
@pytest.mark.parametrize("what", [math.inf, math.nan])
def test_nothing_comes_from_hidden_tokens(gpu_device, swan_mod, torch_mod, dtype, hq, hkv, what):
    """Tokens between the first ones and the window that hold infinities or NaNs (in a page, in
    the ring): decode does not see them, nor do the rows of a chunk that are past them."""
    torch = torch_mod
    window, sinks, L = 40, 4, 400
    for buffer in (16, 100):
        made = lambda: R.filled_cache(swan_mod, gpu_device, [L, 90], hq, hkv, buffer, [64, 64], dtype,  # noqa: E731
                                      7)
        good, P_qk, P_vo = made()
        bad, _, _ = made()
        q = _queries(torch, gpu_device, dtype, 2, hq, D, seed=3)
        rows = _queries(torch, gpu_device, dtype, 2, hq, 60, D, seed=4)
        hidden = [5, 63, 64, 200, 299] + ([L - window - 1] if buffer == 16 else [])
        _poison(torch, bad, 0, hidden, what)
        if buffer == 100:
            slot = (L - window - 1) % buffer
            bad.k_ring[0, :, slot] = what
            bad.v_ring[0, :, slot] = what
        want = good.decode(q, P_qk, P_vo, window=window, sinks=sinks)
        assert torch.equal(bad.decode(q, P_qk, P_vo, window=window, sinks=sinks), want)
        want = good.attend(rows, P_qk, P_vo, window=window, sinks=sinks)
        got = bad.attend(rows, P_qk, P_vo, window=window, sinks=sinks)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        # tokens that the first rows of a chunk see and the later ones do not
        at = L - 20
        if buffer == 16:
            _poison(torch, bad, 0, [at], what)
        else:
            bad.v_ring[0, :, at % buffer] = what
            bad.k_ring[0, :, at % buffer] = what
        got = bad.attend(rows, P_qk, None, window=window, sinks=sinks)
        want = good.attend(rows, P_qk, None, window=window, sinks=sinks)
        last = at + window - 1 - L  # the last row that sees it
        assert torch.equal(got[0][0, :, last + 1:], want[0][0, :, last + 1:])
        assert torch.equal(got[0][1], want[0][1])
        assert not torch.isfinite(got[0][0, :, :last + 1]).all()


def test_infinite_values_reach_the_rows_that_see_them(gpu_device, swan_mod, torch_mod):
    """A value that is infinite in one dim: infinite there in the rows that see it, and the
    other dims keep their results."""
    torch = torch_mod
    for dtype in ("f16", "f32"):
        made = lambda: R.filled_cache(swan_mod, gpu_device, [300], 4, 2, 100, [64], dtype, 7)  # noqa: E731
        good, P_qk, _ = made()
        bad, _, _ = made()
        rows = _queries(torch, gpu_device, dtype, 1, 4, 60, D, seed=4, sharp=1)
        at = 280
        bad.v_ring[0, :, at % 100, 9] = math.inf
        want = good.attend(rows, P_qk, None, window=40)[0]
        got = bad.attend(rows, P_qk, None, window=40)[0]
        last = at + 39 - 300
        keep = [d for d in range(D) if d != 9]
        assert torch.equal(got[..., keep], want[..., keep])
        assert torch.all(got[0, :, :last + 1, 9] == math.inf)
        assert torch.equal(got[0, :, last + 1:], want[0, :, last + 1:])


def test_a_window_over_everything_is_no_window(gpu_device, swan_mod, torch_mod):
    """Rows over a cache: bit for bit.  Decode: within the bound (other splits)."""
    torch = torch_mod
    cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [500, 90], 8, 2, 64, [64, 64], "f16", 7)
    rows = _queries(torch, gpu_device, "f16", 2, 8, 30, D, seed=4)
    a = cache.attend(rows, P_qk, P_vo)
    for window, sinks in ((1000, 0), (1, 530)):
        b = cache.attend(rows, P_qk, P_vo, window=window, sinks=sinks)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_calls_on_another_stream_and_captured(gpu_device, swan_mod, torch_mod):
    torch = torch_mod
    cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [900, 90], 8, 2, 64, [64, 64], "f16", 7)
    q = _queries(torch, gpu_device, "f16", 2, 8, D, seed=3)
    rows = _queries(torch, gpu_device, "f16", 2, 8, 30, D, seed=4)
    want = cache.decode(q, P_qk, P_vo, window=300, sinks=4)
    state = cache.attend(rows, P_qk, P_vo, window=300, sinks=4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = cache.decode(q, P_qk, P_vo, stream=side, window=300, sinks=4)
    got2 = cache.attend(rows, P_qk, P_vo, stream=side, window=300, sinks=4)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(got2[0], state[0])
    graphs, outs = [], []
    for sinks in (4, 0):  # two graphs: workspaces of their own
        graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(q)
        with torch.cuda.graph(graph, stream=side):
            cache.decode(q, P_qk, P_vo, out=out, window=300, sinks=sinks)
            s = cache.attend(rows, P_qk, P_vo, window=300, sinks=sinks)
        graphs.append(graph)
        outs.append((out, s))
    wants = [(want, state), (cache.decode(q, P_qk, P_vo, window=300),
                             cache.attend(rows, P_qk, P_vo, window=300))]
    for _ in range(3):
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (out, s), (w, ws) in zip(outs, wants):
            assert torch.equal(out, w) and torch.equal(s[0], ws[0]) and torch.equal(s[1], ws[1])
        cache.decode(q, P_qk, P_vo, window=17)


def test_many_sequences_of_all_k(gpu_device, swan_mod, torch_mod):
    """64 sequences, every k_pad among them, most shorter than the window."""
    torch = torch_mod
    lengths = [1 + 7 * b for b in range(64)]
    ks = [1 + 2 * b for b in range(64)]
    for hq, hkv in ((2, 2), (4, 2)):
        cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, lengths, hq, hkv, 10, ks, "f16", 7)
        q = _queries(torch, gpu_device, "f16", 64, hq, D, seed=3)
        out = cache.decode(q, P_qk, P_vo, window=150, sinks=2)
        torch.cuda.synchronize()
        _check_decode(torch, cache, q, P_qk, P_vo, out, 150, 2, "f16")


def test_pages_beyond_32_bit_offsets(gpu_device, swan_mod, torch_mod):
    """The last head's pages lie past 2^32 bytes: decode, a step and rows see them."""
    torch = torch_mod
    hkv, tokens, capacity = 64, 300, 200000
    cache = swan_mod.SwanCache(1, hkv, hkv, 16, capacity, [128], torch.float32, gpu_device)
    assert cache.k_pages.numel() > 2**32
    P = R.rotations(hkv, 3, gpu_device)
    g = torch.Generator().manual_seed(1)
    rows = torch.randn(1, hkv, tokens, D, generator=g).to(gpu_device)
    cache.append(rows, rows, P, P)
    small = swan_mod.SwanCache(1, hkv, hkv, 16, 400, [128], torch.float32, gpu_device)
    small.append(rows, rows, P, P)
    q = _queries(torch, gpu_device, "f32", 1, hkv, D, seed=3, sharp=1)
    many = _queries(torch, gpu_device, "f32", 1, hkv, 40, D, seed=4, sharp=1)
    for window, sinks in ((100, 4), (250, 0)):
        assert torch.equal(cache.decode(q, P, P, window=window, sinks=sinks),
                           small.decode(q, P, P, window=window, sinks=sinks))
        a = cache.attend(many, P, P, window=window, sinks=sinks)
        b = small.attend(many, P, P, window=window, sinks=sinks)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    k = torch.randn(1, hkv, 1, D, generator=g).to(gpu_device)
    assert torch.equal(cache.step(k, k, q, P, P, window=100, sinks=4),
                       small.step(k, k, q, P, P, window=100, sinks=4))


def test_calls_that_are_refused(gpu_device, swan_mod, torch_mod):
    torch = torch_mod
    cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [90], 4, 2, 16, [64], "f16", 7)
    q = _queries(torch, gpu_device, "f16", 1, 4, D)
    rows = _queries(torch, gpu_device, "f16", 1, 4, 3, D)
    lengths, ring = list(cache.seq_len), cache.k_ring.clone()
    kv = _queries(torch, gpu_device, "f16", 1, 2, 1, D)
    for kw in (dict(window=0), dict(window=-1), dict(window=4, sinks=-1), dict(sinks=3),
               dict(window=4, sinks=70000), dict(window=2.5), dict(window=4, sinks=[1])):
        for call in (lambda: cache.decode(q, P_qk, P_vo, **kw),
                     lambda: cache.step(kv, kv, q, P_qk, P_vo, **kw),
                     lambda: cache.attend(rows, P_qk, P_vo, **kw)):
            with pytest.raises(swan_mod.SwanError):
                call()
    with pytest.raises(swan_mod.SwanError):
        swan_mod.prompt_attention(rows, rows, rows, causal=False, window=3)
    with pytest.raises(swan_mod.SwanError):
        cache.copy_from(cache, [0])
    with pytest.raises(swan_mod.SwanError):
        cache.select([0], 0, [75])  # 74 tokens are pruned
    with pytest.raises(ValueError):
        cache.select([1])
    torch.cuda.synchronize()
    assert cache.seq_len == lengths and torch.equal(cache.k_ring, ring)
