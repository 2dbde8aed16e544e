"""Rows over cached tokens (swan_attend) and decode steps behind a shared prefix, against
the formula in float64 on the rows that the caches hold."""
import math

import pytest

from tests import rows_ref as R
from tests import swan_cases as C

pytestmark = pytest.mark.gpu
D = 128


def _queries(torch, device, shape, dtype, seed, sharp=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * sharp).to(C.torch_dtype(dtype)).to(device)


def _held(sources, b, h, role):
    """The rows of all tokens that query sequence b sees in kv head h."""
    import torch

    rows = [R.cached_rows(c, of[b], h, role) for c, of in sources if of[b] >= 0]
    return torch.cat(rows) if rows else torch.zeros(0, D, dtype=torch.float64)


def _want(sources, q, b, hq, G, P_qk, P_vo, state=None):
    """o, lse of rows q [n][D] over the sources' tokens; the rows turned to P's basis."""
    h = hq // G
    K, V = (_held(sources, b, h, r).to(q.device) for r in (0, 1))
    qh = q.double() @ P_qk[h].double()
    o, lse = R.softmax_rows(qh, K, V, None, state)
    if P_vo is not None:
        o = o @ P_vo[h].double().T
    return o, lse, K, V


FORMATS = [("f16", "same"), ("f16", "e4m3"), ("f32", "same")]
# hq, hkv, buffer, k, k_value, lengths of the caches, of per query sequence, n, rows used
ATTEND = [
    (1, 1, 16, 8, None, [1], [0], 1, None),
    (4, 2, 16, 24, None, [15, 17], [0, 1], 3, None),
    (2, 2, 0, 1, None, [64], [0, 0, 0], 5, [5, 0, 1]),
    (8, 2, 128, 64, None, [128, 700, 0], [0, 1, 2, -1, 1], 40, [40, 7, 40, 40, 33]),
    (6, 2, 16, 77, 51, [300], [0] * 7, 33, None),
    (16, 1, 3, 128, None, [67, 66], [1, 0, 1], 20, None),
    (5, 1, 64, 13, 96, [1500], [0, 0], 1, None),
    (4, 4, 70, 40, None, [200, 90], [0, 1], 129, [129, 128]),
]


@pytest.mark.parametrize("dtype,values", FORMATS)
@pytest.mark.parametrize("hq,hkv,buffer,k,k_value,lengths,of,n,rows", ATTEND)
@pytest.mark.parametrize("absorbed", [False, True])
def test_attend_is_the_formula(gpu_device, swan_mod, torch_mod, hq, hkv, buffer, k, k_value,
                               lengths, of, n, rows, dtype, values, absorbed):
    torch = torch_mod
    cache, P_qk, P_vo = R.filled_cache(
        swan_mod, gpu_device, lengths, hq, hkv, buffer, [k] * len(lengths), dtype, 3, values,
        None if k_value is None else [k_value] * len(lengths))
    P_vo = None if absorbed else P_vo
    B = len(of)
    q = _queries(torch, gpu_device, (B, hq, n, D), dtype, 5)
    used = rows or [n] * B
    for b in range(B):
        q[b, :, used[b]:] = math.nan
    out = (torch.full((B, hq, n, D), 3.0, device=gpu_device),
           torch.full((B, hq, n), 3.0, device=gpu_device))
    o, lse = cache.attend(q, P_qk, P_vo, of=of, n=rows, out=out)
    torch.cuda.synchronize()
    for b in range(B):
        assert torch.all(o[b, :, used[b]:] == 3) and torch.all(lse[b, :, used[b]:] == 3)
        for h in range(hq):
            if used[b] == 0:
                continue
            got, glse = o[b, h, :used[b]], lse[b, h, :used[b]]
            rows_b = q[b, h, :used[b]]
            want, wlse, K, V = _want([(cache, of)], rows_b, b, h, hq // hkv, P_qk, P_vo)
            if not len(K):
                assert torch.all(got == 0) and torch.all(glse == -math.inf)
                continue
            # p is rounded as the format says, the state is float32
            tol = R.bound(dtype, rows_b, K, V, want, len(K), "f32", turned=not absorbed)
            R.close(got, want, tol, f"sequence {b}, head {h}")
            norms = rows_b.double().norm(dim=-1).max() * K.norm(dim=-1).max() / math.sqrt(D)
            err = 2.0 ** -16 * norms.item() + 2.0 ** -10 * (dtype == "f16") + 2.0 ** -17
            R.close(glse, wlse, err + 0 * wlse, "lse")


@pytest.mark.parametrize("dtype,values", FORMATS)
@pytest.mark.parametrize("k,k_value", [(48, 64), (100, 96)])
def test_many_rows_of_a_sequence(gpu_device, swan_mod, torch_mod, k, k_value, dtype, values):
    """Chunks that fill workgroups of 256 rows, the last ones partly; few and many components
    per page, and buffers that are not whole tiles."""
    torch = torch_mod
    hq, hkv, lengths, of = 32, 8, [1100, 1001, 1150, 60], [0, 1, 2, 0, 2, 1, 3, 2]
    used = [100, 99, 130, 100, 1, 65, 128, 97]
    cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, lengths, hq, hkv, 60, [k] * 4, dtype,
                                       4, values, [k_value] * 4)
    q = _queries(torch, gpu_device, (8, hq, 130, D), dtype, 9)
    o, lse = cache.attend(q, P_qk, P_vo, of=of, n=used)
    for b in range(8):
        for h in range(0, hq, 3):
            rows = q[b, h, :used[b]]
            want, wlse, K, V = _want([(cache, of)], rows, b, h, hq // hkv, P_qk, P_vo)
            tol = R.bound(dtype, rows, K, V, want, len(K), "f32", turned=True)
            R.close(o[b, h, :used[b]], want, tol, f"sequence {b}, head {h}")
            norms = rows.double().norm(dim=-1).max() * K.norm(dim=-1).max() / math.sqrt(D)
            err = 2.0 ** -16 * norms.item() + 2.0 ** -10 * (dtype == "f16") + 2.0 ** -17
            R.close(lse[b, h, :used[b]], wlse, err + 0 * wlse, "lse")


@pytest.mark.parametrize("dtype,values", FORMATS)
def test_two_sources_and_the_chunk_itself(gpu_device, swan_mod, torch_mod, dtype, values):
    """A shared prefix, the sequences' own tokens, then the chunk's rows, causal: as the
    softmax over all of them; the prefix of another format of the same element type."""
    torch = torch_mod
    hq, hkv, B, n = 8, 2, 3, 70
    own, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [100, 0, 333], hq, hkv, 16, [24, 32, 48],
                                     dtype, 1, values, spare=100)
    other = "same" if values == "e4m3" or dtype == "f32" else "e4m3"
    past, _, _ = R.filled_cache(swan_mod, gpu_device, [500, 65], hq, hkv, 64, [40, 64], dtype, 2,
                                other, P=(P_qk, P_vo))
    prefix = swan_mod.Prefix(past, [1, 0, -1])
    used = [70, 64, 1]
    q = _queries(torch, gpu_device, (B, hq, n, D), dtype, 6)
    k = _queries(torch, gpu_device, (B, hkv, n, D), dtype, 7, 0.5)
    v = _queries(torch, gpu_device, (B, hkv, n, D), dtype, 8, 1.0)
    state = own.attend(q, P_qk, P_vo, n=used, prefix=prefix)
    got = swan_mod.prompt_attention(q, k, v, n=used, m=used, state=state)
    torch.cuda.synchronize()
    sources = [(past, prefix.of), (own, [0, 1, 2])]
    for b in range(B):
        for h in range(hq):
            rows = q[b, h, :used[b]]
            o, lse, K, V = _want(sources, rows, b, h, hq // hkv, P_qk, P_vo)
            kb, vb = k[b, h // 4, :used[b]], v[b, h // 4, :used[b]]
            seen = torch.ones(used[b], used[b], dtype=torch.bool, device=gpu_device).tril()
            want, _ = R.softmax_rows(rows, kb, vb, seen, (o, lse))
            tol = R.bound(dtype, rows, kb, vb, want, len(K) + used[b])
            if len(K):
                tol = tol + R.bound(dtype, rows, K, V, o, len(K), "f32", turned=True)
            R.close(got[b, h, :used[b]], want, tol, f"sequence {b}, head {h}")


DECODE = [  # hq, hkv, prefix lengths, of, own lengths, buffer of prefix, own, k
    (1, 1, [1], [0], [0], 4, 4, [8]),
    (4, 4, [200], [0, 0, 0], [1, 0, 40], 16, 16, [24] * 3),
    (8, 2, [1000, 64], [0, 1, -1, 0, 1], [300, 0, 77, 128, 1], 64, 128, [64] * 5),
    (16, 2, [300], [0] * 9, [5] * 9, 0, 0, [40] * 9),
    (16, 1, [90], [0, 0], [3, 30], 16, 16, [20, 20]),
    (12, 1, [700], [0] * 40, [1] * 40, 32, 16, [128] * 40),
    (32, 8, [2049], [0] * 4, [70, 71, 72, 0], 128, 64, [32, 48, 64, 96]),
    (6, 2, [0, 129], [0, 1], [9, 0], 128, 8, [33, 51]),
    (4, 4, [500], [0, 0, -1], [200, 0, 150], 32, 32, [32, 64, 96]),
]


@pytest.mark.parametrize("dtype,values", FORMATS)
@pytest.mark.parametrize("hq,hkv,plen,of,lens,pbuf,buffer,k", DECODE)
@pytest.mark.parametrize("absorbed", [False, True])
def test_decode_behind_a_prefix(gpu_device, swan_mod, torch_mod, hq, hkv, plen, of, lens, pbuf,
                                buffer, k, dtype, values, absorbed):
    torch = torch_mod
    own, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, lens, hq, hkv, buffer, k, dtype, 11,
                                     values)
    past, _, _ = R.filled_cache(swan_mod, gpu_device, plen, hq, hkv, pbuf, [48] * len(plen), dtype,
                                12, values, k_value=[30] * len(plen), P=(P_qk, P_vo))
    P_vo = None if absorbed else P_vo
    B = len(of)
    prefix = swan_mod.Prefix(past, of)
    q = _queries(torch, gpu_device, (B, hq, D), dtype, 13)
    out = own.decode(q, P_qk, P_vo, prefix=prefix)
    torch.cuda.synchronize()

    def check(out, q):
        sources = [(past, of), (own, list(range(B)))]
        for b in range(B):
            for h in range(hq):
                rows = q[b, h][None]
                want, _, K, V = _want(sources, rows, b, h, hq // hkv, P_qk, P_vo)
                tol = R.bound(dtype, rows, K, V, want, len(K), turned=not absorbed)
                R.close(out[b, h][None], want, tol, f"sequence {b}, head {h}")

    check(out, q)
    # a step: the same append as without a prefix, then attention over both
    plain = swan_mod.SwanCache(B, hq, hkv, buffer, own.desc.sparse_capacity, k, own.dtype,
                               gpu_device, sparse_values=values)
    for name in ("k_pages", "v_pages", "k_ring", "v_ring"):
        getattr(plain, name).copy_(getattr(own, name))
    plain.seq_len = list(own.seq_len)
    q2 = _queries(torch, gpu_device, (B, hq, D), dtype, 14)
    new = [_queries(torch, gpu_device, (B, hkv, 1, D), dtype, 15 + r, 1.0) for r in (0, 1)]
    out = own.step(*new, q2, P_qk, P_vo, prefix=prefix)
    plain.step(*new, q2, P_qk, P_vo)
    torch.cuda.synchronize()
    assert own.seq_len == plain.seq_len == [L + 1 for L in lens]
    for name in ("k_pages", "v_pages", "k_ring", "v_ring"):
        assert torch.equal(getattr(own, name), getattr(plain, name)), name
    check(out, q2)


def test_the_same_as_a_copy_for_every_sequence(gpu_device, swan_mod, torch_mod):
    """Behind an unpruned prefix (k = 128) and before it: decode over one cache that holds
    prefix and own tokens alike gives the same up to rounding."""
    torch = torch_mod
    hq, hkv, B = 8, 2, 4
    P = (R.rotations(hkv, 1, gpu_device), R.rotations(hkv, 2, gpu_device))
    g = torch.Generator().manual_seed(3)
    rows = [torch.randn(1, hkv, 400, D, generator=g).half().to(gpu_device) for _ in range(2)]
    mine = [torch.randn(B, hkv, 50, D, generator=g).half().to(gpu_device) for _ in range(2)]
    make = lambda b: swan_mod.SwanCache(b, hq, hkv, 64, 400, [128] * b, torch.float16,  # noqa: E731
                                        gpu_device)
    past, own, whole = make(1), make(B), make(B)
    past.append(*rows, *P)
    own.append(*mine, *P)
    whole.append(*[torch.cat([r.expand(B, -1, -1, -1), x], 2).contiguous()
                   for r, x in zip(rows, mine)], *P)
    q = _queries(torch, gpu_device, (B, hq, D), "f16", 4, 1.0)
    a = own.decode(q, *P, prefix=swan_mod.Prefix(past))
    b = whole.decode(q, *P)
    assert C.max_rel_err(a.cpu().numpy(), b.double().cpu().numpy()) < 2e-3


def test_large_queries_and_cached_extremes(gpu_device, swan_mod, torch_mod):
    """Queries whose rotation passes binary16's range, zero queries, one key far above the
    rest: finite where the formula is."""
    torch = torch_mod
    cache, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [300], 4, 1, 16, [32], "f16", 21)
    q = _queries(torch, gpu_device, (1, 4, 2, D), "f16", 22, 1.0)
    q[0, 0] = 0
    q[0, 1, 0] = (P_qk[0, :, 3].double() * 60000).half()
    q[0, 2, 1] *= 2.0 ** -14
    q[0, 3] = 60000.0
    o, lse = cache.attend(q, P_qk, None)
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    K, V = (R.cached_rows(cache, 0, 0, r) for r in (0, 1))
    assert torch.allclose(o[0, 0].double(), V.mean(0).expand(2, D), atol=2e-3)
    qh = q[0, 1, 0].double() @ P_qk[0].double()
    best = V[(K @ qh).argmax()]
    s = (K @ qh) / math.sqrt(D)
    assert s.topk(2).values.diff().abs().item() > 20
    assert torch.allclose(o[0, 1, 0].double(), best, atol=2e-3)


def test_streams_graphs_and_repeats(gpu_device, swan_mod, torch_mod):
    torch = torch_mod
    hq, hkv, B = 8, 2, 3
    own, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [100, 3, 50], hq, hkv, 16, [32, 64, 32],
                                     "f16", 31)
    past, _, _ = R.filled_cache(swan_mod, gpu_device, [900], hq, hkv, 64, [48], "f16", 32,
                                P=(P_qk, P_vo))
    prefix = swan_mod.Prefix(past)
    q = _queries(torch, gpu_device, (B, hq, D), "f16", 33)
    rows = _queries(torch, gpu_device, (B, hq, 9, D), "f16", 34)
    want = own.decode(q, P_qk, P_vo, prefix=prefix)
    state = own.attend(rows, P_qk, P_vo, prefix=prefix)
    for _ in range(5):
        assert torch.equal(want, own.decode(q, P_qk, P_vo, prefix=prefix))
        for a, b in zip(state, own.attend(rows, P_qk, P_vo, prefix=prefix)):
            assert torch.equal(a, b)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = own.decode(q, P_qk, P_vo, prefix=prefix, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    got = own.attend(rows, P_qk, P_vo, prefix=prefix, stream=side)
    side.synchronize()
    assert torch.equal(got[0], state[0]) and torch.equal(got[1], state[1])
    # two captured graphs with a workspace each, replayed with eager calls between
    outs, graphs = [torch.zeros_like(q), tuple(torch.zeros_like(t) for t in state)], []
    for call in (lambda: own.decode(q, P_qk, P_vo, out=outs[0], prefix=prefix),
                 lambda: own.attend(rows, P_qk, P_vo, prefix=prefix, out=outs[1])):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
    for turn in range(3):
        q.mul_(0.9)
        rows.mul_(0.9)
        for t in (outs[0], *outs[1]):
            t.zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in (outs[0], *outs[1])]
        assert torch.equal(kept[0], own.decode(q, P_qk, P_vo, prefix=prefix)), turn
        for a, b in zip(kept[1:], own.attend(rows, P_qk, P_vo, prefix=prefix)):
            assert torch.equal(a, b), turn


def test_calls_on_two_streams_at_once(gpu_device, swan_mod, torch_mod):
    """Decode calls behind a prefix of one cache, enqueued on two streams without waiting:
    each has a workspace of its own."""
    torch = torch_mod
    hq, hkv, B = 8, 2, 3
    own, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [300, 3, 50], hq, hkv, 16, [32, 64, 32],
                                     "f16", 41)
    past, _, _ = R.filled_cache(swan_mod, gpu_device, [4000], hq, hkv, 64, [48], "f16", 42,
                                P=(P_qk, P_vo))
    prefix = swan_mod.Prefix(past)
    qs = [_queries(torch, gpu_device, (B, hq, D), "f16", 43 + i) for i in range(2)]
    want = [own.decode(q, P_qk, P_vo, prefix=prefix) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            got[i].append(own.decode(qs[i], P_qk, P_vo, prefix=prefix, stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i]), i


def test_pages_beyond_32_bit_offsets(gpu_device, swan_mod, torch_mod):
    """Arrays of 13 GB: the second sequence's pages lie beyond 6.4 GB of each."""
    torch = torch_mod
    hq, hkv = 16, 8
    past, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [70, 333], hq, hkv, 16, [128, 128], "f16",
                                      51, spare=2 ** 21)
    assert past.k_pages.numel() > 12 * 2 ** 30
    own, _, _ = R.filled_cache(swan_mod, gpu_device, [90, 1], hq, hkv, 16, [40, 40], "f16", 52,
                               P=(P_qk, P_vo))
    of = [1, 0]
    q = _queries(torch, gpu_device, (2, hq, 33, D), "f16", 53)
    o, lse = past.attend(q, P_qk, P_vo, of=of)
    out = own.decode(q[:, :, 0].contiguous(), P_qk, P_vo, prefix=swan_mod.Prefix(past, of))
    for b in range(2):
        for h in (0, 7, 15):
            want, _, K, V = _want([(past, of)], q[b, h], b, h, 2, P_qk, P_vo)
            tol = R.bound("f16", q[b, h], K, V, want, len(K), "f32", turned=True)
            R.close(o[b, h], want, tol, f"rows {b} {h}")
            want, _, K, V = _want([(past, of), (own, [0, 1])], q[b, h, :1], b, h, 2, P_qk, P_vo)
            tol = R.bound("f16", q[b, h, :1], K, V, want, len(K), turned=True)
            R.close(out[b, h][None], want, tol, f"decode {b} {h}")
