// Host side of include/swan_long.h: argument validation (always before anything is enqueued),
// plans and kernel launches.
#include <math.h>

#include "swan_host.h"
#include "swan_long.h"

using namespace swan_host;

namespace {

// a swan_rotary's checks, into the kernels' form
swan_status rotary_form(const swan_rotary* r, int32_t head_dim, swan::RotaryForm& f) {
  if (!r) return fail(SWAN_ERR_INVALID_ARG, "rotary is NULL");
  if (r->dims < 8 || r->dims > head_dim || r->dims % 8 != 0)
    return fail(SWAN_ERR_INVALID_ARG, "rotary: dims %d: a multiple of 8 within 8..%d", r->dims,
                head_dim);
  if (r->interleaved != 0 && r->interleaved != 1)
    return fail(SWAN_ERR_INVALID_ARG, "rotary: interleaved %d: 0 or 1", r->interleaved);
  if (!(r->magnitude > 0.0) || isinf(r->magnitude))
    return fail(SWAN_ERR_INVALID_ARG, "rotary: magnitude must be finite, > 0");
  if (!r->freq_host) return fail(SWAN_ERR_INVALID_ARG, "rotary: freq_host is NULL");
  f.magnitude = r->magnitude;
  f.half = r->dims / 2;
  f.interleaved = r->interleaved;
  for (int j = 0; j < swan::kD / 2; ++j) {
    f.freq[j] = j < f.half ? r->freq_host[j] : 0.0;
    if (!isfinite(f.freq[j]))
      return fail(SWAN_ERR_INVALID_ARG, "rotary: freq_host[%d] is not finite", j);
  }
  return SWAN_OK;
}

// Pages per workgroup, so that the launch and the join of its partials are shortest: pages[j]
// of sequence j, weighed by their entries, for each of its `units`.  LDS holds four workgroups
// a CU, 1024 in all, which is taken for every launch, though those of more than 80 components a
// role have one wave a SIMD, half as many; and one launch is taken for the whole batch, though
// sequences of several k go out in one for each of their tiers, one after another (16 sequences
// of 32 heads on 8 over windows of 4096 with k of 32, 48, 64 and 96 in turn 127 us, with k = 60
// 50; of 32 heads without groups 196 and 136).  A plan's time is taken as that of its longest
// split, or of all pages spread evenly, in one such round, or as rounds, or as spread evenly with
// half a workgroup's time more; then `rings` workgroups of the ring, of 5, which find room beside
// a first round that leaves some (32 sequences x 8 kv heads: 75 us with 848 workgroups, 92 with
// 1000 and with 1048).
// 2 us to start, and for a page (of `entries` in both roles) 1024 of them at 10 TB/s (8-bit
// values no less: their LDS work is that of 16-bit ones).  Of eleven plans measured for each of
// nine shapes (1 to 32 sequences, 8 to 64 heads, one k a batch) it takes the best or one within
// 3 %: 16 x 32 heads over 300 to 4096 tokens 84 us with 8 pages, 102 with 2, 100 with 22; 2 x 32
// heads over 1000 18 with 2, 24 with 1 (whose 1088 workgroups take two rounds) and with 8.
int plan_window(int32_t dtype, int entries, int groups, const int* pages, int units, int heads,
                double rings) {
  constexpr double kSlots = 1024, kStart = 2.0, kRing = 5.0;
  const double page = 64.0 * entries * (dtype == SWAN_F32 ? 5 : 3) * kSlots / 10e6;
  int64_t total = 0;
  int longest = 1;
  for (int j = 0; j < groups; ++j) {
    total += (int64_t)pages[j] * units;
    longest = pages[j] > longest ? pages[j] : longest;
  }
  const double even = (double)total * page / kSlots;
  int best = longest;
  double least = 1e30;
  // every plan of few pages, then steps of an eighth
  for (int per = (longest + swan::kMaxSplits - 1) / swan::kMaxSplits; per <= longest;
       per += per < 16 ? 1 : per / 8) {
    int64_t splits = 0;
    int most = 1;  // pages of a split
    for (int j = 0; j < groups; ++j) {
      const int ns = (pages[j] + per - 1) / per, each = (pages[j] + ns - 1) / ns;
      splits += ns;
      most = each > most ? each : most;
    }
    const double u = (double)splits * units, one = kStart + most * page;
    double t;
    if (u <= kSlots) {
      const double run = most * page * (u <= 256 ? 0.7 : 1.0);
      t = kStart + (run > even ? run : even);
      if (rings > (kSlots - u) * t / kRing) t += kRing;
    } else {
      const double rounds = ceil(u / kSlots) * one, spread = u * kStart / kSlots + even + 0.5 * one;
      t = (rounds < spread ? rounds : spread) + rings * kRing / kSlots;
    }
    t += (double)splits * heads * (2.0 * 528 / 4e6);
    if (t < least) {
      least = t;
      best = per;
    }
  }
  return best;
}

struct WindowPlan {
  swan::WindowLaunch a;
  AttendPlan prefix;
  int16_t used[SWAN_MAX_BATCH];
  bool has_prefix;
  size_t qhat, bytes;
};

// The checks of a decode call's shape and the plan; need_ptrs: for a launch
swan_status window_prep(const swan_prefix* prefix, const swan_cache* c,
                        const int32_t* seq_len_host, const int32_t* k_active_host,
                        const int32_t* k_value_host, int32_t window, int32_t sinks, bool need_ptrs,
                        WindowPlan& pl) {
  swan_status st = check_cache_shape(c);
  if (st != SWAN_OK) return st;
  if ((st = check_k(c, k_active_host, k_value_host)) != SWAN_OK) return st;
  if (need_ptrs && (st = check_cache_ptrs(c)) != SWAN_OK) return st;
  if ((st = check_window(window, sinks)) != SWAN_OK) return st;
  if (!seq_len_host) return fail(SWAN_ERR_INVALID_ARG, "seq_len_host is NULL");
  swan::WindowLaunch& a = pl.a;
  swan::SeqTab tab;
  int64_t role_bytes[2];
  fill_layout(c, k_active_host, k_value_host, tab, role_bytes);
  int32_t pos[SWAN_MAX_BATCH];
  pl.has_prefix = prefix != nullptr;
  if (prefix) {
    if (!prefix->of_host || !prefix->seq_len_host)
      return fail(SWAN_ERR_INVALID_ARG, "prefix: seq_len_host / of_host is NULL");
    if ((st = check_cache_shape(prefix->cache)) != SWAN_OK) return st;
    if (prefix->cache->n_q_heads != c->n_q_heads || prefix->cache->n_kv_heads != c->n_kv_heads ||
        elem_bytes(prefix->cache->dtype) != elem_bytes(c->dtype))
      return fail(SWAN_ERR_INVALID_ARG, "the prefix's cache differs in heads or element type");
  }
  for (int b = 0; b < c->batch; ++b) {
    const int64_t L = seq_len_host[b];
    if (L < 0 || L > INT32_MAX / 2)
      return fail(SWAN_ERR_INVALID_ARG, "seq_len[%d] = %lld", b, (long long)L);
    if (L - c->buffer_tokens > c->sparse_capacity)
      return fail(SWAN_ERR_CAPACITY, "sequence %d has %lld sparse tokens, capacity %d", b,
                  (long long)(L - c->buffer_tokens), c->sparse_capacity);
    int64_t before = 0;
    if (prefix) {
      const int p = prefix->of_host[b];
      if (p < -1 || p >= prefix->cache->batch)
        return fail(SWAN_ERR_INVALID_ARG, "prefix: of[%d] = %d outside -1..%d", b, p,
                    prefix->cache->batch - 1);
      before = p < 0 ? 0 : prefix->seq_len_host[p];
      if (before < 0 || before > INT32_MAX / 2)
        return fail(SWAN_ERR_INVALID_ARG, "prefix: seq_len[%d] = %lld", p, (long long)before);
    }
    if (before + L < 1)
      return fail(SWAN_ERR_INVALID_ARG, "sequence %d has no token, of its own or of a prefix", b);
    pos[b] = (int32_t)(before + L - 1);
    a.len[b] = (int32_t)L;
    a.lo[b] = (int32_t)(L - window);
    a.sink[b] = sinks > before ? (int32_t)(sinks - before) : 0;
  }
  for (int b = 0; b < SWAN_MAX_BATCH; ++b) {
    if (b >= c->batch) a.len[b] = a.lo[b] = a.sink[b] = 0;
    for (int r = 0; r < 2; ++r) {
      a.kact[r][b] = tab.kact[r][b];
      a.off[r][b] = tab.page_off[r][b];
    }
  }
  const int hpw = swan::decode_heads_per_wave(c->dtype, c->n_q_heads, c->n_kv_heads);
  // splits, a page being one of the most entries among the batch
  auto listed = [&](int b) {
    return swan::WindowPages(a.len[b], c->buffer_tokens, a.lo[b], a.sink[b]).count;
  };
  auto entries = [&](int b) {
    return swan::kpad_of(a.kact[0][b]) + swan::kpad_of(a.kact[1][b]);
  };
  int most = 0, groups = 0, pages[SWAN_MAX_BATCH], seq[SWAN_MAX_BATCH];
  for (int b = 0; b < c->batch; ++b) most = entries(b) > most ? entries(b) : most;
  for (int b = 0; b < c->batch; ++b) {
    const int64_t n = listed(b);
    if (n == 0) continue;
    pages[groups] = (int)((n * entries(b) + most - 1) / most);
    seq[groups++] = b;
  }
  for (int b = 0; b < SWAN_MAX_BATCH; ++b) a.nsplit[b] = 0;
  double rings = 0;
  for (int b = 0; b < c->batch; ++b)
    rings += swan::pages_for(a.len[b] < c->buffer_tokens ? a.len[b] : c->buffer_tokens);
  rings *= hpw > 1 ? 0.5 * c->n_q_heads : c->n_q_heads;
  const int per = groups == 0 ? 1 : plan_window(c->dtype, most, groups, pages, c->n_q_heads / hpw,
                                                c->n_q_heads, rings);
  for (int j = 0; j < groups; ++j) a.nsplit[seq[j]] = (pages[j] + per - 1) / per;
  int slots = 0;
  for (int b = 0; b < SWAN_MAX_BATCH; ++b) {
    pl.used[b] = 0;
    if (b >= c->batch || a.len[b] == 0) continue;
    const int ring = a.len[b] < c->buffer_tokens ? a.len[b] : c->buffer_tokens;
    pl.used[b] = (int16_t)(a.nsplit[b] + swan::pages_for(ring));
    slots = pl.used[b] > slots ? pl.used[b] : slots;
  }
  double blocks = rings;
  for (int b = 0; b < c->batch; ++b) blocks += (double)a.nsplit[b] * (c->n_q_heads / hpw);
  // Few blocks rotate the queries of their heads themselves, each reading its P_qk from L2: a
  // launch less (4 us of the host's time), and less on the GPU too: one sequence of 8 kv heads
  // of 4 query heads over 1024 tokens 13.9 us against 14.9, two 14.2 against 15.8, one of 16 kv
  // heads of 2 12.7 against 14.5.  Not many blocks (8 sequences: 20.6 against 20.4), nor 8 heads,
  // whose sums LDS has no room for.
  a.rotate_here = hpw > 1 && hpw <= swan::kRotateHeads && !prefix && blocks <= 512;
  pl.prefix.slots = 0;
  if (prefix) {
    Window w;
    w.window = window;
    w.sinks = sinks;
    w.pos = pos;
    if ((st = attend_prep(prefix, 1, c->batch, 1, nullptr, need_ptrs, pl.prefix, w)) != SWAN_OK)
      return st;
  }
  a.B = c->batch;
  a.Hq = c->n_q_heads;
  a.Hkv = c->n_kv_heads;
  a.bb = c->buffer_tokens;
  a.npc = swan::pages_for(c->sparse_capacity);
  a.slots = slots + pl.prefix.slots;
  a.dtype = c->dtype;
  a.k_pages = c->k_pages;
  a.v_pages = c->v_pages;
  a.k_ring = c->k_ring;
  a.v_ring = c->v_ring;
  const size_t rows = (size_t)c->batch * c->n_q_heads;
  pl.qhat = round256(rows * swan::kD * sizeof(float));
  pl.bytes = pl.qhat + rows * a.slots * swan::kPartFloats * sizeof(float);
  return SWAN_OK;
}

// The checks of the other arguments, which go into the plan
swan_status window_args(const swan_cache* c, const void* q, const float* P_qk, const float* P_vo,
                        float scale, void* out, void* workspace, size_t workspace_bytes,
                        void* stream, WindowPlan& pl) {
  swan_status st = check_scale(scale);
  if (st != SWAN_OK) return st;
  if (!q || !out || !P_qk) return fail(SWAN_ERR_INVALID_ARG, "q / out / P_qk is NULL");
  if ((((uintptr_t)P_qk | (uintptr_t)P_vo) & 15) != 0)
    return fail(SWAN_ERR_INVALID_ARG, "P_qk / P_vo must be 16-byte aligned");
  if (!workspace || workspace_bytes < pl.bytes)
    return fail(SWAN_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace_bytes, pl.bytes);
  if (((uintptr_t)workspace & 255) != 0)
    return fail(SWAN_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  swan::WindowLaunch& a = pl.a;
  a.q = q;
  a.P_qk = P_qk;
  a.qhat = (float*)workspace;
  a.part = (float*)((char*)workspace + pl.qhat);
  a.qmult = scale_or_default(scale) * 1.4426950408889634f;
  a.qhat_ready = 0;
  a.stream = (hipStream_t)stream;
  return SWAN_OK;
}

hipError_t window_launch(WindowPlan& pl, const float* P_vo, void* out) {
  const swan::WindowLaunch& w = pl.a;
  hipError_t e = swan::launch_window(w);
  if (e != hipSuccess) return e;
  swan::AttendLaunch& a = pl.prefix.a[0];
  if (pl.has_prefix && a.units > 0) {
    a.q = w.qhat;
    a.part = w.part;
    a.slots = w.slots;
    a.slot0 = w.slots - pl.prefix.slots;
    a.stream = w.stream;
    if ((e = swan::launch_attend_pages(a)) != hipSuccess) return e;
  }
  swan::JoinLaunch j;
  j.part = w.part;
  j.o0 = j.lse0 = nullptr;
  j.P_vo = P_vo;
  j.out = out;
  j.o = j.lse = nullptr;
  j.B = w.B;
  j.H = w.Hq;
  j.Hkv = w.Hkv;
  j.n = 1;
  j.slots = w.slots;
  j.dtype = w.dtype;
  j.decode = 1;
  j.own_slots = 0;
  j.own = nullptr;
  j.own_bb = 0;
  for (int b = 0; b < SWAN_MAX_BATCH; ++b) {
    j.used[0][b] = pl.used[b];
    j.used[1][b] = pl.has_prefix && b < w.B ? pl.prefix.used[0][b] : 0;
    j.rows[b] = 1;
  }
  j.base[0] = 0;
  j.base[1] = w.slots - pl.prefix.slots;
  j.stream = w.stream;
  return swan::launch_join(j);
}

}  // namespace

extern "C" {

swan_status swan_rope_rotary(const void* x, void* y, int32_t dtype, int32_t batch, int32_t n_heads,
                             int32_t n, int32_t head_dim, const int32_t* pos0_host,
                             const swan_rotary* rotary, void* stream) {
  swan::RopeLaunch a;
  swan_status st = rope_prep(x, y, dtype, batch, n_heads, n, head_dim, pos0_host, 2.0, stream, a);
  if (st != SWAN_OK) return st;
  swan::RotaryForm f;
  if ((st = rotary_form(rotary, head_dim, f)) != SWAN_OK) return st;
  if (n == 0) return ok();
  if ((int64_t)batch * n > INT32_MAX)
    return fail(SWAN_ERR_UNSUPPORTED, "batch %d x n %d: above 2^31 - 1 rows", batch, n);
  // heads alone, without norms
  swan::QkvRowsLaunch r;
  r.x = x;
  r.head = (int64_t)n * head_dim;
  r.seq = r.head * n_heads;
  r.row = head_dim;
  r.out[0] = y;
  r.out[1] = r.out[2] = nullptr;
  r.w[0] = r.w[1] = nullptr;
  r.wstep = r.w32 = 0;
  r.B = batch;
  r.Hq = n_heads;
  r.Hkv = 0;
  r.n = n;
  r.dtype = dtype;
  r.eps = r.base = 0.0;
  for (int b = 0; b < SWAN_MAX_BATCH; ++b) r.pos0[b] = a.pos0[b];
  r.stream = (hipStream_t)stream;
  return hip_status(swan::launch_qkv_rows(r, &f), "rope launch");
}

swan_status swan_qkv_rows_rotary(const void* qkv, int64_t seq_stride, int64_t row_stride,
                                 int32_t dtype, int32_t batch, int32_t n_q_heads,
                                 int32_t n_kv_heads, int32_t n, int32_t head_dim,
                                 const int32_t* pos0_host, const swan_rotary* rotary,
                                 const void* q_weight, const void* k_weight,
                                 int32_t weights_per_head, int32_t weights_f32, double eps, void* q,
                                 void* k, void* v, void* stream) {
  swan::QkvRowsLaunch a;
  swan_status st = qkv_rows_prep(qkv, seq_stride, row_stride, dtype, batch, n_q_heads, n_kv_heads,
                                 n, head_dim, pos0_host, 2.0, q_weight, k_weight,
                                 weights_per_head, weights_f32, eps, q, k, v, stream, a);
  if (st != SWAN_OK) return st;
  swan::RotaryForm f;
  if ((st = rotary_form(rotary, head_dim, f)) != SWAN_OK) return st;
  if (n == 0) return ok();
  return hip_status(swan::launch_qkv_rows(a, &f), "qkv_rows launch");
}

swan_status swan_prompt_window_workspace_bytes(int32_t dtype, int32_t batch, int32_t n_q_heads,
                                               int32_t n_kv_heads, int32_t n, int32_t m,
                                               int32_t head_dim, const int32_t* n_host,
                                               const int32_t* m_host, int32_t window,
                                               const int32_t* sinks_host, size_t* bytes) {
  if (!bytes) return fail(SWAN_ERR_INVALID_ARG, "bytes is NULL");
  swan_status st = check_window(window, 0);
  if (st != SWAN_OK) return st;
  PromptPlan pl;
  if ((st = prompt_prep(dtype, batch, n_q_heads, n_kv_heads, n, m, head_dim, n_host, m_host, 1, pl,
                        window, sinks_host)) != SWAN_OK)
    return st;
  *bytes = pl.bytes;
  return ok();
}

swan_status swan_prompt_attention_window(const void* q, const void* k, const void* v,
                                         int32_t dtype, int32_t batch, int32_t n_q_heads,
                                         int32_t n_kv_heads, int32_t n, int32_t m,
                                         int32_t head_dim, const int32_t* n_host,
                                         const int32_t* m_host, int32_t window,
                                         const int32_t* sinks_host, float scale, const float* o0,
                                         const float* lse0, void* out, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  const swan_status st = check_window(window, 0);
  if (st != SWAN_OK) return st;
  return prompt_run(q, k, v, dtype, batch, n_q_heads, n_kv_heads, n, m, head_dim, n_host, m_host, 1,
                    window, sinks_host, scale, o0, lse0, out, workspace, workspace_bytes, stream);
}

swan_status swan_attend_window_workspace_bytes(const swan_prefix* sources, int32_t n_sources,
                                               int32_t batch, int32_t n, const int32_t* n_host,
                                               int32_t window, int32_t sinks, size_t* bytes) {
  if (!bytes) return fail(SWAN_ERR_INVALID_ARG, "bytes is NULL");
  swan_status st = check_window(window, sinks);
  if (st != SWAN_OK) return st;
  Window w;
  w.window = window;
  w.sinks = sinks;
  AttendPlan pl;
  if ((st = attend_prep(sources, n_sources, batch, n, n_host, false, pl, w)) != SWAN_OK) return st;
  *bytes = pl.bytes;
  return ok();
}

swan_status swan_attend_window(const swan_prefix* sources, int32_t n_sources, int32_t batch,
                               int32_t n, const int32_t* n_host, int32_t window, int32_t sinks,
                               const void* q, const float* P_qk, const float* P_vo, float scale,
                               float* o, float* lse, void* workspace, size_t workspace_bytes,
                               void* stream) {
  const swan_status st = check_window(window, sinks);
  if (st != SWAN_OK) return st;
  Window w;
  w.window = window;
  w.sinks = sinks;
  return attend_run(sources, n_sources, batch, n, n_host, w, q, P_qk, P_vo, scale, o, lse,
                    workspace, workspace_bytes, stream);
}

swan_status swan_decode_window_workspace_bytes(const swan_prefix* prefix, const swan_cache* c,
                                               const int32_t* seq_len_host,
                                               const int32_t* k_active_host,
                                               const int32_t* k_value_host, int32_t window,
                                               int32_t sinks, size_t* bytes) {
  if (!bytes) return fail(SWAN_ERR_INVALID_ARG, "bytes is NULL");
  WindowPlan pl;
  const swan_status st = window_prep(prefix, c, seq_len_host, k_active_host, k_value_host, window,
                                     sinks, false, pl);
  if (st != SWAN_OK) return st;
  *bytes = pl.bytes;
  return ok();
}

swan_status swan_decode_attention_window(const swan_prefix* prefix, const swan_cache* c,
                                         const int32_t* seq_len_host,
                                         const int32_t* k_active_host,
                                         const int32_t* k_value_host, int32_t window,
                                         int32_t sinks, const void* q, const float* P_qk,
                                         const float* P_vo, float scale, void* out,
                                         void* workspace, size_t workspace_bytes, void* stream) {
  WindowPlan pl;
  swan_status st = window_prep(prefix, c, seq_len_host, k_active_host, k_value_host, window, sinks,
                               true, pl);
  if (st != SWAN_OK) return st;
  if ((st = window_args(c, q, P_qk, P_vo, scale, out, workspace, workspace_bytes, stream, pl)) !=
      SWAN_OK)
    return st;
  return hip_status(window_launch(pl, P_vo, out), "decode launch");
}

swan_status swan_decode_step_window(const swan_prefix* prefix, const swan_cache* c,
                                    const int32_t* seq_len_host, const int32_t* k_active_host,
                                    const int32_t* k_value_host, int32_t window, int32_t sinks,
                                    const void* k_new, const void* v_new, const void* q,
                                    const float* P_qk, const float* P_vo, float scale, void* out,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  // every check of all parts before anything is enqueued
  swan::CompressLaunch ca;
  bool any_new = false;
  swan_status st = compress_prep(c, seq_len_host, k_active_host, k_value_host, k_new, v_new, 1,
                                 nullptr, P_qk, P_vo, stream, ca, any_new);
  if (st != SWAN_OK) return st;
  int32_t after[SWAN_MAX_BATCH];
  for (int b = 0; b < c->batch; ++b) after[b] = seq_len_host[b] + 1;
  WindowPlan pl;
  if ((st = window_prep(prefix, c, after, k_active_host, k_value_host, window, sinks, true, pl)) !=
      SWAN_OK)
    return st;
  if (prefix && ((c->k_pages && c->k_pages == prefix->cache->k_pages) ||
                 (c->k_ring && c->k_ring == prefix->cache->k_ring)))
    return fail(SWAN_ERR_INVALID_ARG, "the prefix's cache is the one appended to");
  if ((st = window_args(c, q, P_qk, P_vo, scale, out, workspace, workspace_bytes, stream, pl)) !=
      SWAN_OK)
    return st;
  if (c->n_q_heads / c->n_kv_heads <= swan::kStepQG) {  // the key waves rotate the queries
    ca.q = q;
    ca.qhat = pl.a.qhat;
    ca.Hq = c->n_q_heads;
    ca.qmult = pl.a.qmult;
    pl.a.qhat_ready = 1;
    pl.a.rotate_here = 0;
  }
  const hipError_t e = swan::launch_compress(ca);
  if (e != hipSuccess) return hip_status(e, "compress launch");
  return hip_status(window_launch(pl, P_vo, out), "decode launch");
}

swan_status swan_copy_sequences(const swan_cache* src, const int32_t* src_len_host,
                                const int32_t* k_active_src, const int32_t* k_value_src,
                                const swan_cache* dst, const int32_t* k_active_dst,
                                const int32_t* k_value_dst, const int32_t* of_host,
                                const int32_t* first_host, const int32_t* drop_host, void* stream) {
  swan_status st = check_cache_shape(src);
  if (st != SWAN_OK) return st;
  if ((st = check_cache_shape(dst)) != SWAN_OK) return st;
  if (src->n_kv_heads != dst->n_kv_heads || src->n_q_heads != dst->n_q_heads ||
      src->buffer_tokens != dst->buffer_tokens || src->dtype != dst->dtype)
    return fail(SWAN_ERR_INVALID_ARG, "src and dst differ in heads, buffer_tokens or dtype");
  if ((st = check_k(src, k_active_src, k_value_src)) != SWAN_OK) return st;
  if ((st = check_k(dst, k_active_dst, k_value_dst)) != SWAN_OK) return st;
  if ((st = check_cache_ptrs(src)) != SWAN_OK) return st;
  if ((st = check_cache_ptrs(dst)) != SWAN_OK) return st;
  if (!src_len_host || !of_host)
    return fail(SWAN_ERR_INVALID_ARG, "src_len_host / of_host is NULL");
  swan::SeqTab ts, td;
  int64_t bytes_src[4], bytes_dst[4];
  fill_layout(src, k_active_src, k_value_src, ts, bytes_src);
  fill_layout(dst, k_active_dst, k_value_dst, td, bytes_dst);
  const int64_t ring = (int64_t)src->n_kv_heads * src->buffer_tokens * swan::kD *
                       elem_bytes(src->dtype);
  bytes_src[2] = bytes_src[3] = ring * src->batch;
  bytes_dst[2] = bytes_dst[3] = ring * dst->batch;
  swan::CopyLaunch a;
  void* const from[4] = {src->k_pages, src->v_pages, src->k_ring, src->v_ring};
  void* const to[4] = {dst->k_pages, dst->v_pages, dst->k_ring, dst->v_ring};
  for (int i = 0; i < 4; ++i) {
    a.src[i] = from[i];
    a.dst[i] = to[i];
    for (int j = 0; j < 4; ++j)
      if (overlap(from[i], bytes_src[i], to[j], bytes_dst[j]))
        return fail(SWAN_ERR_INVALID_ARG, "src's and dst's arrays overlap");
  }
  a.n = a.max_pages = 0;
  for (int b = 0; b < dst->batch; ++b) {
    const int p = of_host[b];
    if (p < -1 || p >= src->batch)
      return fail(SWAN_ERR_INVALID_ARG, "of[%d] = %d outside -1..%d", b, p, src->batch - 1);
    if (p < 0) continue;
    const int64_t L = src_len_host[p];
    if (L < 0 || L > INT32_MAX / 2)
      return fail(SWAN_ERR_INVALID_ARG, "seq_len[%d] = %lld", p, (long long)L);
    const int64_t S = L > src->buffer_tokens ? L - src->buffer_tokens : 0;
    if (S > src->sparse_capacity)
      return fail(SWAN_ERR_CAPACITY, "sequence %d has %lld sparse tokens, capacity %d", p,
                  (long long)S, src->sparse_capacity);
    const int64_t drop = drop_host ? drop_host[b] : 0, first = first_host ? first_host[b] : 0;
    if (drop < 0 || first < 0 || (drop > 0 && first + drop > S))
      return fail(SWAN_ERR_INVALID_ARG,
                  "copy %d leaves out %lld tokens from %lld on: sequence %d has %lld pruned ones", b,
                  (long long)drop, (long long)first, p, (long long)S);
    if (S - drop > dst->sparse_capacity)
      return fail(SWAN_ERR_CAPACITY, "copy %d has %lld sparse tokens, capacity %d", b,
                  (long long)(S - drop), dst->sparse_capacity);
    const int e = a.n++;
    for (int r = 0; r < 2; ++r) {
      if (ts.kact[r][p] != td.kact[r][b])
        return fail(SWAN_ERR_INVALID_ARG, "copy %d has k = %d, sequence %d k = %d (%s)", b,
                    td.kact[r][b], p, ts.kact[r][p], r ? "values" : "keys");
      a.k[r][e] = td.kact[r][b];
      a.off_src[r][e] = ts.page_off[r][p];
      a.off_dst[r][e] = td.page_off[r][b];
    }
    a.from[e] = p;
    a.to[e] = b;
    a.len[e] = (int32_t)L;
    a.first[e] = drop > 0 ? (int32_t)first : INT32_MAX;
    a.drop[e] = (int32_t)drop;
    const int pages = swan::pages_for((int)(S - drop));
    a.max_pages = pages > a.max_pages ? pages : a.max_pages;
  }
  if (a.n == 0) return ok();
  if (src->n_kv_heads > 65535)
    return fail(SWAN_ERR_UNSUPPORTED, "n_kv_heads %d above 65535", src->n_kv_heads);
  a.Hkv = src->n_kv_heads;
  a.bb = src->buffer_tokens;
  a.npc_src = swan::pages_for(src->sparse_capacity);
  a.npc_dst = swan::pages_for(dst->sparse_capacity);
  a.dtype = src->dtype;
  a.stream = (hipStream_t)stream;
  return hip_status(swan::launch_copy(a), "copy launch");
}

}  // extern "C"
