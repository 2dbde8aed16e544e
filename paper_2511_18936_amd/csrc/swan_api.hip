// Host side of the C ABI declared in include/swan.h and swan_layer.h: argument validation
// (always before anything is enqueued), workspace sizing, split planning and
// kernel launches.  No allocation, no host arithmetic on the data path.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <mutex>
#include <string>

#include "swan.h"
#include "swan_host.h"

// ---------------------------------------------------------------------------
// Scratch of swan_decode_attention_noalloc: the decode workspace (q_hat, then
// the partials) in a device array of fixed size, one copy per GPU, held until
// the process ends.  Host code only ever uses the address that
// hipGetSymbolAddress returns for the current device: the array's name is a
// host-side stand-in, not a device address.
// ---------------------------------------------------------------------------
constexpr size_t kScratchBytes = SWAN_NOALLOC_SCRATCH_BYTES;
static __device__ __align__(256) char scratch[kScratchBytes];

namespace swan_host {

namespace {
thread_local std::string g_last_error;
thread_local hipEvent_t g_prof_start = nullptr;
thread_local hipEvent_t g_prof_stop = nullptr;

// Decode tuning of this thread (swan_set_decode_tuning), with the defaults
// resolved: about two sparse waves per wave slot of the GPU (measured best for
// long contexts), short sequences in 4-page splits, launch merging at two
// thirds of the k_pad, three side streams.
struct Tuning {
  int64_t target_waves = 256 * 4 * 2;
  int short_split_pages = 3;  // 0: never
  int merge_pct = 66;         // 0: never
  int side_streams = swan::kSideStreams;
};
thread_local Tuning g_tuning;
}  // namespace

swan_status fail(swan_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  g_last_error = buf;
  return st;
}

swan_status ok() {
  g_last_error.clear();
  return SWAN_OK;
}

// bytes of one element of queries, outputs, new keys / values and the ring
int elem_bytes(int32_t dtype) { return dtype == SWAN_F32 ? 4 : 2; }
// bytes of one sparse value
int value_bytes(int32_t dtype) { return dtype == SWAN_F32 ? 4 : dtype == SWAN_F16 ? 2 : 1; }
bool dtype_ok(int32_t dtype) {
  return dtype == SWAN_F32 || dtype == SWAN_F16 || dtype == SWAN_F16_E4M3;
}

swan_status check_cache_shape(const swan_cache* c) {
  if (!c) return fail(SWAN_ERR_INVALID_ARG, "cache descriptor is NULL");
  if (c->batch < 1 || c->batch > SWAN_MAX_BATCH)
    return fail(SWAN_ERR_INVALID_ARG, "batch %d outside 1..%d", c->batch, SWAN_MAX_BATCH);
  if (c->n_kv_heads < 1 || c->n_q_heads < 1)
    return fail(SWAN_ERR_INVALID_ARG, "head counts must be >= 1 (q %d, kv %d)", c->n_q_heads,
                c->n_kv_heads);
  if (c->n_q_heads % c->n_kv_heads != 0)
    return fail(SWAN_ERR_INVALID_ARG, "n_q_heads %d is not a multiple of n_kv_heads %d",
                c->n_q_heads, c->n_kv_heads);
  if (c->head_dim != SWAN_HEAD_DIM)
    return fail(SWAN_ERR_UNSUPPORTED, "head_dim %d: the GPU path supports %d only", c->head_dim,
                SWAN_HEAD_DIM);
  if (c->buffer_tokens < 0)
    return fail(SWAN_ERR_INVALID_ARG, "buffer_tokens %d < 0", c->buffer_tokens);
  if (c->buffer_tokens > swan::kMaxRing)
    return fail(SWAN_ERR_UNSUPPORTED, "buffer_tokens %d above %d", c->buffer_tokens,
                swan::kMaxRing);
  if (c->sparse_capacity < 0)
    return fail(SWAN_ERR_INVALID_ARG, "sparse_capacity %d < 0", c->sparse_capacity);
  if (!dtype_ok(c->dtype)) return fail(SWAN_ERR_UNSUPPORTED, "dtype %d not supported", c->dtype);
  if (c->reserved != 0) return fail(SWAN_ERR_INVALID_ARG, "reserved field must be 0");
  return SWAN_OK;
}

// k of the keys (k_active_host) and, if not NULL, of the values (k_value_host)
swan_status check_k(const swan_cache* c, const int32_t* k_active_host,
                    const int32_t* k_value_host) {
  if (!k_active_host) return fail(SWAN_ERR_INVALID_ARG, "k_active_host is NULL");
  for (int b = 0; b < c->batch; ++b) {
    const int k = k_active_host[b];
    if (k < 1 || k > c->head_dim)
      return fail(SWAN_ERR_INVALID_ARG, "k_active[%d] = %d outside 1..%d", b, k, c->head_dim);
    if (!k_value_host) continue;
    const int kv = k_value_host[b];
    if (kv < 1 || kv > c->head_dim)
      return fail(SWAN_ERR_INVALID_ARG, "k_value[%d] = %d outside 1..%d", b, kv, c->head_dim);
  }
  return SWAN_OK;
}

swan_status check_cache_ptrs(const swan_cache* c) {
  if (c->sparse_capacity > 0 && (!c->k_pages || !c->v_pages))
    return fail(SWAN_ERR_INVALID_ARG, "k_pages / v_pages is NULL");
  if (c->buffer_tokens > 0 && (!c->k_ring || !c->v_ring))
    return fail(SWAN_ERR_INVALID_ARG, "k_ring / v_ring is NULL");
  const void* ptrs[4] = {c->k_pages, c->v_pages, c->k_ring, c->v_ring};
  for (const void* p : ptrs)
    if (((uintptr_t)p & 15) != 0)
      return fail(SWAN_ERR_INVALID_ARG, "cache arrays must be 16-byte aligned");
  return SWAN_OK;
}

// fills tab.kact and tab.page_off of both roles; bytes[r] = total page bytes of role r
void fill_layout(const swan_cache* c, const int32_t* k_active_host, const int32_t* k_value_host,
                 swan::SeqTab& tab, int64_t bytes[2]) {
  const int npc = swan::pages_for(c->sparse_capacity);
  for (int b = 0; b < SWAN_MAX_BATCH; ++b) {
    for (int r = 0; r < 2; ++r) {
      tab.kact[r][b] = 0;
      tab.page_off[r][b] = 0;
    }
    tab.len[b] = 0;
    tab.nnew[b] = 0;
    tab.nsplit[b] = 1;
    tab.flat[b] = 0;
  }
  for (int r = 0; r < 2; ++r) {
    int64_t off = 0;
    for (int b = 0; b < c->batch; ++b) {
      const int k = k_of(k_active_host, k_value_host, r, b);
      tab.kact[r][b] = k;
      tab.page_off[r][b] = off;
      off += (int64_t)c->n_kv_heads * npc * swan::page_bytes_of(value_bytes(c->dtype), k);
    }
    bytes[r] = off;
  }
}

// Token splits per (sequence, query head): about the thread's target number of
// waves in total, the split count of each sequence following its bytes (a page
// weighs the k_pad of its keys plus that of its values); the splits themselves
// shrink in size (split_begin), and their count is capped so that every split
// keeps a page.  Fills nsplit[b] (may be NULL); returns the largest.
int plan_splits(const swan_cache* c, const int32_t* seq_len_host, const int32_t* k_active_host,
                const int32_t* k_value_host, int32_t* nsplit, int8_t* flat = nullptr) {
  auto weight = [&](int b) {
    return swan::kpad_of(k_of(k_active_host, k_value_host, 0, b)) +
           swan::kpad_of(k_of(k_active_host, k_value_host, 1, b));
  };
  // waves per sequence and split: one per query head, or one per GH query
  // heads of a KV head on the GQA path
  const int hpw = swan::decode_heads_per_wave(c->dtype, c->n_q_heads, c->n_kv_heads);
  const int waves_per_seq = c->n_q_heads / hpw;
  int64_t total = 0;
  for (int b = 0; b < c->batch; ++b) {
    const int S = seq_len_host[b] > c->buffer_tokens ? seq_len_host[b] - c->buffer_tokens : 0;
    total += (int64_t)swan::pages_for(S) * weight(b) * waves_per_seq;
  }
  // A batch of several k_pad on the fused MHA launch (decode_fused.hip) takes
  // twice the waves: its shorter splits balance the tiers' different costs
  // per page (measured: 16k x 8 with k in {32, 48, 64, 96}, 0.222 -> 0.213 ms;
  // the single-k workloads gain nothing from it and GQA loses 8 %).
  bool several_kpad = false;
  for (int b = 1; b < c->batch; ++b)
    several_kpad |= swan::kpad_of(k_of(k_active_host, k_value_host, 0, b)) !=
                        swan::kpad_of(k_of(k_active_host, k_value_host, 0, 0)) ||
                    swan::kpad_of(k_of(k_active_host, k_value_host, 1, b)) !=
                        swan::kpad_of(k_of(k_active_host, k_value_host, 1, 0));
  const bool fused = several_kpad && hpw == 1 &&
                     (c->dtype == SWAN_F16 || c->dtype == SWAN_F16_E4M3);
  const int64_t target_waves = g_tuning.target_waves * (fused ? 2 : 1);
  // A sequence whose shrinking splits the one-page rule cuts to half the count
  // wanted or fewer is short: its waves would each walk many pages one after
  // another, so it gets equal splits of flat_pages pages instead.
  const int flat_pages = g_tuning.short_split_pages;
  int64_t per_wave = (total + target_waves - 1) / target_waves;
  if (per_wave < 1) per_wave = 1;
  int ns_max = 1;
  for (int b = 0; b < c->batch; ++b) {
    const int S = seq_len_host[b] > c->buffer_tokens ? seq_len_host[b] - c->buffer_tokens : 0;
    const int np = swan::pages_for(S);
    const int64_t work = (int64_t)np * weight(b);
    const int want = (int)((work + per_wave - 1) / per_wave);
    int ns = want;
    while (ns > 1 && (int64_t)ns * (ns + 1) / 2 > np) --ns;  // every split keeps a page
    bool fl = false;
    if (flat_pages > 0 && 2 * ns <= want) {
      // short sequence: equal splits of about flat_pages pages instead
      fl = true;
      ns = np / flat_pages < want ? np / flat_pages : want;
    }
    if (ns > swan::kMaxSplits) ns = swan::kMaxSplits;
    if (ns < 1) ns = 1;
    if (nsplit) nsplit[b] = ns;
    if (flat) flat[b] = fl ? 1 : 0;
    if (ns > ns_max) ns_max = ns;
  }
  return ns_max;
}

size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }

// workspace: q_hat, then the partials
size_t decode_ws_bytes(const swan_cache* c, int ns) {
  const size_t units = (size_t)c->batch * c->n_q_heads;
  const size_t qhat = units * swan::kD * sizeof(float);
  const size_t part = units * (size_t)(ns + 1) * swan::kPartFloats * sizeof(float);
  return round256(qhat) + part;
}

// whether two ranges of bytes share one
bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  return a && b && a_bytes > 0 && b_bytes > 0 && (const char*)a < (const char*)b + b_bytes &&
         (const char*)b < (const char*)a + a_bytes;
}

swan_status hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return ok();
  return fail(SWAN_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

std::mutex g_scratch_mu;
void* g_scratch_ptr[swan::kMaxDevices] = {};

// The scratch array's address on the device of `stream` (set up once per
// device, with that device current).
swan_status scratch_for_stream(hipStream_t stream, void** ptr) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_status(e, "hipGetDevice");
  if (dev < 0 || dev >= swan::kMaxDevices)
    return fail(SWAN_ERR_UNSUPPORTED, "device %d: the scratch table holds %d devices", dev,
                swan::kMaxDevices);
  if (stream) {
    hipDevice_t sdev = -1;
    e = hipStreamGetDevice(stream, &sdev);
    if (e != hipSuccess) return hip_status(e, "hipStreamGetDevice");
    if (sdev != dev)
      return fail(SWAN_ERR_INVALID_ARG,
                  "the stream belongs to device %d but device %d is current", (int)sdev, dev);
  }
  std::lock_guard<std::mutex> lk(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* p = nullptr;
    e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess) return hip_status(e, "hipGetSymbolAddress(scratch)");
    if (!p || ((uintptr_t)p & 255) != 0)
      return fail(SWAN_ERR_HIP, "scratch array at an unusable address");
    g_scratch_ptr[dev] = p;
  }
  *ptr = g_scratch_ptr[dev];
  return SWAN_OK;
}

// swan_compress_append's validation, into `a` (nothing is enqueued); any_new:
// some sequence appends a token
swan_status compress_prep(const swan_cache* c, const int32_t* seq_len_host,
                          const int32_t* k_active_host, const int32_t* k_value_host,
                          const void* k_new, const void* v_new, int32_t n_new,
                          const int32_t* n_new_host, const float* P_qk, const float* P_vo,
                          void* stream, swan::CompressLaunch& a, bool& any_new) {
  swan_status st = check_cache_shape(c);
  if (st != SWAN_OK) return st;
  if ((st = check_k(c, k_active_host, k_value_host)) != SWAN_OK) return st;
  if ((st = check_cache_ptrs(c)) != SWAN_OK) return st;
  if (!seq_len_host) return fail(SWAN_ERR_INVALID_ARG, "seq_len_host is NULL");
  if (n_new < 0) return fail(SWAN_ERR_INVALID_ARG, "n_new %d < 0", n_new);
  if (n_new > 0 && (!k_new || !v_new)) return fail(SWAN_ERR_INVALID_ARG, "k_new / v_new is NULL");
  if (!P_qk) return fail(SWAN_ERR_INVALID_ARG, "P_qk is NULL");
  if ((((uintptr_t)P_qk | (uintptr_t)P_vo) & 15) != 0)
    return fail(SWAN_ERR_INVALID_ARG, "P_qk / P_vo must be 16-byte aligned");
  if ((((uintptr_t)k_new | (uintptr_t)v_new) & 15) != 0)
    return fail(SWAN_ERR_INVALID_ARG, "k_new / v_new must be 16-byte aligned");
  int max_evict = 0;
  any_new = false;
  for (int b = 0; b < c->batch; ++b) {
    const int64_t L0 = seq_len_host[b];
    if (L0 < 0) return fail(SWAN_ERR_INVALID_ARG, "seq_len[%d] = %lld < 0", b, (long long)L0);
    const int nb_new = n_new_host ? n_new_host[b] : n_new;
    if (nb_new < 0 || nb_new > n_new)
      return fail(SWAN_ERR_INVALID_ARG, "n_new_host[%d] = %d outside 0..%d", b, nb_new, n_new);
    any_new |= nb_new != 0;
    const int64_t L1 = L0 + nb_new;
    if (L1 > INT32_MAX / 2)
      return fail(SWAN_ERR_INVALID_ARG, "seq_len[%d] + n_new too large", b);
    if (L1 - c->buffer_tokens > c->sparse_capacity)
      return fail(SWAN_ERR_CAPACITY, "sequence %d needs %lld sparse tokens, capacity %d", b,
                  (long long)(L1 - c->buffer_tokens), c->sparse_capacity);
    const int64_t p0 = L0 > c->buffer_tokens ? L0 - c->buffer_tokens : 0;
    const int64_t p1 = L0 < L1 - c->buffer_tokens ? L0 : L1 - c->buffer_tokens;
    if (p1 - p0 > max_evict) max_evict = (int)(p1 - p0);
  }
  int64_t role_bytes[2];
  fill_layout(c, k_active_host, k_value_host, a.tab, role_bytes);
  for (int b = 0; b < c->batch; ++b) {
    a.tab.len[b] = seq_len_host[b];
    a.tab.nnew[b] = n_new_host ? n_new_host[b] : n_new;
  }
  a.k_new = k_new;
  a.v_new = v_new;
  a.P_qk = P_qk;
  a.P_vo = P_vo;
  a.k_pages = c->k_pages;
  a.v_pages = c->v_pages;
  a.k_ring = c->k_ring;
  a.v_ring = c->v_ring;
  a.B = c->batch;
  a.Hkv = c->n_kv_heads;
  a.bb = c->buffer_tokens;
  a.n_pages_cap = swan::pages_for(c->sparse_capacity);
  a.n_new = n_new;
  a.max_evict = max_evict;
  a.prefill_groups = 0;
  a.dtype = c->dtype;
  a.stream = (hipStream_t)stream;
  return SWAN_OK;
}

// The decode entry points' validation and split plan, into `a` (nothing is
// enqueued).  no_alloc: the workspace is this library's scratch array (looked
// up after every host check has passed), a plan that needs more than the
// array is rejected, and the launches stay on `stream` (creating the side
// streams could allocate).
swan_status decode_prep(const swan_cache* c, const int32_t* seq_len_host,
                        const int32_t* k_active_host, const int32_t* k_value_host, const void* q,
                        const float* P_qk, const float* P_vo, float scale, void* out,
                        void* workspace, size_t workspace_bytes, void* stream, bool no_alloc,
                        swan::DecodeLaunch& a, int least = 1) {
  swan_status st = check_cache_shape(c);
  if (st != SWAN_OK) return st;
  if ((st = check_k(c, k_active_host, k_value_host)) != SWAN_OK) return st;
  if ((st = check_cache_ptrs(c)) != SWAN_OK) return st;
  if (!seq_len_host) return fail(SWAN_ERR_INVALID_ARG, "seq_len_host is NULL");
  if (!q || !out || !P_qk) return fail(SWAN_ERR_INVALID_ARG, "q / out / P_qk is NULL");
  if ((((uintptr_t)P_qk | (uintptr_t)P_vo) & 15) != 0)
    return fail(SWAN_ERR_INVALID_ARG, "P_qk / P_vo must be 16-byte aligned");
  for (int b = 0; b < c->batch; ++b) {
    const int64_t L = seq_len_host[b];
    if (L < least)
      return fail(SWAN_ERR_INVALID_ARG, "seq_len[%d] = %lld: need L >= %d", b, (long long)L, least);
    if (L - c->buffer_tokens > c->sparse_capacity)
      return fail(SWAN_ERR_CAPACITY, "sequence %d has %lld sparse tokens, capacity %d", b,
                  (long long)(L - c->buffer_tokens), c->sparse_capacity);
  }
  if (!(scale == scale) || isinf(scale)) return fail(SWAN_ERR_INVALID_ARG, "scale is not finite");
  int64_t role_bytes[2];
  fill_layout(c, k_active_host, k_value_host, a.tab, role_bytes);
  const int ns = plan_splits(c, seq_len_host, k_active_host, k_value_host, a.tab.nsplit,
                            a.tab.flat);
  const size_t need = decode_ws_bytes(c, ns);
  if (no_alloc) {
    if (need > kScratchBytes)
      return fail(SWAN_ERR_WORKSPACE,
                  "this batch needs %zu bytes of decode scratch; swan_decode_attention_noalloc "
                  "holds %zu (use swan_decode_attention with a workspace)", need, kScratchBytes);
    const swan_status sst = scratch_for_stream((hipStream_t)stream, &workspace);
    if (sst != SWAN_OK) return sst;
    workspace_bytes = kScratchBytes;
  }
  if (!workspace || workspace_bytes < need)
    return fail(SWAN_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace_bytes, need);
  if (((uintptr_t)workspace & 255) != 0)
    return fail(SWAN_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  for (int b = 0; b < c->batch; ++b) a.tab.len[b] = seq_len_host[b];
  const float sc = scale > 0.f ? scale : 1.0f / sqrtf((float)c->head_dim);
  a.q = q;
  a.P_qk = P_qk;
  a.P_vo = P_vo;
  a.out = out;
  a.k_pages = c->k_pages;
  a.v_pages = c->v_pages;
  a.k_ring = c->k_ring;
  a.v_ring = c->v_ring;
  const size_t units = (size_t)c->batch * c->n_q_heads;
  a.qhat = (float*)workspace;
  a.part = (float*)((char*)workspace + round256(units * swan::kD * sizeof(float)));
  a.B = c->batch;
  a.Hq = c->n_q_heads;
  a.Hkv = c->n_kv_heads;
  a.bb = c->buffer_tokens;
  a.n_pages_cap = swan::pages_for(c->sparse_capacity);
  a.n_splits = ns;
  a.qmult = sc * 1.4426950408889634f;
  a.dtype = c->dtype;
  a.stream = (hipStream_t)stream;
  a.prof_start = g_prof_start;
  a.prof_stop = g_prof_stop;
  a.merge_pct = g_tuning.merge_pct;
  a.side_streams = no_alloc ? 0 : g_tuning.side_streams;
  return SWAN_OK;
}

// Both decode entry points: validation, split plan, launches.
swan_status decode_impl(const swan_cache* c, const int32_t* seq_len_host,
                        const int32_t* k_active_host, const int32_t* k_value_host, const void* q,
                        const float* P_qk, const float* P_vo, float scale, void* out,
                        void* workspace, size_t workspace_bytes, void* stream, bool no_alloc) {
  swan::DecodeLaunch a;
  const swan_status st = decode_prep(c, seq_len_host, k_active_host, k_value_host, q, P_qk,
                                     P_vo, scale, out, workspace, workspace_bytes, stream,
                                     no_alloc, a);
  if (st != SWAN_OK) return st;
  return hip_status(swan::launch_decode(a), "decode launch");
}

// A decode step's validation, the compress part's and the attention's, into `ca` and `da`
swan_status step_prep(const swan_cache* c, const int32_t* seq_len_host,
                      const int32_t* k_active_host, const int32_t* k_value_host,
                      const void* k_new, const void* v_new, const void* q, const float* P_qk,
                      const float* P_vo, float scale, void* out, void* workspace,
                      size_t workspace_bytes, void* stream, swan::CompressLaunch& ca,
                      swan::DecodeLaunch& da) {
  bool any_new = false;
  swan_status st = compress_prep(c, seq_len_host, k_active_host, k_value_host, k_new, v_new, 1,
                                 nullptr, P_qk, P_vo, stream, ca, any_new);
  if (st != SWAN_OK) return st;
  int32_t len1[SWAN_MAX_BATCH];
  for (int b = 0; b < c->batch; ++b) len1[b] = seq_len_host[b] + 1;
  st = decode_prep(c, len1, k_active_host, k_value_host, q, P_qk, P_vo, scale, out, workspace,
                   workspace_bytes, stream, false, da);
  if (st != SWAN_OK) return st;
  if (c->n_q_heads / c->n_kv_heads <= swan::kStepQG) {  // the key waves rotate the queries
    ca.q = q;
    ca.qhat = da.qhat;
    ca.Hq = da.Hq;
    ca.qmult = da.qmult;
    da.qhat_ready = 1;
  }
  return SWAN_OK;
}

// ---------------------------------------------------------------------------
// attention of several rows per sequence, and of decode steps behind a prefix
// ---------------------------------------------------------------------------
// What a plan of the attend kernels costs, in microseconds as measured: a workgroup's
// start, a tile of 64 keys of a workgroup on a full GPU (`slots` workgroups), and what share
// of that a tile of a workgroup alone on its CU takes.  Pages, binary16, with workgroups of
// 128 rows (two on a CU) or of 256 (`many`): 3.5 against 2 x 2.0 us for a tile of 256 rows,
// so the larger ones where rows fill them (4 x 256 rows over 4 x 8192 keys: 290 against 319
// us on one machine; 8 x 100 rows over 16384 keys 447 against 466).
struct AttendCost {
  int slots;
  double tile, start, alone;
};
AttendCost attend_cost(int32_t dtype, bool pages, bool many = false) {
  if (dtype == SWAN_F32) return {256, pages ? 10.0 : 7.5, 8.0, 1.0};
  if (many) return {256, 3.5, 6.0, 1.0};
  if (pages) return {512, 4.0, 6.0, 0.72};
  return {512, 3.1, 6.0, 0.65};
}

// Tiles of keys per workgroup, so that the launch and the join of its partials are
// shortest: tiles[j] of keys for base[j] row tiles (times kv heads) of group j, `rows` rows
// in all.  Plans that fill the GPU 1/2 (a workgroup alone on a CU), 1, 2, ... times are compared.  uneven: a row tile may have fewer tiles than the
// others of its group (causal), so workgroups even out; join: also one part has to be joined.
// least: the cost.
int plan_tiles(const AttendCost& c, int groups, const int64_t* base, const int* tiles,
               int64_t rows, bool uneven, bool join, double& least) {
  int longest = 1;
  double total = 0;
  for (int j = 0; j < groups; ++j) {
    longest = tiles[j] > longest ? tiles[j] : longest;
    total += (double)base[j] * tiles[j] * (uneven ? 0.5 : 1.0);
  }
  auto units = [&](int per) {
    int64_t u = 0;
    for (int j = 0; j < groups; ++j) u += base[j] * ((tiles[j] + per - 1) / per > 1 ? (tiles[j] + per - 1) / per : 1);
    return u;
  };
  auto cost = [&](int per) {
    const int64_t u = units(per);
    // (causal: of a row tile's parts about half have keys to see)
    const double full = uneven ? 0.6 * (double)u : (double)u;
    const double waves = ceil(full / c.slots);
    const int parts = (longest + per - 1) / per;
    double run = waves * per;
    if (uneven || u > 4 * c.slots) {  // the GPU stays full until the last ones
      const double even = total / c.slots + 0.5 * per;
      run = even < run ? even : run;
    }
    if (run < per) run = per;
    if (u <= 256) run *= c.alone;
    double t = waves * c.start + run * c.tile;
    if (join || parts > 1) t += 4.0 + (double)rows * parts * (2.0 * 528 / 4e6);
    return t;
  };
  int best = longest;
  least = cost(longest);
  const int64_t fills[] = {256, c.slots, 2 * c.slots, 3 * c.slots, 4 * c.slots, 6 * c.slots};
  for (const int64_t f : fills) {
    const int64_t fill = uneven ? f * 5 / 3 : f;
    int lo = 1, hi = longest;  // the fewest tiles with at most `fill` workgroups
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (units(mid) <= fill) hi = mid;
      else lo = mid + 1;
    }
    const int least_per = (longest + swan::kMaxSlots - 1) / swan::kMaxSlots;
    if (lo < least_per) lo = least_per;
    const double t = cost(lo);
    if (t < least * 0.98) {
      least = t;
      best = lo;
    }
  }
  return best;
}

swan_status check_scale(float scale) {
  if (!(scale == scale) || isinf(scale)) return fail(SWAN_ERR_INVALID_ARG, "scale is not finite");
  if (scale > 0.f && scale < 0x1p-64f)
    return fail(SWAN_ERR_INVALID_ARG, "scale %g below 2^-64", (double)scale);
  return SWAN_OK;
}
float scale_or_default(float scale) {
  return scale > 0.f ? scale : 1.0f / sqrtf((float)SWAN_HEAD_DIM);
}

// every entry of per_host (or NULL) within 0..n
swan_status check_rows(const char* name, const int32_t* per_host, int32_t batch, int32_t n) {
  if (n < 0) return fail(SWAN_ERR_INVALID_ARG, "%s %d < 0", name, n);
  if (n > INT32_MAX / 4) return fail(SWAN_ERR_INVALID_ARG, "%s %d too large", name, n);
  for (int b = 0; per_host && b < batch; ++b)
    if (per_host[b] < 0 || per_host[b] > n)
      return fail(SWAN_ERR_INVALID_ARG, "%s of sequence %d = %d outside 0..%d", name, b,
                  per_host[b], n);
  return SWAN_OK;
}

// A source's checks; queries of `batch` sequences.  need_ptrs: for a launch.
swan_status check_source(const swan_prefix* s, int32_t batch, bool need_ptrs) {
  if (!s) return fail(SWAN_ERR_INVALID_ARG, "prefix is NULL");
  swan_status st = check_cache_shape(s->cache);
  if (st != SWAN_OK) return st;
  const swan_cache* c = s->cache;
  if ((st = check_k(c, s->k_active_host, s->k_value_host)) != SWAN_OK) return st;
  if (need_ptrs && (st = check_cache_ptrs(c)) != SWAN_OK) return st;
  if (!s->seq_len_host || !s->of_host)
    return fail(SWAN_ERR_INVALID_ARG, "prefix: seq_len_host / of_host is NULL");
  for (int p = 0; p < c->batch; ++p) {
    const int64_t L = s->seq_len_host[p];
    if (L < 0 || L > INT32_MAX / 2)
      return fail(SWAN_ERR_INVALID_ARG, "prefix: seq_len[%d] = %lld", p, (long long)L);
    if (L - c->buffer_tokens > c->sparse_capacity)
      return fail(SWAN_ERR_CAPACITY, "prefix: sequence %d has %lld sparse tokens, capacity %d", p,
                  (long long)(L - c->buffer_tokens), c->sparse_capacity);
  }
  for (int b = 0; b < batch; ++b)
    if (s->of_host[b] < -1 || s->of_host[b] >= c->batch)
      return fail(SWAN_ERR_INVALID_ARG, "prefix: of[%d] = %d outside -1..%d", b, s->of_host[b],
                  c->batch - 1);
  return SWAN_OK;
}

// key tiles of a cache sequence: pages, then its buffer's
int key_tiles(const swan_cache* c, int L) {
  const int S = L > c->buffer_tokens ? L - c->buffer_tokens : 0;
  return swan::pages_for(S) + swan::pages_for(L < c->buffer_tokens ? L : c->buffer_tokens);
}

// Groups and splits of a source: one group per cache sequence with tokens and query rows.
// Every split has a tile; used[b] = splits of query
// sequence b's group (0: none).  Returns the largest.
// before[b], pos[b]: with a window, the position of the source's first token, and of query
// sequence b's first row.
int plan_pages(const swan_prefix* s, int32_t batch, int32_t n, const int32_t* n_host,
               const Window& w, const int32_t* before, const int32_t* pos, swan::AttendLaunch& a,
               int16_t* used) {
  const swan_cache* c = s->cache;
  const int G = c->n_q_heads / c->n_kv_heads;
  swan::SeqTab tab;
  int64_t bytes[2];
  fill_layout(c, s->k_active_host, s->k_value_host, tab, bytes);
  a.groups = 0;
  int entries = 0;
  bool many = false;  // a group fills more than a tile of kTileRows
  for (int b = 0; b < batch; ++b) used[b] = 0;
  for (int p = 0; p < c->batch; ++p) {
    if (s->seq_len_host[p] == 0) continue;
    const int j = a.groups, e0 = entries;
    int64_t toks = 0;
    for (int b = 0; b < batch; ++b) {
      const int nb = n_host ? n_host[b] : n;
      if (s->of_host[b] != p || nb == 0) continue;
      a.seq[entries] = (uint8_t)b;
      a.tok0[entries] = (int32_t)toks;
      if (w.window > 0) {
        a.lo[entries] = pos[b] - before[b] - w.window + 1;
        a.sink[entries] = (uint16_t)(w.sinks > before[b] ? w.sinks - before[b] : 0);
      }
      ++entries;
      toks += nb;
    }
    if (!toks) continue;
    a.first[j] = e0;
    a.toks[j] = (int32_t)toks;
    a.keys[j] = s->seq_len_host[p];
    a.cseq[j] = p;
    for (int r = 0; r < 2; ++r) {
      a.off[r][j] = tab.page_off[r][p];
      a.kact[r][j] = tab.kact[r][p];
    }
    many |= c->dtype != SWAN_F32 && toks * G > swan::kTileRows;
    ++a.groups;
  }
  int tiles[SWAN_MAX_BATCH];
  int64_t base[SWAN_MAX_BATCH], wide[SWAN_MAX_BATCH], rows = 0;  // row tiles x kv heads
  a.first[a.groups] = entries;
  for (int j = 0; j < a.groups; ++j) {
    const int64_t r = (int64_t)a.toks[j] * G;
    tiles[j] = key_tiles(c, a.keys[j]);
    if (w.window > 0) {  // (the most that a row tile has: Seen::find of all rows)
      const int L = a.keys[j], S = L > c->buffer_tokens ? L - c->buffer_tokens : 0;
      int lo = INT32_MAX, sink = 0;
      for (int e = a.first[j]; e < a.first[j + 1]; ++e) {
        lo = a.lo[e] < lo ? a.lo[e] : lo;
        sink = a.sink[e] > sink ? a.sink[e] : sink;
      }
      const int skip = lo >= S ? swan::pages_for(S) : (lo > 0 ? lo : 0) / swan::kPage;
      const int sink_tiles = swan::pages_for(sink < S ? sink : S);
      tiles[j] -= skip - (sink_tiles < skip ? sink_tiles : skip);
      if (tiles[j] < 1) tiles[j] = 1;
    }
    base[j] = (r + swan::kTileRows - 1) / swan::kTileRows * c->n_kv_heads;
    wide[j] = (r + swan::kManyRows - 1) / swan::kManyRows * c->n_kv_heads;
    rows += (int64_t)a.toks[j] * c->n_q_heads;
  }
  double cost, cost_many;
  int per = plan_tiles(attend_cost(c->dtype, true), a.groups, base, tiles, rows, false, true, cost);
  a.tile_rows = swan::kTileRows;
  if (many) {
    const int p = plan_tiles(attend_cost(c->dtype, true, true), a.groups, wide, tiles, rows, false,
                             true, cost_many);
    if (cost_many < cost) {
      per = p;
      a.tile_rows = swan::kManyRows;
      memcpy(base, wide, sizeof(base));
    }
  }
  int most = 0;
  int64_t units = 0;
  for (int j = 0; j < a.groups; ++j) {
    const int ns = (tiles[j] + per - 1) / per;
    a.nsplit[j] = ns;
    a.unit0[j] = (int32_t)units;
    units += base[j] * ns;
    for (int e = a.first[j]; e < a.first[j + 1]; ++e) used[a.seq[e]] = (int16_t)ns;
    most = ns > most ? ns : most;
  }
  a.unit0[a.groups] = (int32_t)units;
  a.units = units > INT32_MAX ? -1 : (int)units;
  a.by_g.set((uint32_t)G);
  a.by_hkv.set((uint32_t)c->n_kv_heads);
  a.B = batch;
  a.Hq = c->n_q_heads;
  a.Hkv = c->n_kv_heads;
  a.n = n;
  a.bb = c->buffer_tokens;
  a.npc = swan::pages_for(c->sparse_capacity);
  a.k = c->k_pages;
  a.v = c->v_pages;
  a.k_ring = c->k_ring;
  a.v_ring = c->v_ring;
  a.dtype = c->dtype;
  a.o0 = nullptr;
  a.lse0 = nullptr;
  a.out = nullptr;
  a.qmult = 0.f;
  a.m = a.causal = 0;
  a.window = w.window;
  return most;
}

swan_status check_window(int32_t window, int32_t sinks) {
  if (window < 1) return fail(SWAN_ERR_INVALID_ARG, "window %d < 1", window);
  if (sinks < 0 || sinks > swan::kMaxSinks)
    return fail(SWAN_ERR_INVALID_ARG, "sinks %d outside 0..%d", sinks, swan::kMaxSinks);
  return SWAN_OK;
}

swan_status attend_prep(const swan_prefix* sources, int32_t n_sources, int32_t batch, int32_t n,
                        const int32_t* n_host, bool need_ptrs, AttendPlan& pl, const Window& w) {
  if (!sources || n_sources < 1 || n_sources > 2)
    return fail(SWAN_ERR_INVALID_ARG, "sources is NULL, or n_sources %d outside 1..2", n_sources);
  if (batch < 1 || batch > SWAN_MAX_BATCH)
    return fail(SWAN_ERR_INVALID_ARG, "batch %d outside 1..%d", batch, SWAN_MAX_BATCH);
  swan_status st = check_rows("n", n_host, batch, n);
  if (st != SWAN_OK) return st;
  for (int s = 0; s < n_sources; ++s)
    if ((st = check_source(&sources[s], batch, need_ptrs)) != SWAN_OK) return st;
  const swan_cache* c = sources[0].cache;
  if (n_sources == 2) {
    const swan_cache* d = sources[1].cache;
    if (c->n_q_heads != d->n_q_heads || c->n_kv_heads != d->n_kv_heads ||
        elem_bytes(c->dtype) != elem_bytes(d->dtype))
      return fail(SWAN_ERR_INVALID_ARG, "the sources differ in heads or element type");
  }
  if ((int64_t)batch * c->n_q_heads * n > INT32_MAX)
    return fail(SWAN_ERR_UNSUPPORTED, "%d sequences x %d heads x %d rows: above 2^31 - 1", batch,
                c->n_q_heads, n);
  // positions: the first source's tokens, the second's, the rows
  int32_t before[2][SWAN_MAX_BATCH] = {}, pos[SWAN_MAX_BATCH] = {};
  for (int b = 0; w.window > 0 && b < batch; ++b) {
    int64_t at = 0;
    for (int s = 0; s < n_sources; ++s) {
      before[s][b] = (int32_t)at;
      if (sources[s].of_host[b] >= 0) at += sources[s].seq_len_host[sources[s].of_host[b]];
    }
    if (at + n > INT32_MAX)
      return fail(SWAN_ERR_UNSUPPORTED, "sequence %d: %lld cached tokens and %d rows: above 2^31 - 1",
                  b, (long long)at, n);
    pos[b] = w.pos ? w.pos[b] : (int32_t)at;
  }
  pl.slots = 0;
  for (int s = 0; s < 2; ++s) {
    pl.base[s] = pl.slots;
    if (s < n_sources) {
      pl.slots += plan_pages(&sources[s], batch, n, n_host, w, before[s], pos, pl.a[s], pl.used[s]);
      if (pl.a[s].units < 0) return fail(SWAN_ERR_UNSUPPORTED, "too many rows for one call");
    } else {
      pl.a[s].groups = 0;
      for (int b = 0; b < SWAN_MAX_BATCH; ++b) pl.used[s][b] = 0;
    }
  }
  const size_t rows = (size_t)batch * c->n_q_heads * n;
  pl.qhat = round256(rows * swan::kD * sizeof(float));
  pl.bytes = pl.qhat + rows * pl.slots * swan::kPartFloats * sizeof(float);
  return SWAN_OK;
}

swan_status prompt_prep(int32_t dtype, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                        int32_t n, int32_t m, int32_t head_dim, const int32_t* n_host, const int32_t* m_host,
                        int32_t causal, PromptPlan& pl, int32_t window, const int32_t* sinks_host) {
  if (!dtype_ok(dtype)) return fail(SWAN_ERR_UNSUPPORTED, "dtype %d not supported", dtype);
  if (batch < 1 || batch > SWAN_MAX_BATCH)
    return fail(SWAN_ERR_INVALID_ARG, "batch %d outside 1..%d", batch, SWAN_MAX_BATCH);
  if (n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads != 0)
    return fail(SWAN_ERR_INVALID_ARG, "n_q_heads %d is not a multiple of n_kv_heads %d", n_q_heads,
                n_kv_heads);
  if (head_dim != SWAN_HEAD_DIM)
    return fail(SWAN_ERR_UNSUPPORTED, "head_dim %d: the GPU path supports %d only", head_dim,
                SWAN_HEAD_DIM);
  swan_status st = check_rows("n", n_host, batch, n);
  if (st != SWAN_OK) return st;
  if ((st = check_rows("m", m_host, batch, m)) != SWAN_OK) return st;
  if (causal != 0 && causal != 1) return fail(SWAN_ERR_INVALID_ARG, "causal %d", causal);
  for (int b = 0; window > 0 && sinks_host && b < batch; ++b)
    if ((st = check_window(window, sinks_host[b])) != SWAN_OK) return st;
  if ((int64_t)batch * n_q_heads * n > INT32_MAX)
    return fail(SWAN_ERR_UNSUPPORTED, "%d sequences x %d heads x %d rows: above 2^31 - 1", batch,
                n_q_heads, n);
  swan::AttendLaunch& a = pl.a;
  const int G = n_q_heads / n_kv_heads;
  // sequences with the most keys first: the longest workgroups start first
  int order[SWAN_MAX_BATCH], count = 0;
  for (int b = 0; b < batch; ++b) {
    pl.used[b] = 0;
    if ((n_host ? n_host[b] : n) == 0) continue;
    int at = count++;
    const int keys = m_host ? m_host[b] : m;
    while (at > 0 && (m_host ? m_host[order[at - 1]] : m) < keys) {
      order[at] = order[at - 1];
      --at;
    }
    order[at] = b;
  }
  int tiles[SWAN_MAX_BATCH];
  int64_t base[SWAN_MAX_BATCH], rows = 0, all = 0, seen = 0;
  for (int j = 0; j < count; ++j) {
    const int b = order[j];
    a.first[j] = j;
    a.seq[j] = (uint8_t)b;
    a.cseq[j] = b;
    a.tok0[j] = 0;
    a.toks[j] = n_host ? n_host[b] : n;
    a.keys[j] = m_host ? m_host[b] : m;
    tiles[j] = (a.keys[j] + swan::kTileKeys - 1) / swan::kTileKeys;
    all += tiles[j];
    if (window > 0) {  // the tiles that a row tile's windows and the first keys take at most
      a.sink[j] = (uint16_t)(sinks_host ? sinks_host[b] : 0);
      const int64_t most = ((int64_t)window + swan::kTileRows / G + 1 + a.sink[j] +
                            swan::kTileKeys - 1) / swan::kTileKeys;
      if (most < tiles[j]) tiles[j] = (int)most;
    }
    seen += tiles[j];
    base[j] = ((int64_t)a.toks[j] * G + swan::kTileRows - 1) / swan::kTileRows * n_kv_heads;
    rows += (int64_t)a.toks[j] * n_q_heads;
  }
  a.first[count] = count;
  a.groups = count;
  double cost;
  // (windows that leave out half of a prompt's tiles make its row tiles alike, and mask more of
  // their tiles: float32 10 us each with the mask)
  AttendCost costs = attend_cost(dtype, false);
  if (window > 0 && dtype == SWAN_F32) costs.tile = 10.0;
  const int per = plan_tiles(costs, count, base, tiles, rows, causal != 0 && 2 * seen > all, false,
                             cost);
  int64_t units = 0;
  int most = 1;
  for (int j = 0; j < count; ++j) {
    const int ns = tiles[j] > per ? (tiles[j] + per - 1) / per : 1;
    a.nsplit[j] = ns;
    a.unit0[j] = (int32_t)units;
    units += base[j] * ns;
    most = ns > most ? ns : most;
    pl.used[order[j]] = (int16_t)ns;
    if (units > INT32_MAX) return fail(SWAN_ERR_UNSUPPORTED, "too many rows for one call");
  }
  a.unit0[count] = (int32_t)units;
  a.units = (int)units;
  a.by_g.set((uint32_t)G);
  a.by_hkv.set((uint32_t)n_kv_heads);
  a.B = batch;
  a.Hq = n_q_heads;
  a.Hkv = n_kv_heads;
  a.n = n;
  a.m = m;
  a.causal = causal;
  a.window = window;
  a.slots = most;
  a.slot0 = 0;
  a.k_ring = a.v_ring = nullptr;
  a.bb = a.npc = 0;
  pl.bytes = most == 1 ? 0
                       : (size_t)batch * n_q_heads * n * most * swan::kPartFloats * sizeof(float);
  return SWAN_OK;
}

// decode entry points with a prefix: the prefix's plan beside the own cache's
swan_status prefix_prep(const swan_prefix* prefix, const swan_cache* c, bool need_ptrs,
                        AttendPlan& pl) {
  swan_status st = check_cache_shape(c);
  if (st != SWAN_OK) return st;
  if ((st = attend_prep(prefix, 1, c->batch, 1, nullptr, need_ptrs, pl)) != SWAN_OK) return st;
  const swan_cache* p = prefix->cache;
  if (p->n_q_heads != c->n_q_heads || p->n_kv_heads != c->n_kv_heads ||
      elem_bytes(p->dtype) != elem_bytes(c->dtype))
    return fail(SWAN_ERR_INVALID_ARG, "the prefix's cache differs in heads or element type");
  return SWAN_OK;
}

size_t prefix_part_bytes(const swan_cache* c, const AttendPlan& pl) {
  return (size_t)c->batch * c->n_q_heads * pl.slots * swan::kPartFloats * sizeof(float);
}

// the shortest own length that a decode call behind `prefix` takes: 0 where every
// sequence has a prefix token
swan_status check_some_token(const swan_prefix* prefix, const swan_cache* c,
                             const int32_t* seq_len_host) {
  if (!seq_len_host) return fail(SWAN_ERR_INVALID_ARG, "seq_len_host is NULL");
  for (int b = 0; b < c->batch; ++b) {
    const int p = prefix->of_host[b];
    if (seq_len_host[b] < 1 && (p < 0 || prefix->seq_len_host[p] < 1))
      return fail(SWAN_ERR_INVALID_ARG, "sequence %d has no token, of its own or of a prefix", b);
  }
  return SWAN_OK;
}

// after decode_prep of the own cache: attention over both, joined
hipError_t launch_decode_prefix(swan::DecodeLaunch& da, AttendPlan& pl, void* workspace,
                                size_t decode_bytes) {
  da.leave_partials = 1;
  hipError_t e = swan::launch_decode(da);
  if (e != hipSuccess) return e;
  swan::AttendLaunch& a = pl.a[0];
  a.q = da.qhat;
  a.part = (float*)((char*)workspace + round256(decode_bytes));
  a.slots = pl.slots;
  a.slot0 = 0;
  a.stream = da.stream;
  if (a.units > 0 && (e = swan::launch_attend_pages(a)) != hipSuccess) return e;
  swan::JoinLaunch j;
  j.part = a.part;
  j.o0 = j.lse0 = nullptr;
  j.P_vo = da.P_vo;
  j.out = da.out;
  j.o = j.lse = nullptr;
  j.B = da.B;
  j.H = da.Hq;
  j.Hkv = da.Hkv;
  j.n = 1;
  j.slots = pl.slots;
  j.dtype = da.dtype;
  j.decode = 1;
  j.own_slots = da.n_splits;
  j.own = da.part;
  j.own_bb = da.bb;
  j.own_tab = da.tab;
  for (int b = 0; b < SWAN_MAX_BATCH; ++b) {
    j.used[0][b] = b < da.B ? pl.used[0][b] : 0;
    j.used[1][b] = 0;
    j.rows[b] = 1;
  }
  j.base[0] = j.base[1] = 0;
  j.stream = da.stream;
  return swan::launch_join(j);
}

swan_status attend_run(const swan_prefix* sources, int32_t n_sources, int32_t batch, int32_t n,
                       const int32_t* n_host, const Window& w, const void* q, const float* P_qk,
                        const float* P_vo, float scale, float* o, float* lse, void* workspace,
                        size_t workspace_bytes, void* stream) {
  AttendPlan pl;
  swan_status st = attend_prep(sources, n_sources, batch, n, n_host, true, pl, w);
  if (st != SWAN_OK) return st;
  if ((st = check_scale(scale)) != SWAN_OK) return st;
  int32_t rows[SWAN_MAX_BATCH] = {};
  bool any = false;
  for (int b = 0; b < batch; ++b) {
    rows[b] = n_host ? n_host[b] : n;
    any |= rows[b] > 0;
  }
  if (!any) return ok();
  if (!q || !P_qk || !o || !lse) return fail(SWAN_ERR_INVALID_ARG, "q / P_qk / o / lse is NULL");
  if ((((uintptr_t)q | (uintptr_t)P_qk | (uintptr_t)P_vo | (uintptr_t)o) & 15) != 0)
    return fail(SWAN_ERR_INVALID_ARG, "q / P_qk / P_vo / o must be 16-byte aligned");
  if (!workspace || workspace_bytes < pl.bytes)
    return fail(SWAN_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace_bytes, pl.bytes);
  if (((uintptr_t)workspace & 255) != 0)
    return fail(SWAN_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  const swan_cache* c = sources[0].cache;
  const int64_t n_rows = (int64_t)batch * c->n_q_heads * n;
  if (overlap(o, n_rows * SWAN_HEAD_DIM * 4, lse, n_rows * 4))
    return fail(SWAN_ERR_INVALID_ARG, "o and lse overlap");
  float* qhat = (float*)workspace;
  float* part = (float*)((char*)workspace + pl.qhat);
  swan::RotateLaunch r;
  r.x = q;
  r.P = P_qk;
  r.y = qhat;
  r.mult = scale_or_default(scale) * 1.4426950408889634f;
  r.x_dtype = c->dtype == SWAN_F32 ? SWAN_F32 : SWAN_F16;
  r.transposed = 0;
  r.B = batch;
  r.H = c->n_q_heads;
  r.Hkv = c->n_kv_heads;
  r.n = n;
  for (int b = 0; b < SWAN_MAX_BATCH; ++b) r.rows[b] = b < batch ? rows[b] : 0;
  r.stream = (hipStream_t)stream;
  hipError_t e = swan::launch_rotate_rows(r);
  if (e != hipSuccess) return hip_status(e, "rotate launch");
  for (int s = 0; s < n_sources; ++s) {
    swan::AttendLaunch& a = pl.a[s];
    if (a.units == 0) continue;
    a.q = qhat;
    a.part = part;
    a.slots = pl.slots;
    a.slot0 = pl.base[s];
    a.stream = (hipStream_t)stream;
    if ((e = swan::launch_attend_pages(a)) != hipSuccess) return hip_status(e, "attend launch");
  }
  swan::JoinLaunch j;
  j.part = part;
  j.o0 = j.lse0 = nullptr;
  j.P_vo = nullptr;
  j.out = nullptr;
  j.o = P_vo ? qhat : o;  // q_hat's place is free by now
  j.lse = lse;
  j.B = batch;
  j.H = c->n_q_heads;
  j.Hkv = c->n_kv_heads;
  j.n = n;
  j.slots = pl.slots;
  j.dtype = c->dtype;
  j.decode = 0;
  j.own_slots = 0;
  j.own = nullptr;
  j.own_bb = 0;
  for (int b = 0; b < SWAN_MAX_BATCH; ++b) {
    for (int s = 0; s < 2; ++s) j.used[s][b] = b < batch ? pl.used[s][b] : 0;
    j.rows[b] = b < batch ? rows[b] : 0;
  }
  j.base[0] = pl.base[0];
  j.base[1] = pl.base[1];
  j.stream = (hipStream_t)stream;
  if ((e = swan::launch_join(j)) != hipSuccess) return hip_status(e, "join launch");
  if (!P_vo) return ok();
  r.x = qhat;
  r.P = P_vo;
  r.y = o;
  r.mult = 1.f;
  r.x_dtype = SWAN_F32;
  r.transposed = 1;
  return hip_status(swan::launch_rotate_rows(r), "rotate launch");
}

swan_status prompt_run(const void* q, const void* k, const void* v, int32_t dtype,
                       int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                       int32_t n, int32_t m, int32_t head_dim, const int32_t* n_host,
                       const int32_t* m_host, int32_t causal, int32_t window,
                       const int32_t* sinks_host, float scale,
                       const float* o0, const float* lse0, void* out,
                       void* workspace, size_t workspace_bytes, void* stream) {
  PromptPlan pl;
  swan_status st = prompt_prep(dtype, batch, n_q_heads, n_kv_heads, n, m, head_dim, n_host, m_host,
                               causal, pl, window, sinks_host);
  if (st != SWAN_OK) return st;
  if ((st = check_scale(scale)) != SWAN_OK) return st;
  if ((o0 == nullptr) != (lse0 == nullptr))
    return fail(SWAN_ERR_INVALID_ARG, "pass both parts of the state or neither");
  if (pl.a.groups == 0) return ok();
  bool any_key = false;
  for (int j = 0; j < pl.a.groups; ++j) any_key |= pl.a.keys[j] > 0;
  if (!q || !out || (any_key && (!k || !v)))
    return fail(SWAN_ERR_INVALID_ARG, "q / k / v / out is NULL");
  const void* ptrs[5] = {q, k, v, o0, out};
  for (const void* p : ptrs)
    if (((uintptr_t)p & 15) != 0)
      return fail(SWAN_ERR_INVALID_ARG, "q / k / v / o0 / out must be 16-byte aligned");
  if (pl.bytes > 0) {
    if (!workspace || workspace_bytes < pl.bytes)
      return fail(SWAN_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace_bytes,
                  pl.bytes);
    if (((uintptr_t)workspace & 255) != 0)
      return fail(SWAN_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  }
  const int64_t es = elem_bytes(dtype), row = (int64_t)batch * SWAN_HEAD_DIM;
  const int64_t q_bytes = row * n_q_heads * n * es, kv_bytes = row * n_kv_heads * m * es;
  if (overlap(out, q_bytes, q, q_bytes) || overlap(out, q_bytes, k, kv_bytes) ||
      overlap(out, q_bytes, v, kv_bytes) || overlap(out, q_bytes, o0, row * n_q_heads * n * 4) ||
      overlap(out, q_bytes, lse0, (int64_t)batch * n_q_heads * n * 4))
    return fail(SWAN_ERR_INVALID_ARG, "out overlaps q, k, v or the state");
  swan::AttendLaunch& a = pl.a;
  a.q = q;
  a.o0 = o0;
  a.lse0 = lse0;
  a.out = out;
  a.part = pl.bytes > 0 ? (float*)workspace : nullptr;
  a.k = k;
  a.v = v;
  a.qmult = scale_or_default(scale) * 1.4426950408889634f;
  a.dtype = dtype == SWAN_F32 ? SWAN_F32 : SWAN_F16;
  a.stream = (hipStream_t)stream;
  hipError_t e = swan::launch_attend_dense(a);
  if (e != hipSuccess || !a.part) return hip_status(e, "prompt attention launch");
  swan::JoinLaunch j;
  j.part = a.part;
  j.o0 = o0;
  j.lse0 = lse0;
  j.P_vo = nullptr;
  j.out = out;
  j.o = j.lse = nullptr;
  j.B = batch;
  j.H = n_q_heads;
  j.Hkv = n_kv_heads;
  j.n = n;
  j.slots = a.slots;
  j.dtype = a.dtype;
  j.decode = 0;
  j.own_slots = 0;
  j.own = nullptr;
  j.own_bb = 0;
  for (int b = 0; b < SWAN_MAX_BATCH; ++b) {
    j.used[0][b] = b < batch ? pl.used[b] : 0;
    j.used[1][b] = 0;
    j.rows[b] = b < batch ? (n_host ? n_host[b] : n) : 0;
  }
  j.base[0] = j.base[1] = 0;
  j.stream = a.stream;
  return hip_status(swan::launch_join(j), "join launch");
}

swan_status rope_prep(const void* x, void* y, int32_t dtype, int32_t batch, int32_t n_heads,
                      int32_t n, int32_t head_dim, const int32_t* pos0_host, double base,
                      void* stream, swan::RopeLaunch& a) {
  if (!dtype_ok(dtype)) return fail(SWAN_ERR_UNSUPPORTED, "dtype %d not supported", dtype);
  if (head_dim != SWAN_HEAD_DIM)
    return fail(SWAN_ERR_UNSUPPORTED, "head_dim %d: the GPU path supports %d only", head_dim,
                SWAN_HEAD_DIM);
  if (batch < 1 || batch > SWAN_MAX_BATCH || n_heads < 1 || n < 0)
    return fail(SWAN_ERR_INVALID_ARG, "batch %d, n_heads %d, n %d", batch, n_heads, n);
  if (!(base > 1.0) || isinf(base)) return fail(SWAN_ERR_INVALID_ARG, "base must be > 1");
  if (!pos0_host) return fail(SWAN_ERR_INVALID_ARG, "pos0_host is NULL");
  if (n == 0) return SWAN_OK;
  if (!x || !y) return fail(SWAN_ERR_INVALID_ARG, "x / y is NULL");
  if ((((uintptr_t)x | (uintptr_t)y) & 15) != 0)
    return fail(SWAN_ERR_INVALID_ARG, "x / y must be 16-byte aligned");
  a.x = x;
  a.y = y;
  a.B = batch;
  a.H = n_heads;
  a.n = n;
  a.dtype = dtype;
  for (int b = 0; b < SWAN_MAX_BATCH; ++b) {
    if (b < batch && (pos0_host[b] < 0 || (int64_t)pos0_host[b] + n > INT32_MAX))
      return fail(SWAN_ERR_INVALID_ARG, "pos0[%d] = %d out of range", b, pos0_host[b]);
    a.pos0[b] = b < batch ? pos0_host[b] : 0;
  }
  a.base = base;
  a.stream = (hipStream_t)stream;
  return SWAN_OK;
}

swan_status qkv_rows_prep(const void* qkv, int64_t seq_stride, int64_t row_stride, int32_t dtype,
                          int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t n,
                          int32_t head_dim, const int32_t* pos0_host, double base,
                          const void* q_weight, const void* k_weight, int32_t weights_per_head,
                          int32_t weights_f32, double eps, void* q, void* k, void* v,
                          void* stream, swan::QkvRowsLaunch& a) {
  if (!dtype_ok(dtype)) return fail(SWAN_ERR_UNSUPPORTED, "dtype %d not supported", dtype);
  if (head_dim != SWAN_HEAD_DIM)
    return fail(SWAN_ERR_UNSUPPORTED, "head_dim %d: the GPU path supports %d only", head_dim,
                SWAN_HEAD_DIM);
  if (batch < 1 || batch > SWAN_MAX_BATCH || n < 0)
    return fail(SWAN_ERR_INVALID_ARG, "batch %d, n %d", batch, n);
  if (n_q_heads < 0 || n_kv_heads < 0 || n_q_heads + (int64_t)n_kv_heads < 1 ||
      n_q_heads + 2 * (int64_t)n_kv_heads > 65535)
    return fail(SWAN_ERR_INVALID_ARG, "n_q_heads %d, n_kv_heads %d", n_q_heads, n_kv_heads);
  if ((int64_t)batch * n > INT32_MAX)
    return fail(SWAN_ERR_INVALID_ARG, "batch %d x n %d: above 2^31 - 1 rows", batch, n);
  if (!(base > 1.0) || isinf(base)) return fail(SWAN_ERR_INVALID_ARG, "base must be > 1");
  if (!(eps >= 0.0) || isinf(eps)) return fail(SWAN_ERR_INVALID_ARG, "eps must be finite, >= 0");
  if ((weights_per_head != 0 && weights_per_head != 1) || (weights_f32 != 0 && weights_f32 != 1))
    return fail(SWAN_ERR_INVALID_ARG, "weights_per_head %d, weights_f32 %d: 0 or 1",
                weights_per_head, weights_f32);
  if (!pos0_host) return fail(SWAN_ERR_INVALID_ARG, "pos0_host is NULL");
  if (n == 0) return SWAN_OK;
  const int64_t width = (n_q_heads + 2 * (int64_t)n_kv_heads) * SWAN_HEAD_DIM;
  if (row_stride < width || row_stride % 8 != 0 || seq_stride < 0 || seq_stride % 8 != 0)
    return fail(SWAN_ERR_INVALID_ARG,
                "strides %lld (sequence) and %lld (row of %lld): multiples of 8, a row at least",
                (long long)seq_stride, (long long)row_stride, (long long)width);
  if (!qkv || (n_q_heads && !q) || (n_kv_heads && (!k || !v)))
    return fail(SWAN_ERR_INVALID_ARG, "qkv / q / k / v is NULL");
  const void* ptrs[6] = {qkv, q, k, v, q_weight, k_weight};
  for (const void* p : ptrs)
    if (((uintptr_t)p & 15) != 0)
      return fail(SWAN_ERR_INVALID_ARG, "pointers must be 16-byte aligned");
  a.x = qkv;
  a.seq = seq_stride;
  a.row = row_stride;
  a.head = SWAN_HEAD_DIM;
  a.out[0] = q;
  a.out[1] = k;
  a.out[2] = v;
  a.w[0] = q_weight;
  a.w[1] = k_weight;
  a.wstep = weights_per_head ? SWAN_HEAD_DIM : 0;
  a.w32 = weights_f32;
  a.B = batch;
  a.Hq = n_q_heads;
  a.Hkv = n_kv_heads;
  a.n = n;
  a.dtype = dtype;
  a.eps = eps;
  a.base = base;
  for (int b = 0; b < SWAN_MAX_BATCH; ++b) {
    if (b < batch && (pos0_host[b] < 0 || (int64_t)pos0_host[b] + n > INT32_MAX))
      return fail(SWAN_ERR_INVALID_ARG, "pos0[%d] = %d out of range", b, pos0_host[b]);
    a.pos0[b] = b < batch ? pos0_host[b] : 0;
  }
  // the outputs and the rows read share no byte
  const int64_t es = elem_bytes(dtype), each = (int64_t)batch * n * SWAN_HEAD_DIM * es;
  const void* lo[4] = {qkv, q, k, v};
  const int64_t size[4] = {((batch - 1) * seq_stride + (n - 1) * row_stride + width) * es,
                           each * n_q_heads, each * n_kv_heads, each * n_kv_heads};
  for (int x = 0; x < 4; ++x)
    for (int y = x + 1; y < 4; ++y)
      if (overlap(lo[x], size[x], lo[y], size[y]))
        return fail(SWAN_ERR_INVALID_ARG, "qkv, q, k and v overlap");
  a.stream = (hipStream_t)stream;
  return SWAN_OK;
}

}  // namespace swan_host

using namespace swan_host;

extern "C" {

const char* swan_last_error(void) { return g_last_error.c_str(); }

int32_t swan_version(void) { return 205; }

swan_status swan_page_bytes(int32_t dtype, int32_t k_active, size_t* bytes) {
  if (!bytes) return fail(SWAN_ERR_INVALID_ARG, "bytes is NULL");
  if (!dtype_ok(dtype)) return fail(SWAN_ERR_UNSUPPORTED, "dtype %d not supported", dtype);
  if (k_active < 1 || k_active > SWAN_HEAD_DIM)
    return fail(SWAN_ERR_INVALID_ARG, "k_active %d outside 1..%d", k_active, SWAN_HEAD_DIM);
  *bytes = (size_t)swan::page_bytes_of(value_bytes(dtype), k_active);
  return ok();
}

swan_status swan_cache_bytes(const swan_cache* c, const int32_t* k_active_host,
                             const int32_t* k_value_host, size_t* k_page_bytes,
                             size_t* v_page_bytes, size_t* ring_bytes) {
  swan_status st = check_cache_shape(c);
  if (st != SWAN_OK) return st;
  if ((st = check_k(c, k_active_host, k_value_host)) != SWAN_OK) return st;
  if (!k_page_bytes || !v_page_bytes || !ring_bytes)
    return fail(SWAN_ERR_INVALID_ARG, "output pointer is NULL");
  swan::SeqTab tab;
  int64_t bytes[2];
  fill_layout(c, k_active_host, k_value_host, tab, bytes);
  *k_page_bytes = (size_t)bytes[0];
  *v_page_bytes = (size_t)bytes[1];
  *ring_bytes = (size_t)c->batch * c->n_kv_heads * c->buffer_tokens * c->head_dim *
                elem_bytes(c->dtype);
  return ok();
}

swan_status swan_calibrate_workspace_bytes(int32_t d, size_t* bytes) {
  if (!bytes) return fail(SWAN_ERR_INVALID_ARG, "bytes is NULL");
  if (d != SWAN_HEAD_DIM)
    return fail(SWAN_ERR_UNSUPPORTED, "d %d: the GPU path supports %d only", d, SWAN_HEAD_DIM);
  *bytes = swan::kCalibWorkspace;
  return ok();
}

swan_status swan_calibrate_rotation(const float* rows, int64_t n_rows, int32_t d, float* P_out,
                                    float* sigma_out, void* workspace, size_t workspace_bytes,
                                    void* stream) {
  return swan_calibrate_rotations(rows, 1, &n_rows, d, P_out, sigma_out, workspace,
                                  workspace_bytes, stream);
}

swan_status swan_calibrate_rotations(const float* rows, int32_t count,
                                     const int64_t* n_rows_host, int32_t d, float* P_out,
                                     float* sigma_out, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  if (d != SWAN_HEAD_DIM)
    return fail(SWAN_ERR_UNSUPPORTED, "d %d: the GPU path supports %d only", d, SWAN_HEAD_DIM);
  if (!rows || !P_out) return fail(SWAN_ERR_INVALID_ARG, "rows / P_out is NULL");
  if (count < 1 || !n_rows_host)
    return fail(SWAN_ERR_INVALID_ARG, "count %d < 1, or n_rows_host is NULL", count);
  for (int32_t p = 0; p < count; ++p)
    if (n_rows_host[p] < 1 || n_rows_host[p] > INT64_MAX / 4096)
      return fail(SWAN_ERR_INVALID_ARG, "n_rows %lld (problem %d) < 1 or too large",
                  (long long)n_rows_host[p], p);
  const size_t need = swan::kCalibWorkspace * (size_t)count;
  if (!workspace || workspace_bytes < need)
    return fail(SWAN_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace_bytes, need);
  if (((uintptr_t)workspace & 15) != 0)
    return fail(SWAN_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  constexpr size_t kMat = (size_t)swan::kD * swan::kD;
  swan::CalibLaunch a;
  a.rows = rows;
  a.stream = (hipStream_t)stream;
  int64_t row = 0;
  for (int32_t p0 = 0; p0 < count; p0 += swan::kMaxCalib) {
    a.count = count - p0 < swan::kMaxCalib ? count - p0 : swan::kMaxCalib;
    for (int p = 0; p < a.count; ++p) {
      a.row0[p] = row;
      a.n_rows[p] = n_rows_host[p0 + p];
      row += a.n_rows[p];
    }
    a.P_out = P_out + p0 * kMat;
    a.sigma_out = sigma_out ? sigma_out + (size_t)p0 * swan::kD : nullptr;
    a.gram = (double*)((char*)workspace + swan::kCalibWorkspace * (size_t)p0);
    a.vecs = a.gram + a.count * kMat;
    a.part = a.vecs + a.count * kMat;
    a.lam = a.part + a.count * swan::kCalibPart;
    a.status = (int32_t*)(a.lam + (size_t)a.count * swan::kD);
    a.graded = a.status + 2 * a.count;
    hipError_t e = swan::launch_calibrate(a);
    if (e != hipSuccess) return hip_status(e, "calibrate launch");
    int32_t st_host[2 * swan::kMaxCalib] = {};  // each problem's (converged, sweeps)
    e = hipMemcpyAsync(st_host, a.status, 2 * a.count * sizeof(int32_t), hipMemcpyDeviceToHost,
                       a.stream);
    if (e != hipSuccess) return hip_status(e, "calibrate status copy");
    e = hipStreamSynchronize(a.stream);
    if (e != hipSuccess) return hip_status(e, "calibrate synchronize");
    for (int p = 0; p < a.count; ++p)
      if (!st_host[2 * p])
        return fail(SWAN_ERR_NO_CONVERGENCE,
                    "Jacobi eigensolver did not converge in %d sweeps (problem %d)",
                    st_host[2 * p + 1], p0 + p);
  }
  return ok();
}

swan_status swan_compress_append(const swan_cache* c, const int32_t* seq_len_host,
                                 const int32_t* k_active_host, const int32_t* k_value_host,
                                 const void* k_new, const void* v_new, int32_t n_new,
                                 const int32_t* n_new_host, const float* P_qk, const float* P_vo,
                                 void* stream) {
  swan::CompressLaunch a;
  bool any_new = false;
  const swan_status st = compress_prep(c, seq_len_host, k_active_host, k_value_host, k_new, v_new,
                                       n_new, n_new_host, P_qk, P_vo, stream, a, any_new);
  if (st != SWAN_OK) return st;
  if (!any_new) return ok();
  return hip_status(swan::launch_compress(a), "compress launch");
}

swan_status swan_decode_workspace_bytes(const swan_cache* c, const int32_t* seq_len_host,
                                        const int32_t* k_active_host,
                                        const int32_t* k_value_host, size_t* bytes) {
  swan_status st = check_cache_shape(c);
  if (st != SWAN_OK) return st;
  if ((st = check_k(c, k_active_host, k_value_host)) != SWAN_OK) return st;
  if (!seq_len_host || !bytes) return fail(SWAN_ERR_INVALID_ARG, "NULL argument");
  *bytes = decode_ws_bytes(c, plan_splits(c, seq_len_host, k_active_host, k_value_host, nullptr));
  return ok();
}

swan_status swan_decode_attention(const swan_cache* c, const int32_t* seq_len_host,
                                  const int32_t* k_active_host, const int32_t* k_value_host,
                                  const void* q, const float* P_qk, const float* P_vo, float scale,
                                  void* out, void* workspace, size_t workspace_bytes,
                                  void* stream) {
  return decode_impl(c, seq_len_host, k_active_host, k_value_host, q, P_qk, P_vo, scale, out,
                     workspace, workspace_bytes, stream, false);
}

swan_status swan_decode_attention_noalloc(const swan_cache* c, const int32_t* seq_len_host,
                                          const int32_t* k_active_host,
                                          const int32_t* k_value_host, const void* q,
                                          const float* P_qk, const float* P_vo, float scale,
                                          void* out, void* stream) {
  return decode_impl(c, seq_len_host, k_active_host, k_value_host, q, P_qk, P_vo, scale, out,
                     nullptr, 0, stream, true);
}

swan_status swan_decode_step(const swan_cache* c, const int32_t* seq_len_host,
                             const int32_t* k_active_host, const int32_t* k_value_host,
                             const void* k_new, const void* v_new, const void* q,
                             const float* P_qk, const float* P_vo, float scale, void* out,
                             void* workspace, size_t workspace_bytes, void* stream) {
  // every check of both halves before anything is enqueued
  swan::CompressLaunch ca;
  swan::DecodeLaunch da;
  const swan_status st = step_prep(c, seq_len_host, k_active_host, k_value_host, k_new, v_new, q,
                                   P_qk, P_vo, scale, out, workspace, workspace_bytes, stream, ca,
                                   da);
  if (st != SWAN_OK) return st;
  const hipError_t e = swan::launch_compress(ca);
  if (e != hipSuccess) return hip_status(e, "compress launch");
  return hip_status(swan::launch_decode(da), "decode launch");
}

swan_status swan_change_k(const swan_cache* src, const int32_t* k_active_src,
                          const int32_t* k_value_src, const swan_cache* dst,
                          const int32_t* k_active_dst, const int32_t* k_value_dst,
                          const int32_t* seq_len_host, void* stream) {
  swan_status st = check_cache_shape(src);
  if (st != SWAN_OK) return st;
  if ((st = check_cache_shape(dst)) != SWAN_OK) return st;
  if (src->batch != dst->batch || src->n_q_heads != dst->n_q_heads ||
      src->n_kv_heads != dst->n_kv_heads || src->buffer_tokens != dst->buffer_tokens ||
      src->dtype != dst->dtype)
    return fail(SWAN_ERR_INVALID_ARG,
                "src and dst differ in batch, heads, buffer_tokens or dtype");
  if ((st = check_k(src, k_active_src, k_value_src)) != SWAN_OK) return st;
  if ((st = check_k(dst, k_active_dst, k_value_dst)) != SWAN_OK) return st;
  if ((st = check_cache_ptrs(src)) != SWAN_OK) return st;
  if ((st = check_cache_ptrs(dst)) != SWAN_OK) return st;
  if (src->k_ring != dst->k_ring || src->v_ring != dst->v_ring)
    return fail(SWAN_ERR_INVALID_ARG, "dst must share src's ring arrays (the buffer is unchanged)");
  if (!seq_len_host) return fail(SWAN_ERR_INVALID_ARG, "seq_len_host is NULL");
  int max_pages = 0;
  for (int b = 0; b < src->batch; ++b) {
    const int64_t L = seq_len_host[b];
    if (L < 0) return fail(SWAN_ERR_INVALID_ARG, "seq_len[%d] = %lld < 0", b, (long long)L);
    const int64_t S = L > src->buffer_tokens ? L - src->buffer_tokens : 0;
    if (S > src->sparse_capacity || S > dst->sparse_capacity)
      return fail(SWAN_ERR_CAPACITY, "sequence %d has %lld sparse tokens, capacities %d / %d", b,
                  (long long)S, src->sparse_capacity, dst->sparse_capacity);
    const int np = swan::pages_for((int)S);
    if (np > max_pages) max_pages = np;
  }
  swan::SeqTab ts, td;
  int64_t bytes_src[2], bytes_dst[2];
  fill_layout(src, k_active_src, k_value_src, ts, bytes_src);
  fill_layout(dst, k_active_dst, k_value_dst, td, bytes_dst);
  // no destination page array may overlap a source one
  const char* sa[2] = {(const char*)src->k_pages, (const char*)src->v_pages};
  const char* da[2] = {(const char*)dst->k_pages, (const char*)dst->v_pages};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j)
      if (bytes_src[i] > 0 && bytes_dst[j] > 0 && da[j] < sa[i] + bytes_src[i] &&
          sa[i] < da[j] + bytes_dst[j])
        return fail(SWAN_ERR_INVALID_ARG, "dst page arrays overlap src page arrays");
  for (int r = 0; r < 2; ++r) {
    swan::ChangeKLaunch a;
    a.src = sa[r];
    a.dst = (char*)da[r];
    a.B = src->batch;
    a.Hkv = src->n_kv_heads;
    a.bb = src->buffer_tokens;
    a.npc_src = swan::pages_for(src->sparse_capacity);
    a.npc_dst = swan::pages_for(dst->sparse_capacity);
    a.max_pages = max_pages;
    a.dtype = src->dtype;
    for (int b = 0; b < SWAN_MAX_BATCH; ++b) {
      a.len[b] = b < src->batch ? seq_len_host[b] : 0;
      a.k_src[b] = ts.kact[r][b];
      a.k_dst[b] = td.kact[r][b];
      a.off_src[b] = ts.page_off[r][b];
      a.off_dst[b] = td.page_off[r][b];
    }
    a.stream = (hipStream_t)stream;
    const hipError_t e = swan::launch_change_k(a);
    if (e != hipSuccess) return hip_status(e, "change_k launch");
  }
  return ok();
}

swan_status swan_rope(const void* x, void* y, int32_t dtype, int32_t batch, int32_t n_heads,
                      int32_t n, int32_t head_dim, const int32_t* pos0_host, double base,
                      void* stream) {
  swan::RopeLaunch a;
  const swan_status st = rope_prep(x, y, dtype, batch, n_heads, n, head_dim, pos0_host, base, stream, a);
  if (st != SWAN_OK) return st;
  return n == 0 ? ok() : hip_status(swan::launch_rope(a), "rope launch");
}

swan_status swan_qkv_rows(const void* qkv, int64_t seq_stride, int64_t row_stride, int32_t dtype,
                          int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t n,
                          int32_t head_dim, const int32_t* pos0_host, double base,
                          const void* q_weight, const void* k_weight, int32_t weights_per_head,
                          int32_t weights_f32, double eps, void* q, void* k, void* v,
                          void* stream) {
  swan::QkvRowsLaunch a;
  const swan_status st = qkv_rows_prep(qkv, seq_stride, row_stride, dtype, batch, n_q_heads,
                                       n_kv_heads, n, head_dim, pos0_host, base, q_weight, k_weight,
                                       weights_per_head, weights_f32, eps, q, k, v, stream, a);
  if (st != SWAN_OK) return st;
  return n == 0 ? ok() : hip_status(swan::launch_qkv_rows(a), "qkv_rows launch");
}

swan_status swan_attend_workspace_bytes(const swan_prefix* sources, int32_t n_sources,
                                        int32_t batch, int32_t n, const int32_t* n_host,
                                        size_t* bytes) {
  if (!bytes) return fail(SWAN_ERR_INVALID_ARG, "bytes is NULL");
  AttendPlan pl;
  const swan_status st = attend_prep(sources, n_sources, batch, n, n_host, false, pl);
  if (st != SWAN_OK) return st;
  *bytes = pl.bytes;
  return ok();
}

swan_status swan_attend(const swan_prefix* sources, int32_t n_sources, int32_t batch, int32_t n,
                        const int32_t* n_host, const void* q, const float* P_qk,
                        const float* P_vo, float scale, float* o, float* lse, void* workspace,
                        size_t workspace_bytes, void* stream) {
  return attend_run(sources, n_sources, batch, n, n_host, Window(), q, P_qk, P_vo, scale, o, lse,
                    workspace, workspace_bytes, stream);
}

swan_status swan_prompt_workspace_bytes(int32_t dtype, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                                        int32_t n, int32_t m, int32_t head_dim,
                                        const int32_t* n_host, const int32_t* m_host,
                                        int32_t causal, size_t* bytes) {
  if (!bytes) return fail(SWAN_ERR_INVALID_ARG, "bytes is NULL");
  PromptPlan pl;
  const swan_status st = prompt_prep(dtype, batch, n_q_heads, n_kv_heads, n, m, head_dim, n_host, m_host,
                                     causal, pl);
  if (st != SWAN_OK) return st;
  *bytes = pl.bytes;
  return ok();
}

swan_status swan_prompt_attention(const void* q, const void* k, const void* v, int32_t dtype,
                                  int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                                  int32_t n, int32_t m, int32_t head_dim, const int32_t* n_host,
                                  const int32_t* m_host, int32_t causal, float scale,
                                  const float* o0, const float* lse0, void* out,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  return prompt_run(q, k, v, dtype, batch, n_q_heads, n_kv_heads, n, m, head_dim, n_host, m_host,
                    causal, 0, nullptr, scale, o0, lse0, out, workspace, workspace_bytes, stream);
}

swan_status swan_prefix_workspace_bytes(const swan_prefix* prefix, const swan_cache* c,
                                        const int32_t* seq_len_host,
                                        const int32_t* k_active_host,
                                        const int32_t* k_value_host, size_t* bytes) {
  size_t own = 0;
  swan_status st = swan_decode_workspace_bytes(c, seq_len_host, k_active_host, k_value_host, &own);
  if (st != SWAN_OK) return st;
  if (!bytes) return fail(SWAN_ERR_INVALID_ARG, "bytes is NULL");
  AttendPlan pl;
  if ((st = prefix_prep(prefix, c, false, pl)) != SWAN_OK) return st;
  *bytes = round256(own) + prefix_part_bytes(c, pl);
  return ok();
}

swan_status swan_decode_attention_prefix(const swan_prefix* prefix, const swan_cache* c,
                                         const int32_t* seq_len_host,
                                         const int32_t* k_active_host,
                                         const int32_t* k_value_host, const void* q,
                                         const float* P_qk, const float* P_vo, float scale,
                                         void* out, void* workspace, size_t workspace_bytes,
                                         void* stream) {
  AttendPlan pl;
  swan_status st = prefix_prep(prefix, c, true, pl);
  if (st != SWAN_OK) return st;
  if ((st = check_some_token(prefix, c, seq_len_host)) != SWAN_OK) return st;
  swan::DecodeLaunch da;
  st = decode_prep(c, seq_len_host, k_active_host, k_value_host, q, P_qk, P_vo, scale, out,
                   workspace, workspace_bytes, stream, false, da, 0);
  if (st != SWAN_OK) return st;
  const size_t own = decode_ws_bytes(c, da.n_splits);
  const size_t need = round256(own) + prefix_part_bytes(c, pl);
  if (workspace_bytes < need)
    return fail(SWAN_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace_bytes, need);
  return hip_status(launch_decode_prefix(da, pl, workspace, own), "decode launch");
}

swan_status swan_decode_step_prefix(const swan_prefix* prefix, const swan_cache* c,
                                    const int32_t* seq_len_host, const int32_t* k_active_host,
                                    const int32_t* k_value_host, const void* k_new,
                                    const void* v_new, const void* q, const float* P_qk,
                                    const float* P_vo, float scale, void* out, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  // every check of all parts before anything is enqueued
  AttendPlan pl;
  swan_status st = prefix_prep(prefix, c, true, pl);
  if (st != SWAN_OK) return st;
  if ((c->k_pages && c->k_pages == prefix->cache->k_pages) ||
      (c->k_ring && c->k_ring == prefix->cache->k_ring))
    return fail(SWAN_ERR_INVALID_ARG, "the prefix's cache is the one appended to");
  swan::CompressLaunch ca;
  swan::DecodeLaunch da;
  if ((st = step_prep(c, seq_len_host, k_active_host, k_value_host, k_new, v_new, q, P_qk, P_vo,
                      scale, out, workspace, workspace_bytes, stream, ca, da)) != SWAN_OK)
    return st;
  const size_t own = decode_ws_bytes(c, da.n_splits);
  const size_t need = round256(own) + prefix_part_bytes(c, pl);
  if (workspace_bytes < need)
    return fail(SWAN_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace_bytes, need);
  const hipError_t e = swan::launch_compress(ca);
  if (e != hipSuccess) return hip_status(e, "compress launch");
  return hip_status(launch_decode_prefix(da, pl, workspace, own), "decode launch");
}

swan_status swan_set_decode_tuning(const swan_decode_tuning* t) {
  Tuning n;
  if (t) {
    if (t->target_waves < 0 || t->target_waves > (1 << 20))
      return fail(SWAN_ERR_INVALID_ARG, "target_waves %d outside 0..%d", t->target_waves, 1 << 20);
    if (t->short_split_pages < -1 || t->short_split_pages > 4096)
      return fail(SWAN_ERR_INVALID_ARG, "short_split_pages %d outside -1..4096",
                  t->short_split_pages);
    if (t->merge_pct < -1 || t->merge_pct > 100)
      return fail(SWAN_ERR_INVALID_ARG, "merge_pct %d outside -1..100", t->merge_pct);
    if (t->side_streams < -1 || t->side_streams > swan::kSideStreams)
      return fail(SWAN_ERR_INVALID_ARG, "side_streams %d outside -1..%d", t->side_streams,
                  swan::kSideStreams);
    if (t->target_waves > 0) n.target_waves = t->target_waves;
    if (t->short_split_pages != 0) n.short_split_pages = t->short_split_pages < 0 ? 0 : t->short_split_pages;
    if (t->merge_pct != 0) n.merge_pct = t->merge_pct < 0 ? 0 : t->merge_pct;
    if (t->side_streams != 0) n.side_streams = t->side_streams < 0 ? 0 : t->side_streams;
  }
  g_tuning = n;
  return ok();
}

swan_status swan_set_profile_events(void* start_event, void* stop_event) {
  if ((start_event == nullptr) != (stop_event == nullptr))
    return fail(SWAN_ERR_INVALID_ARG, "pass both events or neither");
  g_prof_start = (hipEvent_t)start_event;
  g_prof_stop = (hipEvent_t)stop_event;
  return ok();
}

}  // extern "C"
