// What the host sides of the C ABI (swan_api.hip, swan_long_api.hip) share: argument checks,
// plans and the calls that several entry points make.
#pragma once

#include "swan.h"
#include "swan_cache_ops.h"
#include "swan_layer.h"
#include "swan_layer_ops.h"

namespace swan_host __attribute__((visibility("hidden"))) {

// the calling thread's message, and the status
swan_status fail(swan_status st, const char* fmt, ...);
swan_status ok();
swan_status hip_status(hipError_t e, const char* what);

// bytes of one element of queries, outputs, new keys / values and the ring; of a sparse value
int elem_bytes(int32_t dtype);
int value_bytes(int32_t dtype);
bool dtype_ok(int32_t dtype);
size_t round256(size_t x);
// whether two ranges of bytes share one
bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes);

swan_status check_cache_shape(const swan_cache* c);
swan_status check_cache_ptrs(const swan_cache* c);
// k of the keys (k_active_host) and, if not NULL, of the values (k_value_host)
swan_status check_k(const swan_cache* c, const int32_t* k_active_host, const int32_t* k_value_host);
swan_status check_scale(float scale);
float scale_or_default(float scale);
// k of role r (0 keys, 1 values) of sequence b
inline int k_of(const int32_t* k_active_host, const int32_t* k_value_host, int r, int b) {
  return (r == 1 && k_value_host) ? k_value_host[b] : k_active_host[b];
}
// fills tab.kact and tab.page_off of both roles; bytes[r] = total page bytes of role r
void fill_layout(const swan_cache* c, const int32_t* k_active_host, const int32_t* k_value_host,
                 swan::SeqTab& tab, int64_t bytes[2]);

// swan_compress_append's validation, into `a` (nothing is enqueued); any_new: some sequence
// appends a token
swan_status compress_prep(const swan_cache* c, const int32_t* seq_len_host,
                          const int32_t* k_active_host, const int32_t* k_value_host,
                          const void* k_new, const void* v_new, int32_t n_new,
                          const int32_t* n_new_host, const float* P_qk, const float* P_vo,
                          void* stream, swan::CompressLaunch& a, bool& any_new);

// A sliding window (0: none) and the first tokens that stay visible.  pos[b]: the position of
// query sequence b's first row, the cached tokens' positions being 0 .. (NULL: behind them).
struct Window {
  int32_t window = 0, sinks = 0;
  const int32_t* pos = nullptr;
};
swan_status check_window(int32_t window, int32_t sinks);

struct AttendPlan {
  swan::AttendLaunch a[2];
  int16_t used[2][SWAN_MAX_BATCH];
  int base[2], slots;
  size_t qhat, bytes;  // bytes of q_hat; of the workspace
};
swan_status attend_prep(const swan_prefix* sources, int32_t n_sources, int32_t batch, int32_t n,
                        const int32_t* n_host, bool need_ptrs, AttendPlan& pl,
                        const Window& w = Window());
swan_status attend_run(const swan_prefix* sources, int32_t n_sources, int32_t batch, int32_t n,
                       const int32_t* n_host, const Window& w, const void* q, const float* P_qk,
                       const float* P_vo, float scale, float* o, float* lse, void* workspace,
                       size_t workspace_bytes, void* stream);

// plan of swan_prompt_attention
struct PromptPlan {
  swan::AttendLaunch a;
  int16_t used[SWAN_MAX_BATCH];
  size_t bytes;
};
// sinks_host: with a window, per sequence (NULL: none)
swan_status prompt_prep(int32_t dtype, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                        int32_t n, int32_t m, int32_t head_dim, const int32_t* n_host,
                        const int32_t* m_host, int32_t causal, PromptPlan& pl, int32_t window = 0,
                        const int32_t* sinks_host = nullptr);
swan_status prompt_run(const void* q, const void* k, const void* v, int32_t dtype, int32_t batch,
                       int32_t n_q_heads, int32_t n_kv_heads, int32_t n, int32_t m,
                       int32_t head_dim, const int32_t* n_host, const int32_t* m_host,
                       int32_t causal, int32_t window, const int32_t* sinks_host, float scale,
                       const float* o0, const float* lse0, void* out, void* workspace,
                       size_t workspace_bytes, void* stream);

// the checks of swan_rope and swan_qkv_rows, into `a` (not where n is 0: nothing to do then)
swan_status rope_prep(const void* x, void* y, int32_t dtype, int32_t batch, int32_t n_heads,
                      int32_t n, int32_t head_dim, const int32_t* pos0_host, double base,
                      void* stream, swan::RopeLaunch& a);
swan_status qkv_rows_prep(const void* qkv, int64_t seq_stride, int64_t row_stride, int32_t dtype,
                          int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t n,
                          int32_t head_dim, const int32_t* pos0_host, double base,
                          const void* q_weight, const void* k_weight, int32_t weights_per_head,
                          int32_t weights_f32, double eps, void* q, void* k, void* v, void* stream,
                          swan::QkvRowsLaunch& a);

}  // namespace swan_host
