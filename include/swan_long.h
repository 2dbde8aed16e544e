/*
 * swan_long.h -- what sequences that run on for long take beyond swan.h and swan_layer.h, in
 * the same library and under the conventions stated there: attention that sees a sliding
 * window and a few first tokens, rotary positions in other forms, and caches whose sequences
 * are copied and shortened.
 */
#ifndef SWAN_LONG_H
#define SWAN_LONG_H

#include "swan_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Rotary positions.  swan_rope turns dims j and j + head_dim/2 by pos * base^(-2j/head_dim);
 * here the first `dims` dims of a head are turned and the others left as they are (bit for
 * bit, where there is no norm), each pair (x, y) becoming
 *     magnitude * (x cos t - y sin t, y cos t + x sin t),   t = pos * freq_host[j],
 * in float64, rounded once to the storage type.
 *  dims          8..head_dim, a multiple of 8;
 *  interleaved   0: dims j and j + dims/2 are pair j, 1: dims 2j and 2j + 1;
 *  magnitude     finite, > 0;
 *  freq_host     [dims/2] radians per position, finite.
 */
typedef struct swan_rotary {
  int32_t dims;
  int32_t interleaved;
  double magnitude;
  const double* freq_host;
} swan_rotary;

/* swan_rope and swan_qkv_rows with a swan_rotary in the place of the base; the other arguments
 * are theirs. */
swan_status swan_rope_rotary(const void* x, void* y, int32_t dtype, int32_t batch, int32_t n_heads,
                             int32_t n, int32_t head_dim, const int32_t* pos0_host,
                             const swan_rotary* rotary, void* stream);
swan_status swan_qkv_rows_rotary(const void* qkv, int64_t seq_stride, int64_t row_stride,
                                 int32_t dtype, int32_t batch, int32_t n_q_heads,
                                 int32_t n_kv_heads, int32_t n, int32_t head_dim,
                                 const int32_t* pos0_host, const swan_rotary* rotary,
                                 const void* q_weight, const void* k_weight,
                                 int32_t weights_per_head, int32_t weights_f32, double eps, void* q,
                                 void* k, void* v, void* stream);

/*
 * Attention with a sliding window: a row at position p sees the keys at positions j <= p with
 *     j > p - window  or  j < sinks,
 * so `window` counts the row's own position (>= 1), and the first `sinks` (0..65535) keys stay
 * visible to all.  Keys that no row of a workgroup's sees are not read.  Values that a row does
 * not see do not reach it, infinities and NaNs included.
 *
 * swan_prompt_attention_window: as swan_prompt_attention with causal = 1; positions are those of
 * k, v, so that row i of sequence b is at i + m_b - n_b.  sinks_host[b] per sequence (NULL:
 * none).  Behind cached tokens (a state of swan_attend_window) the first keys are cached ones:
 * pass what is left of them, max(0, sinks - cached tokens).
 */
swan_status swan_prompt_window_workspace_bytes(int32_t dtype, int32_t batch, int32_t n_q_heads,
                                               int32_t n_kv_heads, int32_t n, int32_t m,
                                               int32_t head_dim, const int32_t* n_host,
                                               const int32_t* m_host, int32_t window,
                                               const int32_t* sinks_host, size_t* bytes);
swan_status swan_prompt_attention_window(const void* q, const void* k, const void* v,
                                         int32_t dtype, int32_t batch, int32_t n_q_heads,
                                         int32_t n_kv_heads, int32_t n, int32_t m,
                                         int32_t head_dim, const int32_t* n_host,
                                         const int32_t* m_host, int32_t window,
                                         const int32_t* sinks_host, float scale, const float* o0,
                                         const float* lse0, void* out, void* workspace,
                                         size_t workspace_bytes, void* stream);

/*
 * swan_attend_window: as swan_attend; the tokens of the first source are at positions 0 .., those
 * of the second behind them, and row i of a sequence stands i positions behind its cached
 * tokens.
 */
swan_status swan_attend_window_workspace_bytes(const swan_prefix* sources, int32_t n_sources,
                                               int32_t batch, int32_t n, const int32_t* n_host,
                                               int32_t window, int32_t sinks, size_t* bytes);
swan_status swan_attend_window(const swan_prefix* sources, int32_t n_sources, int32_t batch,
                               int32_t n, const int32_t* n_host, int32_t window, int32_t sinks,
                               const void* q, const float* P_qk, const float* P_vo, float scale,
                               float* o, float* lse, void* workspace, size_t workspace_bytes,
                               void* stream);

/*
 * swan_decode_attention_window, swan_decode_step_window: as swan_decode_attention and
 * swan_decode_step, or with a prefix (not NULL) as swan_decode_attention_prefix and
 * swan_decode_step_prefix; a scale given is at least 2^-64.  The query is at the position of its
 * sequence's last token.  A step gives the same results as an append and
 * swan_decode_attention_window.  For the workspace of a step ask with the lengths after it.
 * Their plan is their own: swan_set_decode_tuning does not change it, and
 * swan_set_profile_events records nothing around them.
 */
swan_status swan_decode_window_workspace_bytes(const swan_prefix* prefix, const swan_cache* c,
                                               const int32_t* seq_len_host,
                                               const int32_t* k_active_host,
                                               const int32_t* k_value_host, int32_t window,
                                               int32_t sinks, size_t* bytes);
swan_status swan_decode_attention_window(const swan_prefix* prefix, const swan_cache* c,
                                         const int32_t* seq_len_host,
                                         const int32_t* k_active_host,
                                         const int32_t* k_value_host, int32_t window,
                                         int32_t sinks, const void* q, const float* P_qk,
                                         const float* P_vo, float scale, void* out,
                                         void* workspace, size_t workspace_bytes, void* stream);
swan_status swan_decode_step_window(const swan_prefix* prefix, const swan_cache* c,
                                    const int32_t* seq_len_host, const int32_t* k_active_host,
                                    const int32_t* k_value_host, int32_t window, int32_t sinks,
                                    const void* k_new, const void* v_new, const void* q,
                                    const float* P_qk, const float* P_vo, float scale, void* out,
                                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Sequences of a cache to places of another: for each sequence b of dst with of_host[b] >= 0,
 * sequence b becomes sequence of_host[b] of src, whose tokens first_host[b] .. first_host[b] +
 * drop_host[b] - 1 are left out (drop_host NULL: none; first_host NULL: 0).  The copy has
 * src_len_host[of] - drop tokens, numbered anew from 0: a caller that turns keys to absolute
 * positions keeps count of the tokens left out.  A window of W shows a query at the copy's last
 * token (swan_decode_attention_window) the source's tokens from src_len_host[of] - W on, the next row
 * those from one further.  Only pruned tokens can be left out, so first +
 * drop is src_len_host[of] - buffer_tokens at most.  A sequence of dst with of_host[b] = -1 stays
 * as it is, so do the slots behind a copy's last token.  The same source may be taken several
 * times.
 *  src, dst      descriptors with the same heads, buffer_tokens and dtype, whose arrays share no
 *                byte; batch and sparse_capacity may differ;
 *  k_active_*, k_value_*  as in swan_cache_bytes; a sequence and its copy have the same k
 *                (swan_change_k converts).
 * Errors: SWAN_ERR_INVALID_ARG, SWAN_ERR_CAPACITY (a copy's pruned tokens).
 */
swan_status swan_copy_sequences(const swan_cache* src, const int32_t* src_len_host,
                                const int32_t* k_active_src, const int32_t* k_value_src,
                                const swan_cache* dst, const int32_t* k_active_dst,
                                const int32_t* k_value_dst, const int32_t* of_host,
                                const int32_t* first_host, const int32_t* drop_host, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SWAN_LONG_H */
