/*
 * swan_layer.h -- what the layer code (layer.py) calls beyond swan.h, in the
 * same library and under the conventions stated there.
 */
#ifndef SWAN_LAYER_H
#define SWAN_LAYER_H

#include "swan.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * `count` problems of swan_calibrate_rotation at once, side by side on the GPU
 * (the rotations of a layer's heads; the solver of one occupies one compute
 * unit): rows holds the problems' rows one after another, n_rows_host[count] of
 * each (>= 1); P_out [count][d][d], sigma_out [count][d] or NULL, workspace
 * count times what swan_calibrate_workspace_bytes says.  Every problem's result
 * is the same as from a call of its own.
 */
swan_status swan_calibrate_rotations(const float* rows, int32_t count,
                                     const int64_t* n_rows_host, int32_t d, float* P_out,
                                     float* sigma_out, void* workspace, size_t workspace_bytes,
                                     void* stream);

/*
 * A layer's projections as the rows that its cache and attention take: [q | k | v] of
 * every token split into heads, the heads of q and k divided by their root mean square
 * and weighted (where weights are given), then rotated as by swan_rope; v as it is.
 *  qkv           rows of (n_q_heads + 2 n_kv_heads) * head_dim elements of the storage
 *                type of `dtype` (binary16 for SWAN_F16 and SWAN_F16_E4M3): row i of
 *                sequence b at qkv + b * seq_stride + i * row_stride (in elements;
 *                multiples of 8, row_stride at least a row);
 *  n_q_heads     may be 0 (q is then not written), so may n_kv_heads, not both;
 *  pos0_host[b], base  as for swan_rope;
 *  q_weight, k_weight  head_dim weights shared by the heads, or (weights_per_head = 1)
 *                [n_heads][head_dim]; float32 if weights_f32 = 1, else of the storage
 *                type; NULL: no norm of these heads;
 *  eps           x_j / sqrt(mean_j x_j^2 + eps) * w_j; finite, >= 0;
 *  q, k, v       [batch][heads][n][head_dim] of the storage type; they overlap neither
 *                each other nor the rows read.
 * Everything is computed in float64 and rounded once (there is no rounding between norm
 * and rotation), so without weights q and k have swan_rope's bits.  batch * n below 2^31.
 * Pointers 16-byte aligned.
 */
swan_status swan_qkv_rows(const void* qkv, int64_t seq_stride, int64_t row_stride, int32_t dtype,
                          int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t n,
                          int32_t head_dim, const int32_t* pos0_host, double base,
                          const void* q_weight, const void* k_weight, int32_t weights_per_head,
                          int32_t weights_f32, double eps, void* q, void* k, void* v,
                          void* stream);

/*
 * Attention of several rows per sequence.  Its results can be left as a STATE, from which
 * another call continues: per row o, the attention output in float32, and lse, the natural
 * logarithm of its softmax sum, float32 ([batch][n_q_heads][n][head_dim] and
 * [batch][n_q_heads][n]).  A row that has seen no key has o = 0 and lse = -infinity.  The
 * states of two sets of keys join to the state of both, so a chunk of a prompt attends
 * over the cached tokens first (swan_attend) and then over itself (swan_prompt_attention).
 * On the binary16 formats probabilities meet the values as two binary16 parts, within 2^-23
 * of their float32 value; sums, states and accumulators are float32 in every case.
 * Rows past a sequence's n_host[b] are neither read nor written.
 */

/*
 * Cached tokens that query sequences attend to: sequence of_host[b] of `cache` for query
 * sequence b (-1: none), so a prefix that many sequences share is held, and read, once.
 * The tokens are those in the cache when the call runs; `cache`'s n_q_heads, n_kv_heads,
 * head_dim and element type are the queries'.  The last buffer_tokens tokens of a prefix
 * stay dense.  Positions are the caller's: a prefix of L tokens takes 0 .. L - 1.
 */
typedef struct swan_prefix {
  const swan_cache* cache;
  const int32_t* seq_len_host;   /* [cache->batch] tokens cached (0 allowed) */
  const int32_t* k_active_host;  /* as in swan_cache_bytes */
  const int32_t* k_value_host;
  const int32_t* of_host;        /* [query sequences] */
} swan_prefix;

/*
 * Rows over cached tokens: state of q's rows over all tokens of up to two sources (a
 * shared prefix and the sequences' own caches).
 *  sources, n_sources  1 or 2;
 *  batch         query sequences, 1..SWAN_MAX_BATCH; n rows of each, n_host[b] of them
 *                used (NULL: all), no causal mask: every row sees every token;
 *  q             [batch][n_q_heads][n][head_dim] of the caches' element type (post-RoPE);
 *  P_qk, P_vo, scale  as in swan_decode_attention (P_vo NULL: o stays rotated);
 *                a scale given is at least 2^-64;
 *  o, lse        the state (float32), apart from each other;
 *  workspace     as swan_attend_workspace_bytes says, 256-byte aligned.
 */
swan_status swan_attend_workspace_bytes(const swan_prefix* sources, int32_t n_sources,
                                        int32_t batch, int32_t n, const int32_t* n_host,
                                        size_t* bytes);
swan_status swan_attend(const swan_prefix* sources, int32_t n_sources, int32_t batch, int32_t n,
                        const int32_t* n_host, const void* q, const float* P_qk,
                        const float* P_vo, float scale, float* o, float* lse, void* workspace,
                        size_t workspace_bytes, void* stream);

/*
 * Dense attention of a prompt's rows, or of rows over another sequence's keys and values.
 *  q             [batch][n_q_heads][n][head_dim], n_host[b] rows used (NULL: n; 0 allowed);
 *  k, v          [batch][n_kv_heads][m][head_dim], m_host[b] rows used (NULL: m; 0 allowed),
 *                the others not read; all of the storage type of `dtype`;
 *  causal        1: row i sees keys j <= i + m_b - n_b (the last row sees all), 0: all;
 *  scale         <= 0 means 1 / sqrt(head_dim), else at least 2^-64;
 *  o0, lse0      a state to continue from, or both NULL;
 *  out           [batch][n_q_heads][n][head_dim] of the storage type, not overlapping
 *                the inputs; a row that sees no key and has no state gets zeros;
 *  workspace     as swan_prompt_workspace_bytes says (0 possible: then NULL will do),
 *                256-byte aligned.
 * Values that a row does not see do not reach it, infinities and NaNs included.
 */
swan_status swan_prompt_workspace_bytes(int32_t dtype, int32_t batch, int32_t n_q_heads,
                                        int32_t n_kv_heads, int32_t n, int32_t m,
                                        int32_t head_dim, const int32_t* n_host,
                                        const int32_t* m_host, int32_t causal, size_t* bytes);
swan_status swan_prompt_attention(const void* q, const void* k, const void* v, int32_t dtype,
                                  int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                                  int32_t n, int32_t m, int32_t head_dim, const int32_t* n_host,
                                  const int32_t* m_host, int32_t causal, float scale,
                                  const float* o0, const float* lse0, void* out,
                                  void* workspace, size_t workspace_bytes, void* stream);

/*
 * swan_decode_attention and swan_decode_step with a prefix before each sequence's own
 * tokens: the softmax is over the prefix's pages and buffer and the sequence's own.  The
 * prefix's pages are read once for all the sequences that share it.  Own caches may be
 * empty (seq_len_host[b] = 0 for swan_decode_attention_prefix) where there is a prefix
 * token.  `prefix` is only read; its cache is not the one appended to.
 * swan_prefix_workspace_bytes: for swan_decode_attention_prefix with these lengths; for
 * swan_decode_step_prefix ask with the lengths after the step.
 */
swan_status swan_prefix_workspace_bytes(const swan_prefix* prefix, const swan_cache* c,
                                        const int32_t* seq_len_host,
                                        const int32_t* k_active_host,
                                        const int32_t* k_value_host, size_t* bytes);
swan_status swan_decode_attention_prefix(const swan_prefix* prefix, const swan_cache* c,
                                         const int32_t* seq_len_host,
                                         const int32_t* k_active_host,
                                         const int32_t* k_value_host, const void* q,
                                         const float* P_qk, const float* P_vo, float scale,
                                         void* out, void* workspace, size_t workspace_bytes,
                                         void* stream);
swan_status swan_decode_step_prefix(const swan_prefix* prefix, const swan_cache* c,
                                    const int32_t* seq_len_host, const int32_t* k_active_host,
                                    const int32_t* k_value_host, const void* k_new,
                                    const void* v_new, const void* q, const float* P_qk,
                                    const float* P_vo, float scale, void* out, void* workspace,
                                    size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SWAN_LAYER_H */
