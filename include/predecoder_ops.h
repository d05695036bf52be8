/*
 * predecoder_ops.h -- C ABI of the token operators (MI355X, gfx950).
 *
 * The pre-decoder of predecoder.h is local: an output sees its receptive field
 * only.  A layer that looks at a whole volume is a block of attention over its
 * sites, one token for each site of each round (the activations that
 * predecoder_activations gives, [batch][T][H][H][channels], are such tokens).
 * These are the operators of such a block, for inference:
 *
 *   predecoder_rms_norm    root-mean-square norm with the residual's addition,
 *                          its output as it is or in 8 bits with a scale a token
 *   predecoder_matmul8     product of 8-bit codes with scales for each token and
 *                          channel, bias and activation
 *   predecoder_rope        rotary positions with three axes (round, row, column)
 *   predecoder_attention   grouped-head attention with capped scores, a distance
 *                          bias and masks by volume, round and prefix
 *
 * and what a stream of rounds keeps of its past, with what reads it:
 *
 *   predecoder_cache_write, predecoder_cache_read
 *                          keys and values in a ring of places, in 8 bits with a
 *                          scale a row: quantised as they come, and read back
 *   predecoder_attention8  predecoder_attention of new tokens over such a cache
 *   predecoder_linear_attention
 *                          linear attention with a decay for each head: a state of
 *                          fixed size instead of a cache, whole rounds at a time
 *
 * Types.  bf16 (PD_DTYPE_BF16) and fp32 (PD_DTYPE_FP32) values; 8-bit codes are
 * OCP E4M3 (the library's 8-bit format) or signed integers.  Sums, norms and
 * softmax statistics are fp32 (sums of int8 products: exact int32; of E4M3
 * products for a bf16 output: see there); every
 * output is rounded once, to nearest even.  Results are bit-reproducible: no
 * operator uses atomics, and a call's order of sums depends on its sizes,
 * types and alignment alone.
 *
 * Layout.  The last axis of a matrix is contiguous; strides of the other axes
 * are in elements and may be any (rows of a wider tensor, a joint projection, a
 * cache).  Rows at 16-byte aligned addresses with lengths a multiple of 16 bytes take
 * the wide loads; others are right, and slower.
 *
 * Errors, streams.  As in predecoder.h: every function is nothrow and never
 * aborts; misuse that the host can see gives PD_ERR_INVALID_ARG (sizes or
 * strides it has no form for: PD_ERR_UNSUPPORTED) before any device call; a
 * failed launch gives PD_ERR_DEVICE.  All buffers are the caller's device
 * memory, work is enqueued on hip_stream, the host never waits, nothing is
 * allocated (calls may be recorded into HIP graphs).  The operators keep no
 * state: calls on different streams may overlap if their buffers do not.
 * Calls with no token do nothing.
 */
#ifndef PREDECODER_OPS_H
#define PREDECODER_OPS_H

#include "predecoder.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Where a token sits: its round, its row and column on the grid, and the
 * volume (logical qubit, document) that it belongs to.  volume < 0: no token
 * (padding; the unused rest of a cache). */
typedef struct pd_site {
  int32_t t, i, j, volume;
} pd_site;

typedef enum pd_codes { PD_CODES_NONE = 0, PD_CODES_E4M3 = 1, PD_CODES_INT8 = 2 } pd_codes;

/* ---- Root-mean-square norm ----
 *
 *   s = x + residual                      (residual NULL: s = x)
 *   y = s / sqrt(mean(s^2) + eps) * gain  (gain NULL: 1; mean over the row)
 * Each of these outputs may be NULL (one at least must be given):
 *   sum     s rounded to dtype (the next residual); may be x or residual
 *   out     y rounded to dtype; may be x or residual
 *   codes   y / scale rounded to codes_type, and scales (given with codes, fp32,
 *           one a row): scale = max |y| / 448 (E4M3) or / 127 (int8).  A row of
 *           zeros (s or s gain) has scale 0 and codes 0; a row whose sum of squares or
 *           whose s gain is not finite in fp32 has scale NaN and codes 0.
 * A row s of zeros has y 0, also for eps = 0; where the sum of squares alone is
 * past fp32, y is 0.  y is computed from the unrounded s.
 * 1 <= width <= 32768, rows <= 2^40.  An output must be one of the inputs itself
 * (same address and stride) or not overlap them. */
typedef struct pd_norm_args {
  int64_t rows;
  int32_t width;
  int32_t dtype;      /* of x, residual, sum and out: PD_DTYPE_BF16 or PD_DTYPE_FP32 */
  int32_t codes_type; /* pd_codes of codes (PD_CODES_NONE: codes and scales NULL) */
  float eps;          /* >= 0 */
  const void* x;
  int64_t x_stride;
  const void* residual;
  int64_t residual_stride;
  const float* gain; /* [width] */
  void* sum;
  int64_t sum_stride;
  void* out;
  int64_t out_stride;
  void* codes; /* one byte each */
  int64_t codes_stride;
  float* scales; /* [rows] */
} pd_norm_args;

pd_status predecoder_rms_norm(void* hip_stream, const pd_norm_args* args);

/* ---- Product of 8-bit codes ----
 *
 *   out[m][n] = act(a_scales[m] w_scales[n] sum_k a[m][k] w[n][k] + bias[n])
 * a: [M][K] codes of the tokens, w: [N][K] codes of the output channels, both of
 * codes_type.  int8 sums are exact (K <= 131071).  E4M3 sums are fp32 for an fp32
 * out.  For a bf16 out they are the fp8 matrix instruction's: eight neighbouring
 * products at a time, each cut below 2^-13 of the largest of the eight.  That is
 * off by at most 7 2^-13 of every eight's largest |product|, below 2^-10 of the
 * sum of |products|: less than bf16's rounding unless the sum cancels (then take
 * an fp32 out).
 * bias [N] or NULL; act: pd_act (every one of NaN is NaN); out bf16 or fp32
 * (out_dtype).  K = 0 gives act(bias). */
typedef struct pd_matmul8_args {
  int64_t M;
  int32_t N, K;
  int32_t codes_type; /* PD_CODES_E4M3 or PD_CODES_INT8 */
  int32_t out_dtype;
  int32_t act;
  const void* a;
  int64_t a_stride;
  const float* a_scales; /* [M] */
  const void* w;
  int64_t w_stride;
  const float* w_scales; /* [N] */
  const float* bias;     /* [N] or NULL */
  void* out;
  int64_t out_stride;
} pd_matmul8_args;

pd_status predecoder_matmul8(void* hip_stream, const pd_matmul8_args* args);

/* ---- Rotary positions ----
 *
 * The head_dim values of a head are head_dim / 2 pairs (u, v): values m and
 * m + head_dim / 2, or 2 m and 2 m + 1 if interleaved.  The pairs are cut into
 * three runs of sections[0], sections[1] and sections[2] pairs for the axes t, i
 * and j (their sum may be less than head_dim / 2: the rest is copied); pair k of
 * a run of n turns by the angle  p base^(-k / n),  p the token's position on that axis:
 *   (u, v) -> (u cos - v sin, v cos + u sin)       (inverse: by the negative angle)
 * Angles are taken to 2^-24 of a turn up to |p| = 2^23 (base >= 1).  out is x
 * itself (same strides) or does not overlap it; rows of out do not overlap each
 * other.  head_dim even, at most 256. */
typedef struct pd_rope_args {
  int64_t tokens;
  int32_t heads, head_dim;
  int32_t dtype; /* PD_DTYPE_BF16 or PD_DTYPE_FP32 */
  int32_t sections[3];
  int32_t interleaved, inverse; /* 0 or 1 */
  double base;                  /* > 0 */
  const pd_site* sites;         /* [tokens], 16-byte aligned */
  const void* x;
  int64_t x_token_stride, x_head_stride;
  void* out;
  int64_t out_token_stride, out_head_stride;
} pd_rope_args;

pd_status predecoder_rope(void* hip_stream, const pd_rope_args* args);

/* No prefix: causal attention sees a token's own and earlier rounds alone. */
#define PD_PREFIX_NONE INT32_MIN

/* ---- Attention ----
 *
 * For query token a of head h, and key token b of head h / (heads / kv_heads):
 *   z = scale q.k;   z = cap tanh(z / cap) if cap > 0;
 *   z -= slopes[h] (|t_a - t_b| + |i_a - i_b| + |j_a - j_b|)  if slopes is given
 *   out = sum_b softmax_b(z) v_b   over the visible tokens b:
 *     volume_a = volume_b >= 0, and with causal t_b <= t_a or t_b < prefix
 * The prefix is all rounds below it, negative ones too: 0 is none where rounds
 * count up from 0, PD_PREFIX_NONE is none everywhere.
 * Without sites (both NULL) every token is visible, and slopes, causal and
 * prefix must be unset.  A query that sees nothing gets zeros; keys and values at
 * invisible places do not reach the result, whatever they hold.  bf16 values;
 * the probabilities are rounded to bf16 for their product with v (2^-8 of each),
 * and their fp32 sum is that of the rounded ones, so that the weights add up to one.
 * head_dim: a multiple of 8, at most 128; all rows (strides and addresses) of q,
 * k, v and out 16-byte aligned; heads a multiple of kv_heads, heads / kv_heads
 * <= 64; |coordinate| < 2^29.  out overlaps no input, and its rows not each other.
 * workspace: device memory of at least predecoder_attention_workspace(args)
 * bytes, 16-byte aligned (NULL if that is 0), not shared by calls that may
 * overlap.
 * Any finite cap >= 0 is taken (0: none): up to 64 within 1e-6 of the cap, above within 2^-20 of the score. */
typedef struct pd_attention_args {
  int32_t batch, heads, kv_heads, head_dim;
  int32_t n_q, n_k; /* tokens of one batch entry */
  float scale, cap;
  int32_t causal, prefix; /* causal 0 or 1; prefix >= 0, or PD_PREFIX_NONE */
  const void* q;
  int64_t q_batch_stride, q_token_stride, q_head_stride;
  const void* k;
  int64_t k_batch_stride, k_token_stride, k_head_stride;
  const void* v;
  int64_t v_batch_stride, v_token_stride, v_head_stride;
  void* out;
  int64_t out_batch_stride, out_token_stride, out_head_stride;
  const pd_site* q_sites; /* [batch][n_q], 16-byte aligned */
  int64_t q_sites_batch_stride; /* in sites; 0: one list for all */
  const pd_site* k_sites;
  int64_t k_sites_batch_stride;
  const float* slopes; /* [heads] */
  void* workspace;
  size_t workspace_bytes;
} pd_attention_args;

/* Bytes of workspace that a call with these arguments uses; 0 for invalid ones.
 * It goes by the sizes, by whether k_sites is NULL and by whether
 * k_sites_batch_stride is 0: set those as in the call.  No pointer is followed. */
size_t predecoder_attention_workspace(const pd_attention_args* args);

pd_status predecoder_attention(void* hip_stream, const pd_attention_args* args);

/* ---- Cache of keys and values in 8 bits ----
 *
 * For each batch entry (a stream) a ring of `capacity` places; a place holds the
 * keys and values of one token, and its site.  All three arrays are whole:
 *   codes   [batch][2][kv_heads][capacity][head_dim], one byte each (0: keys, 1: values)
 *   scales  [batch][2][kv_heads][capacity], fp32
 *   sites   [batch][capacity]
 * A row (the keys or values of one token and head) stands for code scale.  A place
 * whose site has volume < 0 holds no token, and its codes and scales may be
 * anything: a new cache needs its sites set so, and no more.
 * head_dim: a multiple of 16, at most 128; codes and sites 16-byte aligned;
 * batch, kv_heads <= 65535. */
typedef struct pd_cache {
  int32_t batch, kv_heads, head_dim, capacity;
  int32_t codes_type; /* PD_CODES_E4M3 or PD_CODES_INT8 */
  void* codes;
  float* scales;
  pd_site* sites;
} pd_cache;

/* Token m of entry b is at place (at[b] + m) mod capacity (at may be any number,
 * negative ones too); tokens <= capacity, so that no place comes twice (at most 2^30).
 *
 * Write: k and v [batch][tokens][kv_heads][head_dim] into the cache, with their
 * sites.  scale = max |x| / 448 (E4M3) or / 127 (int8) in fp32, codes x / scale
 * rounded once.  A row of zeros, or of values so small that its scale is 0, has
 * scale 0 and codes 0; one with a value that is not finite has scale NaN and codes 0.
 * Tokens of volume < 0 are left out: their places stay as they are.
 * k, v and sites do not overlap the cache.
 *
 * Read: code scale, rounded to dtype, of those places into k and v; zeros where
 * a place holds no token.  sites (may be NULL) gets the places' sites.  Rows of k and
 * v do not overlap each other, nor the cache. */
typedef struct pd_cache_args {
  pd_cache cache;
  int32_t tokens;
  int32_t dtype;     /* of k and v: PD_DTYPE_BF16 or PD_DTYPE_FP32 */
  const int64_t* at; /* [batch] */
  void* k;
  int64_t k_batch_stride, k_token_stride, k_head_stride;
  void* v;
  int64_t v_batch_stride, v_token_stride, v_head_stride;
  pd_site* sites; /* [batch][tokens], 16-byte aligned */
  int64_t sites_batch_stride; /* in sites; write: 0: one list for all */
} pd_cache_args;

pd_status predecoder_cache_write(void* hip_stream, const pd_cache_args* args);
pd_status predecoder_cache_read(void* hip_stream, const pd_cache_args* args);

/* ---- Attention over a cache in 8 bits ----
 *
 * What predecoder_attention computes (there: scores, cap, slopes, masks, prefix,
 * queries that see nothing), of q over the tokens of a cache: keys and values are
 * code scale, not rounded in between.  Scores, maximum and sum are fp32; a
 * probability times a value's scale is kept to 16 bits (2^-16) for the product with the
 * values' codes.  A visible row with scale NaN makes the result NaN; what invisible places
 * hold does not reach it (but E4M3's NaN codes, which predecoder_cache_write never writes,
 * may stand only where there is no token).
 * q and out as there: bf16, all rows 16-byte aligned; heads a multiple of
 * cache.kv_heads, heads / kv_heads <= 64; |coordinate| < 2^29.  q_sites is needed unless n_q
 * is 0.  workspace as there.  A cap is met within 2^-20 of the score or of the cap.
 * PD_ERR_UNSUPPORTED where rows (n_q heads / kv_heads) reach 2^30 or the launch 2^32 threads (512 for
 * each 16 rows of a key head up to 64 rows, 256 for each 128 above, times the splits). */
typedef struct pd_attention8_args {
  pd_cache cache;
  int32_t heads, n_q;
  float scale, cap;
  int32_t causal, prefix; /* causal 0 or 1; prefix >= 0, or PD_PREFIX_NONE */
  const void* q;
  int64_t q_batch_stride, q_token_stride, q_head_stride;
  void* out;
  int64_t out_batch_stride, out_token_stride, out_head_stride;
  const pd_site* q_sites; /* [batch][n_q], 16-byte aligned */
  int64_t q_sites_batch_stride; /* in sites; 0: one list for all */
  const float* slopes; /* [heads] or NULL */
  void* workspace;
  size_t workspace_bytes;
} pd_attention8_args;

/* Bytes of workspace that a call with these arguments uses; 0 for invalid ones.
 * It goes by the sizes alone. */
size_t predecoder_attention8_workspace(const pd_attention8_args* args);

pd_status predecoder_attention8(void* hip_stream, const pd_attention8_args* args);

/* ---- Linear attention with a decay ----
 *
 * The tokens of an entry come in rounds of per_round, token n in round
 * t(n) = floor(n / per_round).  For each key head, with S_(-1) = state (NULL: zeros):
 *   S_t = exp(-slope) S_(t-1) + sum over the tokens m of round t of k_m v_m^T
 *   out_n = scale q_n S_t(n)       for every query head of the key head's group
 * that is  scale sum over t(m) <= t(n) of exp(-slope (t(n) - t(m))) (q_n.k_m) v_m
 * plus what the state brings: a token sees its whole round, as in causal attention.
 * state_out (NULL: not asked for) gets S of the entry's last round; it may be
 * state itself, or does not overlap it.  [batch][kv_heads][head_dim][head_dim]
 * fp32, the key's channel first, whole.
 * lengths [batch] (NULL: n for all): tokens of each entry, taken within 0 and n.  Rows of
 * out behind them stay as they are, and what q, k and v hold there is not read; an
 * entry of length 0 passes its state on.  A last round that is not whole counts
 * as a round.
 * slopes [kv_heads] (NULL: 0): the decay of a round; infinite: only its own round.
 * A value of q, k, v or the state that is not finite makes the results that take it in
 * infinite or NaN, all rounds' from its own on; those before it are as without it.
 * bf16 q, k, v and out; sums and states fp32 (products of bf16 parts that hold 24
 * bits of what is decayed), the weights of pairs inside a chunk and the state's part
 * of a result taken to 16 bits or more, out rounded once.
 * head_dim: a multiple of 8, at most 128; all rows 16-byte aligned; heads a multiple of
 * kv_heads, heads / kv_heads <= 64; n heads / kv_heads < 2^30; batch kv_heads < 2^24, and
 * about 2^23 for more than 64 channels and n != 1.  out overlaps no input, its rows not
 * each other.  workspace as for attention. */
typedef struct pd_linear_attention_args {
  int32_t batch, heads, kv_heads, head_dim;
  int32_t n, per_round; /* per_round >= 1 */
  float scale;
  const void* q;
  int64_t q_batch_stride, q_token_stride, q_head_stride;
  const void* k;
  int64_t k_batch_stride, k_token_stride, k_head_stride;
  const void* v;
  int64_t v_batch_stride, v_token_stride, v_head_stride;
  void* out;
  int64_t out_batch_stride, out_token_stride, out_head_stride;
  const float* slopes;
  const int32_t* lengths;
  const float* state;
  float* state_out;
  void* workspace;
  size_t workspace_bytes;
} pd_linear_attention_args;

/* Bytes of workspace, by the sizes alone; 0 for invalid arguments. */
size_t predecoder_linear_attention_workspace(const pd_linear_attention_args* args);

pd_status predecoder_linear_attention(void* hip_stream, const pd_linear_attention_args* args);

#ifdef __cplusplus
}
#endif

#endif /* PREDECODER_OPS_H */
