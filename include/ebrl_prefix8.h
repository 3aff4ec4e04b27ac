/*
 * ebrl_prefix8 -- prefix caches held in 8 bits, and the operators that work on them.
 *
 * Action generation reads every environment's prefix keys and values once per layer and Euler step
 * (ebrl_actgen.h): they are the largest thing in memory and their stream bounds cross-attention.  Here a
 * prefix is kept as e4m3 codes with one fp32 scale for each block of 32 tokens and head: half the bytes of
 * the bf16 planes, a quarter of the fp32 ones.  Four operators write, read, weigh and shorten such caches;
 * a handle created with kv_dtype = EBRL_E4M3 takes records in place of planes.
 *
 * The record of one environment (capacity C tokens, rows = C rounded up to a multiple of 32):
 *
 *     codes   e4m3   [kv_layers][2][n_kv_heads][rows][head_dim]     plane 0 = K, plane 1 = V
 *     scales  fp32   [kv_layers][2][n_kv_heads][rows / 32]
 *     mask    uint32 [rows / 32]                                    bit t % 32 of word t / 32: queries see token t
 *
 * one behind the other, padded to a multiple of 128 bytes (ebrl_prefix8_record_bytes).  A token's key or
 * value is code * |scale| of its block.  A block that holds a NaN has its scale's sign bit set (quantize and evict
 * do that): a query that sees a token of such a block gets NaN.  Without the sign, codes must not be NaN.  A pool is n_slots records in a row, 128-byte aligned; the operators
 * take it with the slots of a call (host array, NULL: environment i uses slot i) and the prefix lengths
 * (host array).  Rows behind an environment's length are neither read nor written, except that the scale and
 * the mask word of its last, partial block belong to it as a whole.
 *
 * Every operator is asynchronous on `stream` and touches no memory but its arguments; the current device must be
 * the one that holds them.  Host arrays are copied before the call returns.  All arguments are checked before anything is enqueued; a
 * status other than EBRL_OK comes with a text (ebrl_prefix8_last_error).  Calls that may be captured into a
 * CUDA graph: all four (lengths, slots and pointers are then those of the capture).  sm_quota as in
 * ebrl_actgen_submit: 0 = all SMs, else persistent grids of at most that many CTAs.
 */
#ifndef EBRL_PREFIX8_H_
#define EBRL_PREFIX8_H_

#include "ebrl_actgen.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EBRL_PREFIX8_BLOCK 32

typedef struct {
    int32_t kv_layers;    /* >= 1                                                                      */
    int32_t n_kv_heads;   /* >= 1                                                                      */
    int32_t head_dim;     /* 32, 64 or 128                                                             */
    int32_t capacity;     /* tokens a record can hold, 1 .. 2^24                                       */
} ebrl_prefix8_layout_t;

/* Bytes of one record; 0 for a layout that is not covered. */
uint64_t ebrl_prefix8_record_bytes(const ebrl_prefix8_layout_t *layout);

/* Text of the last error of this thread's ebrl_prefix8 calls; valid until its next one. */
const char *ebrl_prefix8_last_error(void);

/* Writes environments' planes into their records.
 *   planes      host [n] of DEVICE pointers; env i: element (layer l, plane p, token t, column c) at
 *               planes[i][((l * 2 + p) * plane_rows[i] + t) * row_stride + c], c = head * head_dim + j;
 *               16-byte aligned, in src_dtype (EBRL_F32 or EBRL_BF16)
 *   len         host [n], 0 .. capacity
 *   plane_rows  host [n], NULL: len (planes as ebrl_actgen_submit takes them)
 *   row_stride  elements, >= n_kv_heads * head_dim and a multiple of 16 bytes; 0: n_kv_heads * head_dim
 *   mask        NULL, or host [n] of DEVICE pointers (each may be NULL: all visible) to len[i] bytes: 0 hides a token
 * For each block and head: s = the power of two with max |x| / s in (224, 448] over the block's visible finite
 * values (1 when they are all zero, never below 2^-126); code = e4m3(x / s), to nearest even, saturated (so Inf
 * becomes the largest value; NaN stays NaN and puts a minus before the scale).  A hidden token gets zero codes whatever its planes hold.
 * Slots of one call must differ. */
ebrl_status_t ebrl_prefix8_quantize(const ebrl_prefix8_layout_t *layout, void *pool, int32_t n_slots, int32_t n,
                                    const int32_t *slots, const void *const *planes, const int32_t *len,
                                    const int32_t *plane_rows, int64_t row_stride, int32_t src_dtype,
                                    const uint8_t *const *mask, int32_t sm_quota, void *stream);

/* Softmax attention of each environment's queries over its record's visible tokens, of one layer:
 *     out = softmax(scale * q k^T) v,   lse = log sum_t exp(scale * q k_t)
 *   q      DEVICE, q_dtype (EBRL_F32 or EBRL_BF16): env i, token h, head a at q + i * q_env_stride + h * q_token_stride
 *          + a * head_dim (strides in elements, addresses multiples of 16 bytes; the stride of a single environment
 *          or token is not looked at).  Head a reads
 *          key/value head a / (n_heads / n_kv_heads).
 *   H      query tokens per environment, 1 .. 1024
 *   out    DEVICE, q_dtype, laid out like q with its own strides; may be q itself
 *   lse    DEVICE fp32 [n][H][n_heads], or NULL
 *   scale  softmax scale, finite (usually 1 / sqrt(head_dim))
 * A row that sees no token gives out = 0 and lse = -inf.  Two environments of a call may share a slot.
 * With few environments a prefix is divided among warps, which are joined in shared memory, and a long one is cut into pieces
 * besides, which are joined by a second kernel.
 * split_tokens = 0 lets the call choose (the choice depends on the whole call, so an environment's last bits can
 * depend on its company); -1 never divides or cuts (an environment's result then depends on nothing but itself); a positive
 * multiple of 128 cuts every prefix into pieces of that many tokens.  The pieces' partial results need
 * ebrl_prefix8_attend_workspace bytes (of the same arguments) of DEVICE memory, 16-byte aligned, that no other call in flight uses;
 * 0 bytes: workspace may be NULL.
 * Products are taken on f16 tensor-core operands that hold the codes exactly and q exactly (bf16) or in two
 * terms (fp32); weights are rounded to f16 (bf16 q) or held in two terms; all sums and softmax statistics are fp32. */
uint64_t ebrl_prefix8_attend_workspace(const ebrl_prefix8_layout_t *layout, int32_t n, const int32_t *len, int32_t H,
                                       int32_t n_heads, int32_t split_tokens, int32_t sm_quota);
ebrl_status_t ebrl_prefix8_attend(const ebrl_prefix8_layout_t *layout, const void *pool, int32_t n_slots, int32_t n,
                                  const int32_t *slots, const int32_t *len, int32_t layer, const void *q, int32_t q_dtype,
                                  int32_t H, int32_t n_heads, int64_t q_env_stride, int64_t q_token_stride, void *out,
                                  int64_t o_env_stride, int64_t o_token_stride, float *lse, float scale, int32_t split_tokens,
                                  void *workspace, uint64_t workspace_bytes, int32_t sm_quota, void *stream);

/* The weight each token got: weight[slot][t] (+)= sum over the environment's H * n_heads rows of exp(scale * q k_t - lse),
 * for t < len; hidden tokens get 0.  q as in attend; lse as its output for the same queries (rows with lse = -inf add
 * nothing), of env i, token h, head a at lse + i * lse_env_stride + h * lse_token_stride + a * lse_head_stride.
 *   weight      DEVICE fp32, row of a SLOT at weight + slot * weight_stride, weight_stride >= capacity
 *   accumulate  0: written, else added to what is there
 * Without rows (H or n_heads is 0; q and lse may be NULL) the sum is 0.  It is taken in a fixed order.  Slots of one call must differ. */
ebrl_status_t ebrl_prefix8_weigh(const ebrl_prefix8_layout_t *layout, const void *pool, int32_t n_slots, int32_t n,
                                 const int32_t *slots, const int32_t *len, int32_t layer, const void *q, int32_t q_dtype, int32_t H,
                                 int32_t n_heads, int64_t q_env_stride, int64_t q_token_stride, const float *lse, int64_t lse_env_stride,
                                 int64_t lse_token_stride, int64_t lse_head_stride, float scale, float *weight, int64_t weight_stride,
                                 int32_t accumulate, int32_t sm_quota, void *stream);

/* Shortens records to their heaviest tokens: new length = min(len[i], keep[i]), known to the host.  Which tokens stay goes
 * by (protected, weight, index): the first protect_first and the last protect_last tokens of the prefix as if their weight were
 * +inf, hidden tokens and NaN weights as if it were -inf, ties to the lower index.  Kept tokens keep their order; hidden ones
 * that stay remain hidden.  A block's codes are taken to its new scale (the rule of quantize on code * scale), which
 * loses nothing but what falls below the new block's smallest code when scales are powers of two.  (The largest scale written is
 * 2^127: a caller's own scales beyond it make values that no e4m3 block holds, and those are saturated.)
 *   dst          pool of the same layout and slot numbers: src itself (in place), or memory that does not overlap it
 *   weight       DEVICE fp32, by slot, as in weigh
 *   weight_out   NULL, or like weight: the kept tokens' weights; may be weight itself, or share no memory with it (rows of one stride may alternate)
 *   kept         DEVICE int32, env i of the CALL at kept + i * kept_stride: the kept tokens' old indices, ascending;
 *                kept_stride >= the largest new length.  Entries and rows behind the new length are left as they were.
 * Slots of one call must differ. */
ebrl_status_t ebrl_prefix8_evict(const ebrl_prefix8_layout_t *layout, const void *src, void *dst, int32_t n_slots, int32_t n,
                                 const int32_t *slots, const int32_t *len, const int32_t *keep, int32_t protect_first,
                                 int32_t protect_last, const float *weight, int64_t weight_stride, float *weight_out,
                                 int64_t weight_out_stride, int32_t *kept, int64_t kept_stride, int32_t sm_quota, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* EBRL_PREFIX8_H_ */
