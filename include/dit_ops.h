/*
 * Operators of libdit that need no context: the block-scaled e4m3 product with the quantisers of its
 * operands, and attention over selected key blocks with the selector of its lists.  They are the two
 * heavy parts of a DiT block in reduced arithmetic: the step runs them for contexts created with
 * DIT_FLAG_FP8_BLOCK128 or DIT_FLAG_SPARSE_ATTENTION (dit.h), and a caller with a model of its own can
 * call them directly.
 *
 * Conventions: those of dit.h (C ABI, dit_status, device pointers of the current device, `stream` a
 * cudaStream_t), and
 *   - every call is asynchronous on `stream`, allocates nothing, keeps nothing from one call to the next
 *     and may be captured into a CUDA graph (the first call on a device sets kernel attributes: make it
 *     outside a capture).  Argument errors are found on the host before any launch.
 *   - rows, columns and leading dimensions are in elements unless stated otherwise; a leading dimension
 *     is the distance between the starts of two rows.  Element offsets may exceed 32 bits.
 *   - outputs are written exactly where they are defined: padding columns between a row's last element
 *     and the next row, and rows behind the last one, stay as they were.
 *   - results do not depend on timing: every sum is taken in an order fixed by the shapes of the call, without
 *     atomics.  Quantised values and selected lists depend on their own group or request alone.  The order of a product's sum over the
 *     groups depends on m, n and k, and that of attention for a request of up to 16 query rows on the whole batch, whose longest
 *     request chooses the kernel: such results may differ in their last bits with the rows they are packed with.
 *   - kernels bound their waits; one that gave up leaves its output undefined and sets a status word of
 *     the device, which dit_ops_poll_status reads.
 */
#ifndef DIT_OPS_H_
#define DIT_OPS_H_

#include "dit.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { DIT_TYPE_F16 = 0, DIT_TYPE_BF16 = 1, DIT_TYPE_F32 = 2 } dit_type;

#define DIT_BLOCK 128 /* columns per scale; rows per query block and per key block */

/* Quantises a matrix x [rows, cols] row by row in groups of 128 columns (the last group may be short):
 *   top[m, g]    = max(largest |x| of the group, 2^-100)
 *   scale[g, m]  = top / 448                               (fp32, round to nearest)
 *   code[m, c]   = e4m3 nearest to x[m, c] * (448 / top)   (ties to even, |code| <= 448)
 * so that x ~ code * scale.  The scales lie group-major: scales[g * ld_scales + m], g < ceil(cols / 128).
 * A group that holds a NaN gets a NaN scale and NaN codes; one that holds an infinity an infinite scale,
 * so that its products are NaN.
 *   x       device, type f16, bf16 or f32, element-aligned, ld >= cols
 *   codes   device bytes, 16-byte aligned, ld_codes >= cols and a multiple of 16 (what dit_gemm_block128
 *           wants of its operands)
 *   scales  device fp32, ld_scales >= rows
 * rows == 0 is a no-op.  DIT_ERR_INVALID_ARG for NULL pointers, bad types, leading dimensions or
 * alignment; DIT_ERR_SHAPE for cols < 1 or rows or cols above 2^31 - 1024. */
dit_status dit_quantize_block128(const void *x, dit_type type, int64_t ld, int64_t rows, int64_t cols, void *codes,
                                 int64_t ld_codes, float *scales, int64_t ld_scales, void *stream);

/* The same for a weight w [in, out] (y = x w, as everywhere in this library): one scale for each block of
 * 128 x 128 elements, the codes transposed:
 *   codes [out, ld_codes], ld_codes >= in and a multiple of 16;  scales [ceil(out / 128), ceil(in / 128)] */
dit_status dit_quantize_weight_block128(const void *w, dit_type type, int64_t ld, int64_t in_dim, int64_t out_dim,
                                        void *codes, int64_t ld_codes, float *scales, void *stream);

/* Product of two quantised operands, both with k contiguous in a row:
 *   out[m, n] = sum_g a_scales[g, m] * b_scales[n / 128, g] * (sum over the group's k of a[m, k] b[n, k]) + bias[n]
 * Each group's inner sum is a tensor-core sum of exact products in fp32; the two scales are multiplied first, in fp32 as well (so
 * their product has to lie inside fp32's normal range: below it bits are lost, above it a sum of zero gives NaN); the scaled sum over
 * the groups is held in fp32 and rounded once into out.  16-bit outputs clamp to the largest finite value.
 *   a        device e4m3 codes [m, lda], 16-byte aligned, lda >= k and a multiple of 16; columns k.. are not used
 *   a_scales device fp32 [ceil(k / 128), ld_a_scales], ld_a_scales >= m   (dit_quantize_block128)
 *   b        device e4m3 codes [n, ldb], likewise;  b_scales device fp32 [ceil(n / 128), ceil(k / 128)]
 *   bias     device fp32 [n] or NULL
 *   out      device [m, ld_out] of out_type, element-aligned, ld_out >= n; must not overlap the operands
 * m == 0 is a no-op; DIT_ERR_SHAPE for n or k < 1 or a size above 2^31 - 1024. */
typedef struct {
  const void *a;
  const float *a_scales;
  const void *b;
  const float *b_scales;
  const float *bias;
  void *out;
  int64_t lda, ld_a_scales, ldb, ld_out;
  int64_t m, n, k;
  dit_type out_type;
} dit_gemm_block128_args;
dit_status dit_gemm_block128(const dit_gemm_block128_args *args, void *stream);

/* A batch of attention problems over packed rows, as the step packs its requests: request r owns q_lens[r] rows of q
 * (and of the output) and kv_lens[r] rows of k and v, one request after the other.  Head h is columns
 * h * head_dim .. of each.  The lengths are HOST arrays, read before the call returns; they differ for a few new rows that
 * read a longer stored context, and are equal in a denoising step.  A request may have no rows of q, or none of k.
 *   Query block i of a request is its rows 128 i .. 128 i + 127, key block j likewise (the last one may be short);
 *   blocks are counted from each request's own first row.  Query blocks are numbered through the batch,
 *   request after request: n_query_blocks = sum of ceil(q_lens[r] / 128).
 *   q, k, v   device, type f16 or bf16, 16-byte aligned, leading dimensions multiples of 8 and >= n_heads * head_dim
 *             (three column ranges of one packed [rows, 3 * width] buffer are fine)
 *   head_dim  64 or 128; n_requests <= DIT_MAX_REQUESTS; at most 16384 key blocks in a request (DIT_ERR_SHAPE beyond) */
typedef struct {
  const void *q, *k, *v;
  int64_t ld_q, ld_k, ld_v;
  dit_type type;
  int32_t n_heads, head_dim, n_requests;
  const int32_t *q_lens, *kv_lens;
} dit_attention_batch;

/* Selects key blocks by a cheap score: the product of the mean of the query block's rows with the mean of the key
 * block's rows, taken in 64-bit arithmetic.  Each query block of each head keeps the
 * min(keep[r], key blocks of its request) key blocks with the largest scores; of equal scores the lower block
 * wins; a NaN counts as less than any number.  Key blocks that hold one of the request's last tail_rows[r] rows (its text
 * tokens) come before every score; where there are more of them than keep[r], the lowest of them.  v is not read.
 *   keep, tail_rows  HOST [n_requests], keep >= 1 (beyond a request's key blocks: all of them), tail_rows >= 0 or NULL (no tail)
 *   block_index      device int32 [n_heads, n_query_blocks, ld_index], ld_index >= the largest keep: the selected key
 *                    blocks in ascending order, then -1 up to the largest keep of the batch
 *   block_count      device int32 [n_heads, n_query_blocks]
 *   workspace        device, 16-byte aligned, dit_select_blocks_workspace(batch) bytes; its contents need not be
 *                    kept between calls, and calls that may run at the same time need workspaces of their own
 * DIT_ERR_SHAPE for lengths whose sum leaves int32, head_dim other than 64 or 128, or more than 16384 key blocks in a
 * request; DIT_ERR_CAPACITY for too many requests or too small a workspace. */
size_t dit_select_blocks_workspace(const dit_attention_batch *batch);
dit_status dit_select_blocks(const dit_attention_batch *batch, const int32_t *keep, const int32_t *tail_rows,
                             int32_t *block_index, int32_t *block_count, int64_t ld_index, void *workspace,
                             size_t workspace_bytes, void *stream);

/* Softmax attention of every query row over the keys of its query block's listed key blocks:
 *   out[i] = sum_j softmax_j(scale * q_i . k_j) v_j,   j over the rows of the listed blocks of row i's request
 * The lists are those of dit_select_blocks or the caller's own: the first block_count entries of each list count, clamped
 * to [0, ld_index]; their order does not matter, an entry listed twice counts once, and entries outside the
 * request's key blocks are ignored.  A row without any key gets zeros.  Rows of other requests are never
 * part of a result, whatever they hold.  Scores, their differences, the softmax and the sums are held in fp32, so scaled scores may
 * be of any size as long as q_i . k_j itself and the difference of two of them stay inside fp32; probabilities are rounded
 * to the inputs' type for the second product, as the step's attention does.  An infinite value makes its channel of the rows that
 * list it infinite, or NaN where its probability rounds to zero or the other infinity is listed as well; finite values above 2^98 may
 * do the same by the sums, which are taken before the division.  Finite results clamp to the type's largest value.  A row all of whose
 * scores are -infinity gets zeros.
 *   scale   0 for 1 / sqrt(head_dim); at most 2e38
 *   out     device, the inputs' type, rows as q's, 16-byte aligned, ld_out a multiple of 8 and >= n_heads * head_dim;
 *           must not overlap the inputs */
dit_status dit_block_attention(const dit_attention_batch *batch, const int32_t *block_index, const int32_t *block_count,
                               int64_t ld_index, float scale, void *out, int64_t ld_out, void *stream);

/* ------------------------------------------------------------------------------------------------------------
 * Microscaled 4-bit floating point.  A matrix [rows, cols] is held as e2m1 codes (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives) with one
 * scale for each `group` of 16 or 32 consecutive columns of a row (the last group may be short):
 *   group 32   scale = 2^e, e the smallest integer with top <= 6 * 2^e, top = max(max |x| of the group, 2^-100)
 *              code = e2m1 nearest to x * 2^-e
 *   group 16   scale = s * 2^e, e the smallest integer with row_top <= 6 * 448 * 2^e, row_top = max(max |x| of the row, 2^-100)
 *              s = e4m3 nearest to top * 2^-e / 6, code = e2m1 nearest to (x * 2^-e) / s, 0 where s is 0
 * (quotients rounded to fp32 first; ties to even; codes beyond 6 clamp).
 *   codes       device bytes [rows, ld_codes], 16-byte aligned, ld_codes a multiple of 16 and >= (cols + 1) / 2 (bytes): column 2 i in the
 *               low half of byte i, column 2 i + 1 in the high half; where cols is odd the last high half is 0
 *   scales      device bytes, 16-byte aligned, dit_fp4_scale_bytes(rows, cols, group): tiles of 128 rows x 4 groups, 512 bytes each,
 *               [ceil(rows / 128)][ceil(cols / (4 * group))], in them byte (row % 32) * 16 + (row % 128) / 32 * 4 + group % 4:
 *               the e4m3 number s (group 16; its sign bit is 0) or e + 127 (group 32; 255 is NaN).  The quantisers write whole tiles, zeros
 *               where there is no row or group; scales that a caller makes need finite values for the groups behind a row's last one up to
 *               its tile's end
 *   row_scales  device fp32 [rows]: 2^e (group 16).  NULL (group 32)
 * A row (group 16) or group (group 32) that holds a NaN or an infinity gets codes 0 and a NaN row scale or scale.
 * cols, k and n are at least 1 and at most 2^30, rows and m at most 2^31 - 1024 (DIT_ERR_SHAPE); other groups are DIT_ERR_INVALID_ARG.  Results
 * must not overlap what they are made from. */

/* Bytes of the scales of a [rows, cols] matrix; 0 for sizes or groups that the calls below refuse. */
size_t dit_fp4_scale_bytes(int64_t rows, int64_t cols, int32_t group);

/* x  device [rows, cols], type f16, bf16 or f32, element-aligned, ld >= cols.  rows == 0 is a no-op. */
dit_status dit_quantize_fp4(const void *x, dit_type type, int64_t ld, int64_t rows, int64_t cols, int32_t group, void *codes,
                            int64_t ld_codes, void *scales, float *row_scales, void *stream);

/* The same for a weight w [in, out] (y = x w), transposed: codes [out, ld_codes] with in columns, scales of an [out, in] matrix,
 * row_scales [out]. */
dit_status dit_quantize_weight_fp4(const void *w, dit_type type, int64_t ld, int64_t in_dim, int64_t out_dim, int32_t group, void *codes,
                                   int64_t ld_codes, void *scales, float *row_scales, void *stream);

/* The values code * scale * row_scale (row_scales NULL: 1), the last product rounded to fp32, then to out_type (16-bit outputs
 * clamp to the largest finite value).
 *   out  device [rows, ld_out] of out_type, element-aligned, ld_out >= cols.  rows == 0 is a no-op. */
dit_status dit_dequantize_fp4(const void *codes, int64_t ld_codes, const void *scales, const float *row_scales, int64_t rows, int64_t cols,
                              int32_t group, void *out, dit_type out_type, int64_t ld_out, void *stream);

/* Product of two such operands of the same group, both with k along a row:
 *   out[m, n] = a_rows[m] * b_rows[n] * sum_k (a's code * scale)[m, k] * (b's code * scale)[n, k] + bias[n]
 * The sum is the tensor cores', in fp32; the row scales (each NULL for 1) and the bias follow in fp32; rounded once into out, 16-bit outputs
 * clamp to the largest finite value.  Sums and products of two groups' scales have to lie inside fp32's range; row scales may have any size, the
 * result leaves the range only where the whole product does.
 *   a, a_scales, a_rows   [m, k] as above, lda in bytes;  b, b_scales, b_rows  [n, k] likewise;  bias  device fp32 [n] or NULL
 *   out  device [m, ld_out] of out_type, element-aligned, ld_out >= n; must not overlap the operands
 * m == 0 is a no-op. */
typedef struct {
  const void *a, *a_scales;
  const float *a_rows;
  const void *b, *b_scales;
  const float *b_rows;
  const float *bias;
  void *out;
  int64_t lda, ldb, ld_out;
  int64_t m, n, k;
  int32_t group;
  dit_type out_type;
} dit_gemm_fp4_args;
dit_status dit_gemm_fp4(const dit_gemm_fp4_args *args, void *stream);

/* Rotary positions.  The first rotary_dim channels of each head are turned in pairs, (a, b) -> magnitude * (a cos t - b sin t,
 * a sin t + b cos t) with t = position * f_i, i < rotary_dim / 2: channels (2 i, 2 i + 1) where `interleaved`, (i, i + rotary_dim / 2)
 * otherwise; the other channels are copied.  inverse: by -t, which takes a rotation of magnitude 1 back and is the transposed map, i.e. the
 * gradient of the rotation.
 *   f_i = base^(-2 i / rotary_dim), for longer contexts than the trained one scaled:
 *     trained_len == 0:  f_i / factor
 *     trained_len > 0:   f_i (g + (1 - g) / factor), g = clamp((trained_len * f_i / (2 pi) - low) / (high - low), 0, 1): pairs that turn
 *                        more than `high` times over the trained context stay, those that turn fewer than `low` times are stretched
 *   x, out      device [rows, n_heads * head_dim], type f16, bf16 or f32, element-aligned, leading dimensions >= n_heads * head_dim.  out
 *               may be x itself (with the same leading dimension) and must not overlap it otherwise.  Adjacent columns of a packed
 *               q | k | v buffer may be turned in one call: n_heads = query heads + key heads
 *   positions   device int32 [rows], any values, or NULL: request r has lens[r] rows at positions first[r], first[r] + 1, ...
 *               (HOST arrays; first NULL: 0, otherwise >= 0; positions end before 2^31)
 * Angles are taken in 64 bits and reduced before they are narrowed: cosine and sine are off by at most 2^-21 up to position 2^24 where base >= 1
 * (no pair turns faster than its position).  Results are rounded once from fp32; infinities and NaN spread within their pair.  rotary_dim even,
 * 2 .. min(head_dim, 256); head_dim <= 4096; base > 0 with finite angles at every position, factor >= 1, high > low where trained_len > 0, all
 * finite.  rows == 0 is a no-op. */
typedef struct {
  const void *x;
  void *out;
  int64_t ld_x, ld_out, rows;
  dit_type type;
  int32_t n_heads, head_dim, rotary_dim, interleaved, inverse;
  double base, factor, trained_len, low, high;
  float magnitude;
  const int32_t *positions;
  int32_t n_requests;
  const int32_t *lens, *first;
} dit_rotary_args;
dit_status dit_rotary(const dit_rotary_args *args, void *stream);

/* Softmax attention of a batch of packed requests with grouped heads: request r owns q_lens[r] rows of q and out and kv_lens[r] rows of k and
 * v, one request after the other; head h is columns h * head_dim .. of q and out and reads key head h / (n_heads / n_kv_heads).
 *   out[i] = sum_j softmax_j(scale * q_i . k_j) v_j
 * over the keys j <= kv_len - q_len + i of row i's request where `causal` (the new rows are the last ones of their context: whole prompts have
 * equal lengths, a single new token has q_len 1), over all keys of the request otherwise.  A row that sees no key gets zeros, and so does
 * one all of whose scores are -infinity.  Keys and values that a row does not see are never part of its result, whatever they hold.
 * Scores, their differences, the softmax and the sums are held in fp32, probabilities are rounded to the inputs' type for the second product (which
 * adds about as much to a result's error as its own rounding to that type does); scores of any size and infinite or NaN values are treated as dit_block_attention treats them.  A request's results do not depend on the
 * values of the others.  Which of two kernels serves a request, and into how many parts long keys are cut, depends on the lengths and heads of the
 * whole batch: results may differ in their last bits with the batch that a request comes in.  The same call gives the same bits.
 *   q, k, v, out  device, type f16 or bf16, 16-byte aligned, leading dimensions multiples of 8 and >= n_heads * head_dim (q, out) or
 *                 n_kv_heads * head_dim (k, v); column ranges of one packed buffer are fine; out must not overlap the inputs
 *   head_dim      64 or 128 (DIT_ERR_SHAPE); n_kv_heads divides n_heads; n_requests <= DIT_MAX_REQUESTS; sums of lengths < 2^31 - 1024
 *   scale         0 for 1 / sqrt(head_dim); at most 2e38
 *   workspace     device, 16-byte aligned, dit_prompt_attention_workspace(args) bytes (sizes only are read; may be 0, then NULL is fine); its
 *                 contents need not be kept between calls, and calls that may run at the same time need workspaces of their own
 * A request may have no rows of q, or none of k. */
typedef struct {
  const void *q, *k, *v;
  void *out;
  int64_t ld_q, ld_k, ld_v, ld_out;
  dit_type type;
  int32_t n_heads, n_kv_heads, head_dim, causal;
  float scale;
  int32_t n_requests;
  const int32_t *q_lens, *kv_lens;
  void *workspace;
  size_t workspace_bytes;
} dit_prompt_attention_args;
size_t dit_prompt_attention_workspace(const dit_prompt_attention_args *args);
dit_status dit_prompt_attention(const dit_prompt_attention_args *args, void *stream);

/* Reads and clears (with a synchronisation of the current device) the status word that a kernel of this
 * header sets when a bounded wait ran out: DIT_OK or DIT_ERR_TIMEOUT. */
dit_status dit_ops_poll_status(void);

#ifdef __cplusplus
}
#endif
#endif /* DIT_OPS_H_ */
