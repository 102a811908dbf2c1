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

/* Reads and clears (with a synchronisation of the current device) the status word that a kernel of this
 * header sets when a bounded wait ran out: DIT_OK or DIT_ERR_TIMEOUT. */
dit_status dit_ops_poll_status(void);

#ifdef __cplusplus
}
#endif
#endif /* DIT_OPS_H_ */
