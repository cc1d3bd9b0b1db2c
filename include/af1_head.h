/*
 * af1_head.h -- C ABI of the output head and its losses on AMD MI355X
 * (gfx950), built as libaf1_head.so.
 *
 * The linears of a decoder are factorized (af1.h); what follows them is not.
 * This library holds that part: a linear whose weight is kept in 8-bit
 * floating point with a scale for each block of 128 x 128 (the output head,
 * and any linear that is left unfactorized), and what is read off its logits:
 * the log probabilities of given tokens with the entropy and the best
 * alternatives, and the KL divergence to a full-precision teacher that the
 * scale-only reconstruction minimises (Sec. 4.1, label eq:scale_only_kl),
 * with the gradients that af1_linear_backward starts from.
 *
 * Conventions (beyond those of af1.h)
 * -----------------------------------
 * Shapes: dimensions need not be multiples of 32.  A call of zero tokens or
 *   rows is valid and enqueues nothing.
 * Pointers: logits, tokens, log probabilities and what else belongs to tokens
 *   may be slices of larger arrays and need their element's alignment only;
 *   every other array, the linear's x and y among them, 16 bytes, as in af1.h.
 * Types: dense arrays are fp32, bfloat16 or binary16 (af1_src_dtype, without
 *   AF1_SRC_I8), row-major.
 * Results repeat bit for bit: every sum is taken in a fixed order.
 * Workspaces need no initialisation and carry nothing from call to call;
 *   calls that may overlap in time need distinct ones.
 * Errors: as in af1.h, in the order NULL, DTYPE, SHAPE, BATCH, then the
 *   arrays' NULL, ALIGN, WORKSPACE, ALIAS.
 */
#ifndef AF1_HEAD_H
#define AF1_HEAD_H

#include "af1.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AF1_HEAD_MAX_TOKENS (1 << 20)
#define AF1_HEAD_MAX_VOCAB (1 << 24)
#define AF1_HEAD_MAX_TOP 32

/* 8-bit formats (OCP): e4m3 has no infinity and reaches 448, e5m2 57344. */
typedef enum af1_fp8_format {
    AF1_FP8_E4M3 = 0,
    AF1_FP8_E5M2 = 1
} af1_fp8_format;

/*
 * A rows x cols matrix in 8 bits.  Blocks of 128 x 128 entries share a scale
 * 2^e, e the smallest integer with amax <= MAX * 2^e (amax over the block's
 * finite entries, MAX the format's largest value; e = 0 for amax = 0, and at
 * least -127).  An entry x is kept as the code of x * 2^-e, rounded to nearest
 * even.  Powers of two scale without rounding, and the matrix cores apply them
 * inside the product.
 *   codes  : ceil(rows/128) x ceil(cols/128) tiles, row-major, of 128 x 128
 *            codes, row-major (16 KiB a tile); zero outside the matrix.
 *   scales : one byte e + 127 a tile, in the same order.
 * NaN and infinite entries become NaN (e5m2 keeps infinities).
 * rows, cols in 1 .. AF1_MAX_DIM.
 */
typedef struct af1_fp8_matrix {
    int64_t rows;
    int64_t cols;
    int32_t format;     /* af1_fp8_format */
    int32_t reserved;   /* set to 0 */
    const uint8_t *codes;
    const uint8_t *scales;
} af1_fp8_matrix;

/* Bytes of the codes and of the scales; 0 for dimensions out of range. */
AF1_API size_t af1_fp8_code_bytes(int64_t rows, int64_t cols);
AF1_API size_t af1_fp8_scale_bytes(int64_t rows, int64_t cols);

/*
 * af1_fp8_quantize -- codes and scales of a dense matrix.
 *   src    : device, rows x cols of src_dtype, contiguous.
 *   codes, scales : device, written (af1_fp8_code_bytes, af1_fp8_scale_bytes).
 * Bit-exact and deterministic.
 */
AF1_API af1_status af1_fp8_quantize(const void *src, int32_t src_dtype, int64_t rows,
                                    int64_t cols, int32_t format, uint8_t *codes,
                                    uint8_t *scales, void *stream);

/*
 * af1_fp8_dequantize -- the values that a matrix stands for, rows x cols of
 * dst_dtype, contiguous.  Exact in fp32, and in bfloat16 wherever the value is
 * not below its normal range; binary16 rounds (nearest even).  Codes of entries
 * that rounded up to 2^128 are infinite.
 */
AF1_API af1_status af1_fp8_dequantize(const af1_fp8_matrix *W, void *dst, int32_t dst_dtype,
                                      void *stream);

/*
 * af1_fp8_transpose -- the transposed matrix (cols x rows), which the gradient
 * of a linear's input reads: blocks are square, so codes and scales are moved
 * and nothing is rounded.  codes, scales: written, sized for (cols, rows).
 */
AF1_API af1_status af1_fp8_transpose(const af1_fp8_matrix *W, uint8_t *codes, uint8_t *scales,
                                     void *stream);

/*
 * af1_fp8_linear -- y = q(x) W^T for T tokens, W of m = rows by n = cols.
 *   x : device, [T, n] of x_dtype, contiguous.  Each token's pieces of 128
 *       columns are rounded to x_format at a power-of-two scale of their own
 *       (the rule of af1_fp8_matrix).  Use e5m2, with its wider range, for
 *       gradients.
 *   y : device, [T, m] of y_dtype (AF1_SRC_F32, AF1_SRC_BF16), written.
 *   T : 0 .. AF1_HEAD_MAX_TOKENS.
 *   ws: device, at least af1_fp8_linear_workspace_bytes(m, n, T) bytes.  Fewer
 *       tokens may need more (they are split over more ranges of columns): one
 *       workspace for calls of several T has the largest of their sizes.
 * Sums: with y in fp32, and for T <= 16 with y in either type, products are
 * exact and accumulated in fp32 on the matrix cores.  With y in bfloat16 and
 * more tokens the 8-bit matrix instructions may sum them, which add the eight
 * products of columns 8 i .. 8 i + 7 first and cut each, toward zero, below
 * 2^-13 of the largest of the eight; these sums are accumulated in fp32.  Beside
 * the roundings of x and y that is little (about 2^-14 of the norm of y), but
 * where products of one eight cancel what is left may be lost: ask for fp32 then,
 * at up to twice the time.
 * The input gradient dx = dy W is the same call with the transposed matrix.  y
 * must not overlap x, W or ws.
 */
AF1_API size_t af1_fp8_linear_workspace_bytes(int64_t m, int64_t n, int64_t T);
AF1_API af1_status af1_fp8_linear(const af1_fp8_matrix *W, const void *x, int32_t x_dtype,
                                  int32_t x_format, int64_t T, void *y, int32_t y_dtype,
                                  void *ws, size_t ws_bytes, void *stream);

/*
 * af1_token_logprobs -- for the logits of T tokens over a vocabulary of V,
 * with z = scale * logits (scale is an inverse temperature) and
 * lse = log sum_j exp z_j:
 *     logprob = z_target - lse          entropy = lse - sum_j p_j z_j
 *     the k largest z_j - lse with their indices, equal logits in the order of
 *     their indices, NaN before everything.
 *   logits  : device, T rows of V, `ld` elements apart (ld >= V).
 *   targets : device, int64[T], or NULL (then logprob is not written).  A
 *             negative target is no token: its logprob is 0.  One of V or more
 *             gives NaN.
 *   logprob, entropy, lse : device, fp32[T], written; each may be NULL.
 *   k       : 0 .. AF1_HEAD_MAX_TOP.  top_logprob: fp32[T, k]; top_index:
 *             int64[T, k]; places beyond V hold -infinity and -1.
 *   saved   : device, fp32[T, 4] (16-byte aligned), written for the backward;
 *             may be NULL.
 *   ws      : device, af1_token_logprobs_workspace_bytes(T, V, k) bytes.
 * Masked logits (-infinity) have probability 0 and add nothing.  A row whose
 * logits are all -infinity has lse and log probabilities of -infinity and
 * entropy 0.  A row with NaN or +infinity has NaN results (its indices are
 * still ordered).  scale: positive, at most 2.3e38 (AF1_ERR_SHAPE).
 * One pass over the logits; sums in fp32, about the largest logit.
 */
AF1_API size_t af1_token_logprobs_workspace_bytes(int64_t T, int64_t V, int32_t k);
AF1_API af1_status af1_token_logprobs(const void *logits, int32_t dtype, int64_t T, int64_t V,
                                      int64_t ld, float scale, const int64_t *targets,
                                      float *logprob, float *entropy, float *lse, int32_t k,
                                      float *top_logprob, int64_t *top_index, float *saved,
                                      void *ws, size_t ws_bytes, void *stream);

/*
 * af1_token_logprobs_backward -- the gradient of
 *     sum_t g_logprob[t] logprob[t] + g_entropy[t] entropy[t]:
 *     dlogits_j = scale (g_logprob ([j = target] - p_j)
 *                        - g_entropy p_j (log p_j + entropy))
 *   logits .. scale, targets : as in the forward.  saved: what it wrote.
 *   g_logprob, g_entropy : device, fp32[T]; either may be NULL (zeros).
 *             targets may be NULL if g_logprob is.
 *   dlogits : device, T rows of V of the logits' type, `ldd` elements apart,
 *             written; elements between rows are left as they were.  It may be
 *             the logits' own array where ldd = ld, and must not overlap any
 *             array otherwise.
 * A token whose two factors are zero, or whose logits are all -infinity, gets
 * zeros whatever its logits hold.  A negative target takes no part in
 * g_logprob; one of V or more gives NaN in the whole row unless its g_logprob is
 * zero (or NULL), and so does a factor that is NaN.
 */
AF1_API af1_status af1_token_logprobs_backward(const void *logits, int32_t dtype, int64_t T,
                                               int64_t V, int64_t ld, float scale,
                                               const int64_t *targets, const float *saved,
                                               const float *g_logprob, const float *g_entropy,
                                               void *dlogits, int64_t ldd, void *stream);

/*
 * af1_distill_kl -- the loss of the scale-only reconstruction (Sec. 4.1, label
 * eq:scale_only_kl) and its gradient.  With p the teacher's and q the
 * student's softmax of scale * logits:
 *     kl[t] = sum_j p_j (log p_j - log q_j)
 *     dstudent_j = weight[t] scale (q_j - p_j)
 * the gradient of sum_t weight[t] kl[t].
 *   student, teacher : device, T rows of V of `dtype`, ld_s and ld_t apart.
 *   weight   : device, fp32[T], or NULL for ones (a mean over tokens is 1/T,
 *              padding 0).
 *   kl       : device, fp32[T], written; it does not depend on weight, and a
 *              padding token's may be NaN or infinite (leave it out of a sum).
 *   dstudent : device, T rows of V of dtype, ldd apart, written; NULL for the
 *              loss alone.  It may be the student's own array where ldd = ld_s,
 *              and must not overlap any array otherwise.
 *   ws       : device, af1_distill_kl_workspace_bytes(T, V) bytes.
 * kl is summed from the differences of the two logits, not of two logarithms,
 * so a small divergence errs by some 1e-8, not by 1e-6; none is below 0.
 * Entries whose p_j is 0 in fp32 add nothing.  Where the student masks
 * (-infinity) an entry of the teacher's, kl is infinite.  A token whose teacher
 * masks everything has kl 0; its gradient is zero, and so are those of tokens
 * of weight 0 and of tokens whose student masks everything.  NaN or +infinity
 * in a row gives NaN.
 */
AF1_API size_t af1_distill_kl_workspace_bytes(int64_t T, int64_t V);
AF1_API af1_status af1_distill_kl(const void *student, const void *teacher, int32_t dtype,
                                  int64_t T, int64_t V, int64_t ld_s, int64_t ld_t, float scale,
                                  const float *weight, float *kl, void *dstudent, int64_t ldd,
                                  void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* AF1_HEAD_H */
