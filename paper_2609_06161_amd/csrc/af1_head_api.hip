// C ABI of the output head and its losses (declared in include/af1_head.h).
// As in af1_api.hip, every argument error is returned before anything is
// enqueued.
#include <math.h>
#include <stdint.h>

#include <atomic>

#include "af1_check.h"
#include "af1_head.h"
#include "af1_head_internal.h"

namespace af1h {

int device_cus() {
  static std::atomic<int> cache[64];
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  cus = cache[dev].load(std::memory_order_relaxed);
  if (cus > 0) return cus;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
      cus <= 0)
    return 256;
  cache[dev].store(cus, std::memory_order_relaxed);
  return cus;
}

}  // namespace af1h

using namespace af1::check;
using af1h::blocks_up;

namespace {

bool head_dim_ok(int64_t d) { return d >= 1 && d <= AF1_MAX_DIM; }
bool dense_ok(int32_t t) { return t == AF1_SRC_F32 || t == AF1_SRC_BF16 || t == AF1_SRC_F16; }
bool format_ok(int32_t f) { return f == AF1_FP8_E4M3 || f == AF1_FP8_E5M2; }
uint64_t dense_size(int32_t t) { return t == AF1_SRC_F32 ? 4 : 2; }

af1_status check_matrix(const af1_fp8_matrix *W) {
  if (!W) return AF1_ERR_NULL;
  if (!format_ok(W->format)) return AF1_ERR_DTYPE;
  if (!head_dim_ok(W->rows) || !head_dim_ok(W->cols)) return AF1_ERR_SHAPE;
  if (!W->codes || !W->scales) return AF1_ERR_NULL;
  return AF1_OK;
}

Span code_span(const void *p, int64_t rows, int64_t cols) {
  return span(p, af1_fp8_code_bytes(rows, cols));
}
Span scale_span(const void *p, int64_t rows, int64_t cols) {
  return span(p, af1_fp8_scale_bytes(rows, cols));
}

// Logits, tokens and the vectors read off them may be slices: their own
// element's alignment is enough.
bool aligned_to(const void *p, uint64_t bytes) {
  return reinterpret_cast<uintptr_t>(p) % bytes == 0;
}
template <typename... P>
bool aligned4(const P *...p) {
  return (aligned_to(p, 4) && ...);
}

// T rows of V elements, ld apart.
Span row_span(const void *p, int64_t T, int64_t V, int64_t ld, int32_t dtype) {
  return span(p, (uint64_t)((T - 1) * ld + V) * dense_size(dtype));
}

bool rows_ok(int64_t V, int64_t ld) {
  return V >= 1 && V <= AF1_HEAD_MAX_VOCAB && ld >= V && ld <= ((int64_t)1 << 32);
}
bool tokens_ok(int64_t T) { return T >= 0 && T <= AF1_HEAD_MAX_TOKENS; }
// the kernels multiply by scale log2(e), which has to be finite
bool scale_ok(float s) { return s > 0.f && s <= 2.3e38f; }

// Whether any two of the spans overlap, the first `outs` of them (written)
// against all; spans of absent arrays are empty.
template <int N>
bool any_alias(const Span (&s)[N], int outs) {
  for (int i = 0; i < outs; ++i)
    for (int j = i + 1; j < N; ++j)
      if (overlap(s[i], s[j])) return true;
  return false;
}

Span maybe(const void *p, uint64_t bytes) { return span(p, p ? bytes : 0); }

}  // namespace

extern "C" {

size_t af1_fp8_code_bytes(int64_t rows, int64_t cols) {
  if (!head_dim_ok(rows) || !head_dim_ok(cols)) return 0;
  return (size_t)blocks_up(rows) * blocks_up(cols) * af1h::kBlk * af1h::kBlk;
}

size_t af1_fp8_scale_bytes(int64_t rows, int64_t cols) {
  if (!head_dim_ok(rows) || !head_dim_ok(cols)) return 0;
  return (size_t)blocks_up(rows) * blocks_up(cols);
}

af1_status af1_fp8_quantize(const void *src, int32_t src_dtype, int64_t rows, int64_t cols,
                            int32_t format, uint8_t *codes, uint8_t *scales, void *stream) {
  if (!dense_ok(src_dtype) || !format_ok(format)) return AF1_ERR_DTYPE;
  if (!head_dim_ok(rows) || !head_dim_ok(cols)) return AF1_ERR_SHAPE;
  if (!src || !codes || !scales) return AF1_ERR_NULL;
  if (!aligned16(src) || !aligned16(codes) || !aligned16(scales)) return AF1_ERR_ALIGN;
  const Span s[] = {code_span(codes, rows, cols), scale_span(scales, rows, cols),
                    span(src, (uint64_t)rows * cols * dense_size(src_dtype))};
  if (any_alias(s, 2)) return AF1_ERR_ALIAS;
  return hip_status(af1h::launch_fp8_quantize(src, src_dtype, rows, cols, format, codes, scales,
                                              as_stream(stream)));
}

af1_status af1_fp8_dequantize(const af1_fp8_matrix *W, void *dst, int32_t dst_dtype,
                              void *stream) {
  if (W && !dense_ok(dst_dtype)) return AF1_ERR_DTYPE;
  const af1_status st = check_matrix(W);
  if (st != AF1_OK) return st;
  if (!dst) return AF1_ERR_NULL;
  if (!aligned16(W->codes) || !aligned16(W->scales) || !aligned16(dst)) return AF1_ERR_ALIGN;
  const Span s[] = {span(dst, (uint64_t)W->rows * W->cols * dense_size(dst_dtype)),
                    code_span(W->codes, W->rows, W->cols),
                    scale_span(W->scales, W->rows, W->cols)};
  if (any_alias(s, 1)) return AF1_ERR_ALIAS;
  return hip_status(af1h::launch_fp8_dequantize(*W, dst, dst_dtype, as_stream(stream)));
}

af1_status af1_fp8_transpose(const af1_fp8_matrix *W, uint8_t *codes, uint8_t *scales,
                             void *stream) {
  const af1_status st = check_matrix(W);
  if (st != AF1_OK) return st;
  if (!codes || !scales) return AF1_ERR_NULL;
  if (!aligned16(W->codes) || !aligned16(W->scales) || !aligned16(codes) || !aligned16(scales))
    return AF1_ERR_ALIGN;
  const Span s[] = {code_span(codes, W->cols, W->rows), scale_span(scales, W->cols, W->rows),
                    code_span(W->codes, W->rows, W->cols),
                    scale_span(W->scales, W->rows, W->cols)};
  if (any_alias(s, 2)) return AF1_ERR_ALIAS;
  return hip_status(af1h::launch_fp8_transpose(*W, codes, scales, as_stream(stream)));
}

size_t af1_fp8_linear_workspace_bytes(int64_t m, int64_t n, int64_t T) {
  if (!head_dim_ok(m) || !head_dim_ok(n) || T < 1 || !tokens_ok(T)) return 0;
  return af1h::fp8_linear_workspace_bytes(m, n, T);
}

af1_status af1_fp8_linear(const af1_fp8_matrix *W, const void *x, int32_t x_dtype,
                          int32_t x_format, int64_t T, void *y, int32_t y_dtype, void *ws,
                          size_t ws_bytes, void *stream) {
  if (!W) return AF1_ERR_NULL;
  if (!dense_ok(x_dtype) || !format_ok(x_format) ||
      (y_dtype != AF1_SRC_F32 && y_dtype != AF1_SRC_BF16))
    return AF1_ERR_DTYPE;
  const af1_status st = check_matrix(W);
  if (st != AF1_OK) return st;
  if (!tokens_ok(T)) return AF1_ERR_BATCH;
  if (T == 0) return AF1_OK;
  if (!x || !y) return AF1_ERR_NULL;
  if (!aligned16(W->codes) || !aligned16(W->scales) || !aligned16(x) || !aligned16(y) ||
      !aligned16(ws))
    return AF1_ERR_ALIGN;
  const size_t need = af1h::fp8_linear_workspace_bytes(W->rows, W->cols, T);
  if (need > 0 && (!ws || ws_bytes < need)) return AF1_ERR_WORKSPACE;
  const Span s[] = {span(y, (uint64_t)T * W->rows * dense_size(y_dtype)), maybe(ws, need),
                    span(x, (uint64_t)T * W->cols * dense_size(x_dtype)),
                    code_span(W->codes, W->rows, W->cols),
                    scale_span(W->scales, W->rows, W->cols)};
  if (any_alias(s, 2)) return AF1_ERR_ALIAS;
  return hip_status(
      af1h::launch_fp8_linear(*W, x, x_dtype, x_format, T, y, y_dtype, ws, as_stream(stream)));
}

size_t af1_token_logprobs_workspace_bytes(int64_t T, int64_t V, int32_t k) {
  if (T < 1 || !tokens_ok(T) || !rows_ok(V, V) || k < 0 || k > AF1_HEAD_MAX_TOP) return 0;
  return af1h::token_logprobs_workspace_bytes(T, V, k);
}

af1_status af1_token_logprobs(const void *logits, int32_t dtype, int64_t T, int64_t V, int64_t ld,
                              float scale, const int64_t *targets, float *logprob, float *entropy,
                              float *lse, int32_t k, float *top_logprob, int64_t *top_index,
                              float *saved, void *ws, size_t ws_bytes, void *stream) {
  if (!dense_ok(dtype)) return AF1_ERR_DTYPE;
  if (!rows_ok(V, ld) || k < 0 || k > AF1_HEAD_MAX_TOP || !scale_ok(scale)) return AF1_ERR_SHAPE;
  if (!tokens_ok(T)) return AF1_ERR_BATCH;
  if (T == 0) return AF1_OK;
  if (!logits || (k > 0 && (!top_logprob || !top_index)) || (logprob && !targets))
    return AF1_ERR_NULL;
  if (!aligned_to(logits, dense_size(dtype)) || !aligned_to(targets, 8) ||
      !aligned4(logprob, entropy, lse) || !aligned16(saved) || !aligned16(ws) ||
      (k > 0 && (!aligned4(top_logprob) || !aligned_to(top_index, 8))))
    return AF1_ERR_ALIGN;
  const size_t need = af1h::token_logprobs_workspace_bytes(T, V, k);
  if (need > 0 && (!ws || ws_bytes < need)) return AF1_ERR_WORKSPACE;
  const uint64_t t = (uint64_t)T;
  const Span s[] = {maybe(logprob, t * 4),
                    maybe(entropy, t * 4),
                    maybe(lse, t * 4),
                    maybe(k > 0 ? top_logprob : nullptr, t * k * 4),
                    maybe(k > 0 ? top_index : nullptr, t * k * 8),
                    maybe(saved, t * 16),
                    maybe(ws, need),
                    row_span(logits, T, V, ld, dtype),
                    maybe(targets, t * 8)};
  if (any_alias(s, 7)) return AF1_ERR_ALIAS;
  return hip_status(af1h::launch_token_logprobs(af1h::Rows{logits, dtype, T, V, ld}, scale,
                                                targets, logprob, entropy, lse, k, top_logprob,
                                                top_index, saved, ws, as_stream(stream)));
}

af1_status af1_token_logprobs_backward(const void *logits, int32_t dtype, int64_t T, int64_t V,
                                       int64_t ld, float scale, const int64_t *targets,
                                       const float *saved, const float *g_logprob,
                                       const float *g_entropy, void *dlogits, int64_t ldd,
                                       void *stream) {
  if (!dense_ok(dtype)) return AF1_ERR_DTYPE;
  if (!rows_ok(V, ld) || !rows_ok(V, ldd) || !scale_ok(scale)) return AF1_ERR_SHAPE;
  if (!tokens_ok(T)) return AF1_ERR_BATCH;
  if (T == 0) return AF1_OK;
  if (!logits || !saved || !dlogits || (g_logprob && !targets)) return AF1_ERR_NULL;
  if (!aligned_to(logits, dense_size(dtype)) || !aligned_to(dlogits, dense_size(dtype)) ||
      !aligned_to(targets, 8) || !aligned16(saved) || !aligned4(g_logprob, g_entropy))
    return AF1_ERR_ALIGN;
  const uint64_t t = (uint64_t)T;
  const bool in_place = dlogits == logits && ldd == ld;
  const Span s[] = {row_span(dlogits, T, V, ldd, dtype), maybe(targets, t * 8), span(saved, t * 16),
                    maybe(g_logprob, t * 4), maybe(g_entropy, t * 4),
                    in_place ? span(logits, 0) : row_span(logits, T, V, ld, dtype)};
  if (any_alias(s, 1)) return AF1_ERR_ALIAS;
  return hip_status(af1h::launch_token_logprobs_backward(af1h::Rows{logits, dtype, T, V, ld}, scale,
                                                         targets, saved, g_logprob, g_entropy,
                                                         dlogits, ldd, as_stream(stream)));
}

size_t af1_distill_kl_workspace_bytes(int64_t T, int64_t V) {
  if (T < 1 || !tokens_ok(T) || !rows_ok(V, V)) return 0;
  return af1h::distill_kl_workspace_bytes(T, V);
}

af1_status af1_distill_kl(const void *student, const void *teacher, int32_t dtype, int64_t T,
                          int64_t V, int64_t ld_s, int64_t ld_t, float scale, const float *weight,
                          float *kl, void *dstudent, int64_t ldd, void *ws, size_t ws_bytes,
                          void *stream) {
  if (!dense_ok(dtype)) return AF1_ERR_DTYPE;
  if (!rows_ok(V, ld_s) || !rows_ok(V, ld_t) || (dstudent && !rows_ok(V, ldd)) ||
      !scale_ok(scale))
    return AF1_ERR_SHAPE;
  if (!tokens_ok(T)) return AF1_ERR_BATCH;
  if (T == 0) return AF1_OK;
  if (!student || !teacher || !kl) return AF1_ERR_NULL;
  if (!aligned_to(student, dense_size(dtype)) || !aligned_to(teacher, dense_size(dtype)) ||
      !aligned_to(dstudent, dense_size(dtype)) || !aligned4(weight, kl) || !aligned16(ws))
    return AF1_ERR_ALIGN;
  const size_t need = af1h::distill_kl_workspace_bytes(T, V);
  if (need > 0 && (!ws || ws_bytes < need)) return AF1_ERR_WORKSPACE;
  const uint64_t t = (uint64_t)T;
  const bool in_place = dstudent == student && ldd == ld_s;
  const Span sd = dstudent ? row_span(dstudent, T, V, ldd, dtype) : span(nullptr, 0);
  const Span ss = row_span(student, T, V, ld_s, dtype);
  const Span s[] = {span(kl, t * 4), maybe(ws, need), sd, row_span(teacher, T, V, ld_t, dtype),
                    maybe(weight, t * 4)};
  if (any_alias(s, 3) || overlap(s[0], ss) || overlap(s[1], ss) || (!in_place && overlap(sd, ss)))
    return AF1_ERR_ALIAS;
  return hip_status(af1h::launch_distill_kl(af1h::Rows{student, dtype, T, V, ld_s}, teacher, ld_t,
                                            scale, weight, kl, dstudent, ldd, ws,
                                            as_stream(stream)));
}

}  // extern "C"
