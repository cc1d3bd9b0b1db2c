// Host-side launchers behind the C ABI of the output head (af1_head.h).
// Arguments are already validated by af1_head_api.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "af1_head.h"

namespace af1h {

constexpr int kBlk = 128;  // rows and columns of a block that share a scale

// Compute units of the current device (queried once per device; 256 if the
// query fails).
int device_cus();

inline int64_t blocks_up(int64_t n) { return (n + kBlk - 1) / kBlk; }

hipError_t launch_fp8_quantize(const void *src, int dtype, int64_t rows, int64_t cols, int format,
                               uint8_t *codes, uint8_t *scales, hipStream_t s);
hipError_t launch_fp8_dequantize(const af1_fp8_matrix &W, void *dst, int dtype, hipStream_t s);
hipError_t launch_fp8_transpose(const af1_fp8_matrix &W, uint8_t *codes, uint8_t *scales,
                                hipStream_t s);

size_t fp8_linear_workspace_bytes(int64_t m, int64_t n, int64_t T);
hipError_t launch_fp8_linear(const af1_fp8_matrix &W, const void *x, int x_dtype, int x_format,
                             int64_t T, void *y, int y_dtype, void *ws, hipStream_t s);

// Rows of logits: T rows of V elements, ld apart.
struct Rows {
  const void *p;
  int dtype;
  int64_t T, V, ld;
};

size_t token_logprobs_workspace_bytes(int64_t T, int64_t V, int k);
hipError_t launch_token_logprobs(const Rows &z, float scale, const int64_t *targets,
                                 float *logprob, float *entropy, float *lse, int k,
                                 float *top_logprob, int64_t *top_index, float *saved, void *ws,
                                 hipStream_t s);
hipError_t launch_token_logprobs_backward(const Rows &z, float scale, const int64_t *targets,
                                          const float *saved, const float *g_logprob,
                                          const float *g_entropy, void *dlogits, int64_t ldd,
                                          hipStream_t s);

size_t distill_kl_workspace_bytes(int64_t T, int64_t V);
hipError_t launch_distill_kl(const Rows &student, const void *teacher, int64_t ld_t, float scale,
                             const float *weight, float *kl, void *dstudent, int64_t ldd,
                             void *ws, hipStream_t s);

}  // namespace af1h
