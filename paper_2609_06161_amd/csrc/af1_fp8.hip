// The 8-bit block-scaled matrix of af1_head.h and its linear.
//
//   y[t, i] = sum_J 2^(ex[t, J] + ew[I, J]) sum_{j in J} cx[t, j] cw[i, j]
//
// over the column blocks J of 128, I = i / 128.  The scales are powers of two,
// which the scaled matrix instructions take as E8M0 operands (a byte e + 127),
// so a block's scale costs no instruction and no rounding: the accumulators
// run through all blocks.  One instruction multiplies 32 x 32 (or 16 x 16)
// outputs over 64 (128) columns; a lane's operand is 32 bytes of one row.
// Which columns those are is free as long as both operands agree, since all of
// a block's columns share one scale.
#include "af1_device.h"
#include "af1_head_internal.h"

namespace af1h {
namespace {

using af1::bf16_to_f32;
using af1::f16_to_f32;
using af1::f32_to_bf16;
using af1::f32_to_f16;

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));

constexpr int64_t kTileBytes = kBlk * kBlk;

template <int kType>
__device__ __forceinline__ float load_dense(const void *p, int64_t i) {
  if constexpr (kType == AF1_SRC_F32) return static_cast<const float *>(p)[i];
  if constexpr (kType == AF1_SRC_BF16) return bf16_to_f32(static_cast<const uint16_t *>(p)[i]);
  return f16_to_f32(static_cast<const uint16_t *>(p)[i]);
}

template <int kType>
__device__ __forceinline__ void store_dense(void *p, int64_t i, float v) {
  if constexpr (kType == AF1_SRC_F32) static_cast<float *>(p)[i] = v;
  if constexpr (kType == AF1_SRC_BF16) static_cast<uint16_t *>(p)[i] = f32_to_bf16(v);
  if constexpr (kType == AF1_SRC_F16) static_cast<uint16_t *>(p)[i] = f32_to_f16(v);
}

// |x| of a finite entry, 0 for the others: what a block's scale is chosen from.
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < __builtin_inff() ? a : 0.f;
}

// Smallest e with amax <= MAX 2^e, MAX = 1.75 * 2^8 (e4m3) or 1.75 * 2^15
// (e5m2), read off amax's exponent and mantissa; 0 for amax = 0.  Subnormal
// amax end at the lowest scale.
template <int kFormat>
__device__ __forceinline__ int block_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - (kFormat == AF1_FP8_E4M3 ? 8 : 15) +
                ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return amax == 0.f ? 0 : e < -127 ? -127 : e;
}

// 2^e for e in -127 .. 127 (2^-127 is subnormal).
__device__ __forceinline__ float pow2(int e) {
  return e == -127 ? __uint_as_float(0x00400000u) : __uint_as_float((uint32_t)(e + 127) << 23);
}

// Codes of four values (already scaled), the first in the low byte.
template <int kFormat>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  int w = 0;
  if constexpr (kFormat == AF1_FP8_E4M3) {
    w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  } else {
    w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
    w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
  }
  return (uint32_t)w;
}

template <int kFormat, int kByte>
__device__ __forceinline__ float decode(uint32_t w) {
  if constexpr (kFormat == AF1_FP8_E4M3) return __builtin_amdgcn_cvt_f32_fp8((int)w, kByte);
  return __builtin_amdgcn_cvt_f32_bf8((int)w, kByte);
}

// ---------------------------------------------------------------------------
// Quantisation, reading back, transposition: one workgroup a tile.
// ---------------------------------------------------------------------------

// Thread t of 256 holds row t / 2, columns 64 (t % 2) .. + 63 of the tile.
template <int kType, int kFormat>
__global__ __launch_bounds__(256) void quantize_kernel(const void *src, int64_t rows, int64_t cols,
                                                       uint8_t *codes, uint8_t *scales) {
  __shared__ float wmax[4];
  const int64_t C = (cols + kBlk - 1) / kBlk, tile = blockIdx.x;
  const int64_t r0 = tile / C * kBlk, c0 = tile % C * kBlk;
  const int t = threadIdx.x;
  const int64_t row = r0 + (t >> 1), col = c0 + (t & 1) * 64;
  float v[64], amax = 0.f;
#pragma unroll
  for (int j = 0; j < 64; ++j) {
    v[j] = row < rows && col + j < cols ? load_dense<kType>(src, row * cols + col + j) : 0.f;
    amax = fmaxf(amax, finite_abs(v[j]));
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor(amax, off, 64));
  if ((t & 63) == 0) wmax[t >> 6] = amax;
  __syncthreads();
  amax = fmaxf(fmaxf(wmax[0], wmax[1]), fmaxf(wmax[2], wmax[3]));
  const int e = block_exponent<kFormat>(amax);
  const float inv = pow2(-e);
  uint4 *dst = reinterpret_cast<uint4 *>(codes + tile * kTileBytes + t * 64);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float *p = v + 16 * q + 4 * i;
      w[i] = encode4<kFormat>(p[0] * inv, p[1] * inv, p[2] * inv, p[3] * inv);
    }
    dst[q] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  if (t == 0) scales[tile] = (uint8_t)(e + 127);
}

template <int kType, int kFormat>
__global__ __launch_bounds__(256) void dequantize_kernel(const uint8_t *codes,
                                                         const uint8_t *scales, int64_t rows,
                                                         int64_t cols, void *dst) {
  const int64_t C = (cols + kBlk - 1) / kBlk, tile = blockIdx.x;
  const int t = threadIdx.x;
  const int64_t row = tile / C * kBlk + (t >> 1), col = tile % C * kBlk + (t & 1) * 64;
  if (row >= rows) return;
  const float scale = pow2((int)scales[tile] - 127);
  const uint32_t *src = reinterpret_cast<const uint32_t *>(codes + tile * kTileBytes + t * 64);
#pragma unroll 4
  for (int q = 0; q < 16; ++q) {
    const uint32_t w = src[q];
    const float v[4] = {decode<kFormat, 0>(w), decode<kFormat, 1>(w), decode<kFormat, 2>(w),
                        decode<kFormat, 3>(w)};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (col + 4 * q + i < cols) store_dense<kType>(dst, row * cols + col + 4 * q + i, v[i] * scale);
  }
}

__global__ __launch_bounds__(256) void transpose_tiles_kernel(const uint8_t *codes,
                                                              const uint8_t *scales, int64_t R,
                                                              int64_t C, uint8_t *codesT,
                                                              uint8_t *scalesT) {
  __shared__ uint8_t tile[kBlk][kBlk + 4];
  const int64_t i = blockIdx.x / C, j = blockIdx.x % C;
  const uint8_t *src = codes + (int64_t)blockIdx.x * kTileBytes;
  uint8_t *dst = codesT + (j * R + i) * kTileBytes;
  for (int b = threadIdx.x; b < kTileBytes; b += 256) tile[b >> 7][b & 127] = src[b];
  __syncthreads();
  for (int b = threadIdx.x; b < kTileBytes; b += 256) dst[b] = tile[b & 127][b >> 7];
  if (threadIdx.x == 0) scalesT[j * R + i] = scales[blockIdx.x];
}

// ---------------------------------------------------------------------------
// The linear
// ---------------------------------------------------------------------------

// Tokens' codes in the workspace: tiles of 128 tokens x 128 columns as the
// weight's, columns behind n zero, rows behind T not written (each output
// depends on its own token's row only).  Scales: 128 bytes a tile, the byte of
// token row at 4 (row % 32) + row / 32, so that one dword holds what a lane of
// a 32-row operand needs for the tile's four row blocks.
struct XTiles {
  uint8_t *codes, *scales;
};

__host__ __device__ inline XTiles x_tiles(void *ws, int64_t n, int64_t T) {
  const int64_t tiles = (T + kBlk - 1) / kBlk * ((n + kBlk - 1) / kBlk);
  return XTiles{static_cast<uint8_t *>(ws), static_cast<uint8_t *>(ws) + tiles * kTileBytes};
}

// Sixteen lanes a token and column block, eight columns a lane.
template <int kType, int kFormat>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const void *x, int64_t T, int64_t n,
                                                            XTiles out) {
  const int64_t C = (n + kBlk - 1) / kBlk;
  const int64_t piece = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int lane = threadIdx.x & 15;
  const int64_t t = piece / C, J = piece % C;
  if (t >= T) return;  // the sixteen lanes together
  const int64_t col = J * kBlk + lane * 8;
  float v[8], amax = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = col + i < n ? load_dense<kType>(x, t * n + col + i) : 0.f;
    amax = fmaxf(amax, finite_abs(v[i]));
  }
#pragma unroll
  for (int off = 8; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor(amax, off, 16));
  const int e = block_exponent<kFormat>(amax);
  const float inv = pow2(-e);
  const int64_t tile = t / kBlk * C + J;
  const int row = (int)(t % kBlk);
  *reinterpret_cast<uint2 *>(out.codes + tile * kTileBytes + row * kBlk + lane * 8) =
      make_uint2(encode4<kFormat>(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                 encode4<kFormat>(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv));
  if (lane == 0) out.scales[tile * kBlk + (row & 31) * 4 + (row >> 5)] = (uint8_t)(e + 127);
}

// Sixteen bfloat16 values of sixteen codes, for two matrix instructions.
template <int kFormat>
__device__ __forceinline__ void to_bf16(const int *w, bf8v (&out)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bf2v lo, hi;
    if constexpr (kFormat == AF1_FP8_E4M3) {
      lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.f, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.f, true);
    } else {
      lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w[i], 1.f, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w[i], 1.f, true);
    }
    const int j = (i & 1) * 4;
    out[i >> 1][j] = lo[0];
    out[i >> 1][j + 1] = lo[1];
    out[i >> 1][j + 2] = hi[0];
    out[i >> 1][j + 3] = hi[1];
  }
}

// tmp += products of 64 columns, exact and unscaled.
template <int kWFormat, int kXFormat>
__device__ __forceinline__ v16f mul_bf16(v8i w, v8i x, v16f tmp) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int wi[4] = {w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]};
    const int xi[4] = {x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
    bf8v a[2], b[2];
    to_bf16<kWFormat>(wi, a);
    to_bf16<kXFormat>(xi, b);
    tmp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[0], tmp, 0, 0, 0);
    tmp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1], b[1], tmp, 0, 0, 0);
  }
  return tmp;
}

// A wave computes 32 rows of the weight x 32 tokens, operands straight from
// memory.  Token tiles hold 128 rows, so the operand reads stay inside them.
template <int kXFormat, int kWFormat, int kOut>
__global__ __launch_bounds__(256) void linear_kernel(const uint8_t *wcodes, const uint8_t *wscales,
                                                     XTiles x, int64_t T, int64_t m, int64_t n,
                                                     void *y) {
  const int64_t C = (n + kBlk - 1) / kBlk;
  const int64_t strips = (m + 31) / 32;
  const int64_t strip = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (strip >= strips) return;
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  const int64_t t0 = (int64_t)blockIdx.y * 32, i0 = strip * 32;
  const uint8_t *xa = x.codes + t0 / kBlk * C * kTileBytes + (t0 % kBlk + r) * kBlk + h * 32;
  const uint8_t *xs = x.scales + t0 / kBlk * C * kBlk + r * 4 + t0 % kBlk / 32;
  const uint8_t *wb = wcodes + i0 / kBlk * C * kTileBytes + (i0 % kBlk + r) * kBlk + h * 32;
  const uint8_t *wsc = wscales + i0 / kBlk * C;
  v16f acc = {};
  for (int64_t J = 0; J < C; ++J) {
    const int sx = xs[J * kBlk], sw = wsc[J];
    v16f tmp = {};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const v8i a = *reinterpret_cast<const v8i *>(wb + J * kTileBytes + s * 64);
      const v8i b = *reinterpret_cast<const v8i *>(xa + J * kTileBytes + s * 64);
      if constexpr (kOut == AF1_SRC_BF16)
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, kWFormat, kXFormat, 0, sw,
                                                              0, sx);
      else
        tmp = mul_bf16<kWFormat, kXFormat>(a, b, tmp);
    }
    if constexpr (kOut != AF1_SRC_BF16)
#pragma unroll
      for (int g = 0; g < 16; ++g) acc[g] += ldexpf(tmp[g], sx + sw - 254);
  }
  const int64_t t = t0 + r;
#pragma unroll
  for (int g = 0; g < 16; ++g) {
    const int64_t i = i0 + (g & 3) + 8 * (g >> 2) + 4 * h;
    if (t < T && i < m) store_dense<kOut>(y, t * m + i, acc[g]);
  }
}

template <int kV>
struct Int {
  static constexpr int value = kV;
};

template <typename F>
auto with_format(int f, F &&g) {
  if (f == AF1_FP8_E4M3) return g(Int<AF1_FP8_E4M3>{});
  return g(Int<AF1_FP8_E5M2>{});
}

template <typename F>
auto with_dense(int t, F &&g) {
  if (t == AF1_SRC_F32) return g(Int<AF1_SRC_F32>{});
  if (t == AF1_SRC_BF16) return g(Int<AF1_SRC_BF16>{});
  return g(Int<AF1_SRC_F16>{});
}

}  // namespace

hipError_t launch_fp8_quantize(const void *src, int dtype, int64_t rows, int64_t cols, int format,
                               uint8_t *codes, uint8_t *scales, hipStream_t s) {
  const unsigned tiles = (unsigned)(blocks_up(rows) * blocks_up(cols));
  return with_dense(dtype, [&](auto t) {
    return with_format(format, [&](auto f) {
      quantize_kernel<t.value, f.value><<<tiles, 256, 0, s>>>(src, rows, cols, codes, scales);
      return hipGetLastError();
    });
  });
}

hipError_t launch_fp8_dequantize(const af1_fp8_matrix &W, void *dst, int dtype, hipStream_t s) {
  const unsigned tiles = (unsigned)(blocks_up(W.rows) * blocks_up(W.cols));
  return with_dense(dtype, [&](auto t) {
    return with_format(W.format, [&](auto f) {
      dequantize_kernel<t.value, f.value>
          <<<tiles, 256, 0, s>>>(W.codes, W.scales, W.rows, W.cols, dst);
      return hipGetLastError();
    });
  });
}

hipError_t launch_fp8_transpose(const af1_fp8_matrix &W, uint8_t *codes, uint8_t *scales,
                                hipStream_t s) {
  const int64_t R = blocks_up(W.rows), C = blocks_up(W.cols);
  transpose_tiles_kernel<<<(unsigned)(R * C), 256, 0, s>>>(W.codes, W.scales, R, C, codes, scales);
  return hipGetLastError();
}

size_t fp8_linear_workspace_bytes(int64_t, int64_t n, int64_t T) {
  return (size_t)blocks_up(T) * blocks_up(n) * (kTileBytes + kBlk);
}

hipError_t launch_fp8_linear(const af1_fp8_matrix &W, const void *x, int x_dtype, int x_format,
                             int64_t T, void *y, int y_dtype, void *ws, hipStream_t s) {
  const int64_t m = W.rows, n = W.cols;
  const XTiles xt = x_tiles(ws, n, T);
  return with_format(x_format, [&](auto xf) {
    const hipError_t e = with_dense(x_dtype, [&](auto t) {
      quantize_rows_kernel<t.value, xf.value>
          <<<(unsigned)((T * blocks_up(n) + 15) / 16), 256, 0, s>>>(x, T, n, xt);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    return with_format(W.format, [&](auto wf) {
      const dim3 g((unsigned)((m + 127) / 128), (unsigned)((T + 31) / 32));
      if (y_dtype == AF1_SRC_F32)
        linear_kernel<xf.value, wf.value, AF1_SRC_F32>
            <<<g, 256, 0, s>>>(W.codes, W.scales, xt, T, m, n, y);
      else
        linear_kernel<xf.value, wf.value, AF1_SRC_BF16>
            <<<g, 256, 0, s>>>(W.codes, W.scales, xt, T, m, n, y);
      return hipGetLastError();
    });
  });
}

}  // namespace af1h
