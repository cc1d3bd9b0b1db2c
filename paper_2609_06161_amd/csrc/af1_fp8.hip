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

typedef int i32x4 __attribute__((ext_vector_type(4)));
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

// The values of a lane's 32 codes, for four matrix instructions.
template <int kFormat>
__device__ __forceinline__ void to_bf16(v8i w, bf8v (&out)[4]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
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

// acc += products of 64 columns at the scales (E8M0): W's is byte 0 of sw, the
// tokens' byte kByte of sx.
template <int kWFormat, int kXFormat, int kByte>
__device__ __forceinline__ v16f mfma_scaled(v8i w, v8i x, v16f acc, int sw, int sx) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, acc, kWFormat, kXFormat, 0, sw,
                                                         kByte, sx);
}

// Four floats and eight bfloat16 that need their element's alignment only.
struct __attribute__((packed, aligned(4))) Four {
  float v[4];
};
struct __attribute__((packed, aligned(2))) Chunk {
  uint32_t v[4];
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return (uint32_t)f32_to_bf16(a) | (uint32_t)f32_to_bf16(b) << 16;
}

// The first `left` (or all) of eight values.
__device__ __forceinline__ void store8_bf16(uint16_t *p, int64_t left, uint4 v) {
  if (left >= 8) {
    *reinterpret_cast<Chunk *>(p) = Chunk{{v.x, v.y, v.z, v.w}};
    return;
  }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < left) p[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
}

// ---------------------------------------------------------------------------
// Tiled product.  A workgroup of kWR x kWC waves computes kTW rows of W x kTX
// tokens; a wave kFR x kFC pieces of 32 x 32.  A step is half a column block
// (64 columns).  Its bytes go from memory straight into one of kStages LDS
// buffers (buffer loads with an LDS destination) and from there into registers
// one step before they are multiplied, so in step s
//   buffer s + 1 has landed and is read into registers,
//   buffers s + 2 .. s + kStages - 1 are on their way, and
//   buffer s, whose operands are in registers, is filled with step s + kStages.
// A step meets the other waves once; nothing in it waits for memory that was
// asked for in the last kStages - 2 steps.  (With two buffers of a whole block
// each, which hold as many bytes, a step waited for copies issued in the step
// before: 1289 us where this takes 992 at 128256 x 4096 and 2048 tokens.)
//
// LDS holds rows of 64 bytes, four chunks of 16.  A copy instruction writes 64
// consecutive chunks (sixteen rows), one a lane, and a lane chooses its
// source: chunk c of row r is kept at position c XOR (r / 4 mod 4).  The LDS
// serves a 16-byte read of 64 lanes in groups of sixteen, of which four have
// equal r mod 4; these then fall in distinct banks (counted: 0.3 conflict
// cycles a read, against 4.1 with rows of 128 bytes and c XOR (r mod 8)).
// ---------------------------------------------------------------------------

typedef __attribute__((address_space(3))) void lds_void;

__device__ __forceinline__ i32x4 make_rsrc(const void *p) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  return i32x4{(int)(uint32_t)a, (int)(uint32_t)(a >> 32), 0x7fffffff, 0x00020000};
}

// One 16-byte chunk a lane from rsrc + voff + soff into 64 chunks at dst.
__device__ __forceinline__ void copy16(i32x4 r, uint8_t *dst, int voff, int soff) {
  const uint32_t m = (uint32_t)(size_t)(lds_void *)dst;
  asm volatile("buffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(voff), "s"(r), "s"(soff), "{m0}"(m)
               : "memory");
}

// One dword, or one byte, a lane from the lane's own address into 64 dwords at
// dst.
__device__ __forceinline__ void copy4(const void *src, uint8_t *dst) {
  const uint32_t m = (uint32_t)(size_t)(lds_void *)dst;
  asm volatile("global_load_lds_dword %0, off" ::"v"(src), "{m0}"(m) : "memory");
}
__device__ __forceinline__ void copy1(const void *src, uint8_t *dst) {
  const uint32_t m = (uint32_t)(size_t)(lds_void *)dst;
  asm volatile("global_load_lds_ubyte %0, off" ::"v"(src), "{m0}"(m) : "memory");
}

// All but kLeft of this wave's copies have landed, its LDS reads are done, and
// every other wave's too.
template <int kLeft>
__device__ __forceinline__ void step_barrier() {
  static_assert(kLeft >= 0 && kLeft < 64, "vmcnt has six bits");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLeft) : "memory");
}

template <int kTW_, int kTX_, int kWR_, int kWC_, int kStages_>
struct Tile {
  static constexpr int kTW = kTW_, kTX = kTX_, kWR = kWR_, kWC = kWC_, kStages = kStages_;
  static constexpr int kWaves = kWR * kWC, kThreads = 64 * kWaves;
  static constexpr int kFR = kTW / kWR / 32, kFC = kTX / kWC / 32;  // pieces a wave
  static constexpr int kCodes = (kTW + kTX) * 64;      // LDS bytes a step
  static constexpr int kStage = kCodes + kWaves * 512;  // and the scales', two slots a wave
  static constexpr int kCopies = kCodes / 1024 / kWaves;  // a wave and step, and two of scales
  static constexpr int kOutRow = kFR * 64 + 16;  // LDS bytes of a token's bf16 outputs
  static constexpr int kOutLds = kWaves * 32 * kOutRow;
  static constexpr int kLds = kStages * kStage > kOutLds ? kStages * kStage : kOutLds;
  static_assert(kCodes % (1024 * kWaves) == 0 && kTW % 16 == 0 && kTX % 16 == 0);
  static_assert((kStages & (kStages - 1)) == 0 && kLds <= 160 * 1024);
};

struct LinearArgs {
  const uint8_t *wcodes, *wscales;
  XTiles x;
  int64_t T, m;
  int C;             // column blocks
  int R, X;          // 128-row blocks of W and of the tokens
  int nW, nX;        // tiles
  void *y;
};

template <typename TT, int kWFormat, int kXFormat, int kOut>
__global__ __launch_bounds__(TT::kThreads) void tile_kernel(LinearArgs g) {
  constexpr int kFR = TT::kFR, kFC = TT::kFC, kS = TT::kStages;
  extern __shared__ uint8_t lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  // workgroups of one XCD (blockIdx mod 8) take a contiguous range of tiles,
  // token tiles fastest, so that they share rows of W in their L2
  const int total = g.nW * g.nX;
  int L = blockIdx.x;
  if ((total & 7) == 0) L = (L & 7) * (total >> 3) + (L >> 3);
  const int w0 = L / g.nX * TT::kTW, x0 = L % g.nX * TT::kTX;  // first row and token
  const int C = g.C;

  // copy roles: piece p = wave kCopies + q is sixteen tile rows, W's first
  const int64_t band = (int64_t)C * kTileBytes;  // bytes of 128 rows
  const int wb0 = w0 >> 7, xb0 = x0 >> 7;
  const i32x4 wr = make_rsrc(g.wcodes + wb0 * band);
  const i32x4 xr = make_rsrc(g.x.codes + xb0 * band);
  const int voff = (lane >> 2) * kBlk + (((lane & 3) ^ (lane >> 4)) << 4);
  int soff[TT::kCopies];
#pragma unroll
  for (int q = 0; q < TT::kCopies; ++q) {
    const int row = 16 * (wave * TT::kCopies + q);
    const bool isw = row < TT::kTW;
    const int at = isw ? (w0 & 127) + row : (x0 & 127) + row - TT::kTW;
    // a tile may reach past the last block: it reads that one again, and what
    // comes of it is not stored
    const int blk = min(at >> 7, (isw ? g.R - 1 - wb0 : g.X - 1 - xb0));
    soff[q] = (int)(blk * band) + (at & 127) * kBlk;
  }
  // operands: rows row0 .. of W and tokens tok0 .. of the tile
  const int row0 = wave / TT::kWC * kFR * 32, tok0 = wave % TT::kWC * kFC * 32;
  const int wblk = min((w0 + row0) >> 7, g.R - 1), xblk = min((x0 + tok0) >> 7, g.X - 1);
  // scales: the tokens' dwords and W's byte of a block, each lane its own
  const uint8_t *wsc = g.wscales + (int64_t)wblk * C;
  const uint8_t *xsc = g.x.scales + (int64_t)xblk * C * kBlk + r * 4;
  // copy k of step s: codes, then the scales
  constexpr int kCopies = TT::kCopies + 2;
  auto copy = [&](int s, int k) {
    uint8_t *st = lds + (s & (kS - 1)) * TT::kStage;
    const int J = s >> 1, p = wave * TT::kCopies + k;
    if (k < TT::kCopies)
      copy16(16 * p < TT::kTW ? wr : xr, st + p * 1024, voff,
             soff[k < TT::kCopies ? k : 0] + J * (int)kTileBytes + (s & 1) * 64);
    else if (k == TT::kCopies)
      copy4(xsc + J * kBlk, st + TT::kCodes + wave * 512);
    else
      copy1(wsc + J, st + TT::kCodes + wave * 512 + 256);
  };

  const int xshift = 8 * (((x0 + tok0) & 127) >> 5);
  struct Operands {
    v8i a[kFR], b[kFC];
    int sw, sx;
  };
  // piece k of step s: W's, the tokens', the scales
  constexpr int kReads = kFR + kFC + 1;
  const int lo = ((2 * h) ^ (r >> 2 & 3)) << 4, hi = lo ^ 16;
  auto read = [&](int s, int k, Operands &o) {
    const uint8_t *st = lds + (s & (kS - 1)) * TT::kStage;
    if (k == 0) {
      const uint32_t *sc = reinterpret_cast<const uint32_t *>(st + TT::kCodes + wave * 512);
      o.sx = (int)(sc[r] >> xshift);
      o.sw = (int)sc[64 + lane];
      return;
    }
    const int piece = k - 1;
    const int row = piece < kFR ? row0 + 32 * piece : TT::kTW + tok0 + 32 * (piece - kFR);
    const uint8_t *p = st + (row + r) * 64;
    const i32x4 u = *reinterpret_cast<const i32x4 *>(p + lo);
    const i32x4 v = *reinterpret_cast<const i32x4 *>(p + hi);
    (piece < kFR ? o.a[piece < kFR ? piece : 0] : o.b[piece < kFR ? 0 : piece - kFR]) =
        v8i{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
  };

  v16f acc[kFR][kFC] = {};
  v16f tmp[kFR][kFC];  // a block's sums, for outputs in fp32
  auto product = [&](const Operands &o, bool second, int i, int j) {
    if constexpr (kOut == AF1_SRC_BF16) {
      // which byte holds a piece's scale is part of the instruction
      if (j == 0) acc[i][0] = mfma_scaled<kWFormat, kXFormat, 0>(o.a[i], o.b[0], acc[i][0], o.sw, o.sx);
      if constexpr (kFC > 1)
        if (j == 1)
          acc[i][1] = mfma_scaled<kWFormat, kXFormat, 1>(o.a[i], o.b[1], acc[i][1], o.sw, o.sx);
      if constexpr (kFC > 2) {
        if (j == 2)
          acc[i][2] = mfma_scaled<kWFormat, kXFormat, 2>(o.a[i], o.b[2], acc[i][2], o.sw, o.sx);
        if (j == 3)
          acc[i][3] = mfma_scaled<kWFormat, kXFormat, 3>(o.a[i], o.b[3], acc[i][3], o.sw, o.sx);
      }
    } else {
      bf8v a[4], b[4];
      to_bf16<kWFormat>(o.a[i], a);
      to_bf16<kXFormat>(o.b[j], b);
      v16f t = second ? tmp[i][j] : v16f{};
#pragma unroll
      for (int q = 0; q < 4; ++q)
        t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[q], b[q], t, 0, 0, 0);
      tmp[i][j] = t;
      if (second) {
        const int e = o.sw + (o.sx >> (8 * j) & 255) - 254;
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[i][j][q] += ldexpf(t[q], e);
      }
    }
  };

  // Step s: its products, and between them the copies of step s + kStages and
  // the reads of step s + 1, the reads in the first half so that the barrier
  // does not wait for them.  A burst of copies in front of the products keeps
  // the wave's issue waiting behind the other waves' bursts.
  constexpr int kProducts = kFR * kFC;
  auto step = [&](int s, const Operands &o, Operands &next, bool second, bool more, bool last) {
#pragma unroll
    for (int p = 0; p < kProducts; ++p) {
      constexpr int kHalf = kProducts > 1 ? kProducts / 2 : 1;
      if (!last && p < kHalf)
#pragma unroll
        for (int k = p * kReads / kHalf; k < (p + 1) * kReads / kHalf; ++k) read(s + 1, k, next);
      if (more)
#pragma unroll
        for (int k = p * kCopies / kProducts; k < (p + 1) * kCopies / kProducts; ++k)
          copy(s + kS, k);
      product(o, second, p / kFC, p % kFC);
      if constexpr (kOut == AF1_SRC_BF16) __builtin_amdgcn_sched_barrier(0);
    }
  };

  // copies of the steps behind the next one
  constexpr int kAhead = (kS - 2) * kCopies;
  const int steps = 2 * C;
  for (int s = 0; s < min(kS, steps); ++s)
#pragma unroll
    for (int k = 0; k < kCopies; ++k) copy(s, k);
  step_barrier<0>();
  Operands o0, o1;
#pragma unroll
  for (int k = 0; k < kReads; ++k) read(0, k, o0);
  int J = 0;
  for (; 2 * J + 1 + kS < steps; ++J) {
    step_barrier<kAhead>();
    step(2 * J, o0, o1, false, true, false);
    step_barrier<kAhead>();
    step(2 * J + 1, o1, o0, true, true, false);
  }
  // nothing more to copy: what is left has been on its way for long
  for (; J < C - 1; ++J) {
    step_barrier<0>();
    step(2 * J, o0, o1, false, false, false);
    step_barrier<0>();
    step(2 * J + 1, o1, o0, true, false, false);
  }
  step_barrier<0>();
  step(2 * J, o0, o1, false, false, false);
  step_barrier<0>();
  step(2 * J + 1, o1, o0, true, false, true);

  // Outputs.  A lane holds, for its token, four consecutive rows of W in each
  // four accumulators.
  if constexpr (kOut == AF1_SRC_F32) {
    float *y = static_cast<float *>(g.y);
#pragma unroll
    for (int j = 0; j < kFC; ++j) {
      const int64_t t = x0 + tok0 + 32 * j + r;
      if (t >= g.T) continue;
#pragma unroll
      for (int i = 0; i < kFR; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t row = (int64_t)w0 + row0 + 32 * i + 8 * q + 4 * h;
          float *p = y + t * g.m + row;
          const v16f &c = acc[i][j];
          if (row + 4 <= g.m) {
            Four f{{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]}};
            *reinterpret_cast<Four *>(p) = f;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (row + e < g.m) p[e] = c[4 * q + e];
          }
        }
    }
  } else {
    // through LDS, 32 tokens at a time, so that a token's entries leave in
    // 16-byte pieces next to each other; each wave uses a region of its own
    uint16_t *y = static_cast<uint16_t *>(g.y);
    step_barrier<0>();
    uint8_t *mine = lds + wave * 32 * TT::kOutRow;
    constexpr int kLanes = kFR * 4;  // lanes a token
#pragma unroll
    for (int j = 0; j < kFC; ++j) {
#pragma unroll
      for (int i = 0; i < kFR; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const v16f &c = acc[i][j];
          const uint32_t lo = pack_bf16(c[4 * q], c[4 * q + 1]);
          const uint32_t hi = pack_bf16(c[4 * q + 2], c[4 * q + 3]);
          *reinterpret_cast<uint2 *>(mine + r * TT::kOutRow + (32 * i + 8 * q + 4 * h) * 2) =
              make_uint2(lo, hi);
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int k = 0; k < kLanes / 2; ++k) {
        const int tok = k * (64 / kLanes) + lane / kLanes, piece = lane % kLanes;
        const uint4 v = *reinterpret_cast<const uint4 *>(mine + tok * TT::kOutRow + piece * 16);
        const int64_t t = x0 + tok0 + 32 * j + tok, row = (int64_t)w0 + row0 + 8 * piece;
        if (t < g.T && row < g.m) store8_bf16(y + t * g.m + row, g.m - row, v);
      }
      __builtin_amdgcn_wave_barrier();
    }
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

template <typename TT, int kWFormat, int kXFormat, int kOut>
hipError_t launch_tiles(LinearArgs g, hipStream_t s) {
  auto kernel = tile_kernel<TT, kWFormat, kXFormat, kOut>;
  g.nW = (int)((g.m + TT::kTW - 1) / TT::kTW);
  g.nX = (int)((g.T + TT::kTX - 1) / TT::kTX);
  kernel<<<(unsigned)g.nW * (unsigned)g.nX, TT::kThreads, TT::kLds, s>>>(g);
  return hipGetLastError();
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
      LinearArgs g{W.codes, W.scales, xt, T, m, (int)blocks_up(n), (int)blocks_up(m),
                   (int)blocks_up(T), 0, 0, y};
      if (y_dtype == AF1_SRC_F32)
        return launch_tiles<Tile<128, 128, 2, 2, 4>, wf.value, xf.value, AF1_SRC_F32>(g, s);
      if (T <= 1024) return launch_tiles<Tile<128, 128, 2, 2, 4>, wf.value, xf.value, AF1_SRC_BF16>(g, s);
      return launch_tiles<Tile<256, 256, 2, 2, 4>, wf.value, xf.value, AF1_SRC_BF16>(g, s);
    });
  });
}

}  // namespace af1h
