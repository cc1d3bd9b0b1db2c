// Device-side helpers of the output head's kernels: dense element types and
// loads of eight elements that need an element's alignment only.
#pragma once
#include "af1_device.h"
#include "af1_head.h"

namespace af1h {

// Element types of dense arrays.
struct F32 {
  using raw = float;
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
};
struct BF16 {
  using raw = uint16_t;
  static __device__ __forceinline__ float get(uint16_t v) { return af1::bf16_to_f32(v); }
  static __device__ __forceinline__ uint16_t put(float v) { return af1::f32_to_bf16(v); }
};
struct F16 {
  using raw = uint16_t;
  static __device__ __forceinline__ float get(uint16_t v) { return af1::f16_to_f32(v); }
  static __device__ __forceinline__ uint16_t put(float v) { return af1::f32_to_f16(v); }
};

template <typename F>
auto with_type(int dtype, F &&f) {
  if (dtype == AF1_SRC_F32) return f(F32{});
  if (dtype == AF1_SRC_BF16) return f(BF16{});
  return f(F16{});
}

// Eight elements as they are stored, aligned as one: rows of odd length or
// stride start anywhere.  16-bit elements stay packed in four registers.
template <typename D>
struct __attribute__((packed, aligned(sizeof(typename D::raw)))) Eight {
  uint32_t w[2 * sizeof(typename D::raw)];
};

template <typename D>
__device__ __forceinline__ Eight<D> load_raw(const typename D::raw *row, int64_t c) {
  return *reinterpret_cast<const Eight<D> *>(row + 8 * c);
}

// The elements i of 0 .. 7 for which in(i), others `fill`.
template <typename D, typename F>
__device__ __forceinline__ Eight<D> load_some(const typename D::raw *p, F &&in, float fill) {
  Eight<D> e;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(e) / 4); ++i) {
    if constexpr (sizeof(typename D::raw) == 4) {
      e.w[i] = __float_as_uint(in(i) ? p[i] : fill);
    } else {
      const uint32_t lo = in(2 * i) ? p[2 * i] : D::put(fill);
      const uint32_t hi = in(2 * i + 1) ? p[2 * i + 1] : D::put(fill);
      e.w[i] = lo | hi << 16;
    }
  }
  return e;
}

template <typename D>
__device__ __forceinline__ void widen(const Eight<D> &e, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (sizeof(typename D::raw) == 4)
      x[i] = __uint_as_float(e.w[i]);
    else
      x[i] = D::get((uint16_t)(e.w[i >> 1] >> (16 * (i & 1))));
  }
}

// Elements 8 c .. 8 c + 7 of a row of V; `fill` stands behind the end.
template <typename D>
__device__ __forceinline__ Eight<D> load_raw_to(const typename D::raw *row, int64_t c, int64_t V,
                                                float fill) {
  if (8 * c + 8 <= V) return load_raw<D>(row, c);
  return load_some<D>(row + 8 * c, [&](int i) { return 8 * c + i < V; }, fill);
}

template <typename D>
__device__ __forceinline__ void load8(const typename D::raw *row, int64_t c, int64_t V, float fill,
                                      float (&x)[8]) {
  widen<D>(load_raw_to<D>(row, c, V, fill), x);
}

// kPast: past the caches.
template <typename D, bool kPast = false>
__device__ __forceinline__ void store8(typename D::raw *row, int64_t c, int64_t V,
                                       const float (&x)[8]) {
  if (8 * c + 8 <= V) {
    Eight<D> e;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(e) / 4); ++i) {
      if constexpr (sizeof(typename D::raw) == 4)
        e.w[i] = __float_as_uint(x[i]);
      else
        e.w[i] = (uint32_t)D::put(x[2 * i]) | (uint32_t)D::put(x[2 * i + 1]) << 16;
    }
    if constexpr (kPast) {
      // an element's alignment at most
      typedef uint32_t raw4 __attribute__((ext_vector_type(4), aligned(2)));
#pragma unroll
      for (int i = 0; i < (int)(sizeof(e) / 16); ++i)
        __builtin_nontemporal_store(raw4{e.w[4 * i], e.w[4 * i + 1], e.w[4 * i + 2], e.w[4 * i + 3]},
                                    reinterpret_cast<raw4 *>(row + 8 * c) + i);
    } else {
      *reinterpret_cast<Eight<D> *>(row + 8 * c) = e;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (8 * c + i < V) row[8 * c + i] = D::put(x[i]);
  }
}

}  // namespace af1h
