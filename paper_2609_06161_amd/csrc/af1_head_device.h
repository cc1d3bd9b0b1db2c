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

// Eight elements, aligned as one: rows of odd length or stride start anywhere.
template <typename R>
struct __attribute__((packed, aligned(sizeof(R)))) Eight {
  R v[8];
};

template <typename D>
__device__ __forceinline__ Eight<typename D::raw> load_raw(const typename D::raw *row, int64_t c) {
  return *reinterpret_cast<const Eight<typename D::raw> *>(row + 8 * c);
}

template <typename D>
__device__ __forceinline__ void widen(const Eight<typename D::raw> &e, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = D::get(e.v[i]);
}

// Elements 8 c .. 8 c + 7 of a row of V; `fill` stands behind the end.
template <typename D>
__device__ __forceinline__ void load8(const typename D::raw *row, int64_t c, int64_t V, float fill,
                                      float (&x)[8]) {
  if (8 * c + 8 <= V) {
    widen<D>(load_raw<D>(row, c), x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 8 * c + i < V ? D::get(row[8 * c + i]) : fill;
  }
}

template <typename D>
__device__ __forceinline__ void store8(typename D::raw *row, int64_t c, int64_t V,
                                       const float (&x)[8]) {
  if (8 * c + 8 <= V) {
    Eight<typename D::raw> e;
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v[i] = D::put(x[i]);
    *reinterpret_cast<Eight<typename D::raw> *>(row + 8 * c) = e;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (8 * c + i < V) row[8 * c + i] = D::put(x[i]);
  }
}

}  // namespace af1h
