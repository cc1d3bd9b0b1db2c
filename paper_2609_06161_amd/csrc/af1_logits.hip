// What is read off a head's logits: log probabilities of given tokens with
// entropy and alternatives, and the KL divergence to a teacher, with their
// gradients (af1_head.h).
//
// Softmax statistics.  With c = scale * log2(e) and m the row's largest logit,
// t_j = (x_j - m) c <= 0 and
//   Z = sum 2^t_j,   W = sum 2^t_j t_j,
//   lse = scale m + ln Z,   entropy = ln Z - ln2 W / Z.
// A thread keeps a running (m, Z, W) of the logits it has seen: when m rises
// to m' both sums are multiplied by 2^((m - m') c), and W gains
// (m - m') c Z.  Partial triples join by the same rule.  The difference x - m
// is taken before the product with c, so that a row of the type's lowest
// values (a mask that is no infinity) neither overflows nor cancels.
#include <math.h>

#include "af1_device.h"
#include "af1_head_internal.h"

// Products and sums are fused only where it is written: a student equal to its
// teacher goes through the same roundings, so their divergence is exactly 0.
#pragma clang fp contract(off)

namespace af1h {
namespace {

using af1::bf16_to_f32;
using af1::f16_to_f32;
using af1::f32_to_bf16;
using af1::f32_to_f16;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_inff();

// Element types of logits.
struct F32 {
  using raw = float;
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
};
struct BF16 {
  using raw = uint16_t;
  static __device__ __forceinline__ float get(uint16_t v) { return bf16_to_f32(v); }
  static __device__ __forceinline__ uint16_t put(float v) { return f32_to_bf16(v); }
};
struct F16 {
  using raw = uint16_t;
  static __device__ __forceinline__ float get(uint16_t v) { return f16_to_f32(v); }
  static __device__ __forceinline__ uint16_t put(float v) { return f32_to_f16(v); }
};

// Eight elements, aligned as one: rows of odd length or stride start anywhere.
template <typename R>
struct __attribute__((packed, aligned(sizeof(R)))) Eight {
  R v[8];
};

// Elements 8 c .. 8 c + 7 of a row of V; `fill` stands behind the end.
template <typename D>
__device__ __forceinline__ void load8(const typename D::raw *row, int64_t c, int64_t V, float fill,
                                      float (&x)[8]) {
  if (8 * c + 8 <= V) {
    const Eight<typename D::raw> e =
        *reinterpret_cast<const Eight<typename D::raw> *>(row + 8 * c);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = D::get(e.v[i]);
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

__device__ __forceinline__ float exp2_hw(float t) { return __builtin_amdgcn_exp2f(t); }

// Running softmax statistics.  NaN logits leave m alone and make Z NaN, and so
// does +infinity (infinity less itself).
struct Stat {
  float m, Z, W;
};
__device__ __forceinline__ Stat no_logits() { return Stat{-kInf, 0.f, 0.f}; }

__device__ __forceinline__ void add8(Stat &s, const float (&x)[8], float c) {
  float m = s.m;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, x[i]);
  // nothing but masked entries so far: any finite base gives them 2^-inf = 0
  const float base = m == -kInf ? 0.f : m;
  const float step = s.m == -kInf ? 0.f : (s.m - base) * c;
  const float f = exp2_hw(step);
  // a step of -infinity empties both sums
  s.W = f == 0.f ? 0.f : f * fmaf(step, s.Z, s.W);
  s.Z *= f;
  s.m = m;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = (x[i] - base) * c;
    const float e = exp2_hw(t);
    s.Z += e;
    s.W = fmaf(e, fmaxf(t, -200.f), s.W);  // 2^-200 is 0 in fp32: masked entries add 0
  }
}

__device__ __forceinline__ Stat join(Stat a, Stat b, float c) {
  Stat r;
  r.m = fmaxf(a.m, b.m);
  const float base = r.m == -kInf ? 0.f : r.m;
  const float sa = a.m == -kInf ? 0.f : (a.m - base) * c, fa = exp2_hw(sa);
  const float sb = b.m == -kInf ? 0.f : (b.m - base) * c, fb = exp2_hw(sb);
  r.Z = fmaf(a.Z, fa, b.Z * fb);
  r.W = (fa == 0.f ? 0.f : fa * fmaf(sa, a.Z, a.W)) + (fb == 0.f ? 0.f : fb * fmaf(sb, b.Z, b.W));
  return r;
}

__device__ __forceinline__ Stat wave_join(Stat s, float c) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    Stat o;
    o.m = __shfl_xor(s.m, off, 64);
    o.Z = __shfl_xor(s.Z, off, 64);
    o.W = __shfl_xor(s.W, off, 64);
    s = join(s, o, c);
  }
  return s;
}

// The block's statistics, in every thread; sh holds one entry a wave.
template <int kThreads>
__device__ __forceinline__ Stat block_join(Stat s, float c, Stat *sh) {
  s = wave_join(s, c);
  if constexpr (kThreads > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
    __syncthreads();
    s = sh[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) s = join(s, sh[w], c);
  }
  return s;
}

// Order of alternatives: larger logit first, then the lower index, NaN before
// everything, -0 equal to +0.  A larger key comes first.
__device__ __forceinline__ uint64_t order_key(float x, int64_t index) {
  uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
  u = x != x ? 0xffffffffu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
  return (uint64_t)u << 32 | (uint32_t)~(uint32_t)index;
}
__device__ __forceinline__ uint32_t key_index(uint64_t key) { return ~(uint32_t)key; }

__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }

// What a row gives once its statistics are known.
struct RowOut {
  const int64_t *targets;
  float *logprob, *entropy, *lse, *saved;
  int k;
  float *top_logprob;
  int64_t *top_index;
  float scale;
};

__device__ __forceinline__ bool empty(const Stat &s) { return s.m == -kInf && s.Z == 0.f; }

__device__ __forceinline__ float log_prob(float x, const Stat &s, float lnZ, float scale) {
  return empty(s) ? -kInf : fmaf(x - s.m, scale, -lnZ);
}

template <typename D>
__device__ void write_row(const RowOut &o, const typename D::raw *row, int64_t r, int64_t V,
                          const Stat &s) {
  const float lnZ = logf(s.Z);
  const float H = empty(s) ? 0.f : lnZ - kLn2 * (s.W / s.Z);
  if (o.entropy) o.entropy[r] = H;
  if (o.lse) o.lse[r] = empty(s) ? -kInf : s.m * o.scale + lnZ;
  if (o.saved)
    reinterpret_cast<float4 *>(o.saved)[r] = make_float4(s.m, s.Z, H, log2f(s.Z));
  if (o.logprob) {
    const int64_t y = o.targets[r];
    o.logprob[r] = y < 0    ? 0.f
                   : y >= V ? __builtin_nanf("")
                            : log_prob(D::get(row[y]), s, lnZ, o.scale);
  }
}

template <typename D, int kThreads>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(const typename D::raw *z, int64_t V,
                                                            int64_t ld, float c, RowOut o) {
  __shared__ Stat sh[kThreads / 64];
  __shared__ uint64_t best[kThreads / 64];
  const int64_t r = blockIdx.x;
  const typename D::raw *row = z + r * ld;
  const int64_t chunks = (V + 7) / 8;
  Stat s = no_logits();
  for (int64_t i = threadIdx.x; i < chunks; i += kThreads) {
    float x[8];
    load8<D>(row, i, V, -kInf, x);
    add8(s, x, c);
  }
  s = block_join<kThreads>(s, c, sh);
  if (threadIdx.x == 0) write_row<D>(o, row, r, V, s);
  // the next alternative is the largest key below the last one
  uint64_t last = ~0ull;
  bool first = true;
  for (int j = 0; j < o.k; ++j) {
    uint64_t b = 0;
    bool have = false;
    for (int64_t i = threadIdx.x; i < V; i += kThreads) {
      const uint64_t key = order_key(D::get(row[i]), i);
      if ((first || key < last) && (!have || key > b)) b = key, have = true;
    }
    b = have ? b : 0;  // the lowest key of all belongs to no entry
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
      b = max64(b, (uint64_t)__shfl_xor((unsigned long long)b, off, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) best[threadIdx.x >> 6] = b;
    __syncthreads();
    b = best[0];
    for (int w = 1; w < kThreads / 64; ++w) b = max64(b, best[w]);
    if (threadIdx.x == 0) {
      const bool there = j < V;
      o.top_index[r * o.k + j] = there ? (int64_t)key_index(b) : -1;
      o.top_logprob[r * o.k + j] =
          there ? log_prob(D::get(row[key_index(b)]), s, logf(s.Z), o.scale) : -kInf;
    }
    last = b;
    first = false;
  }
}

template <typename D, int kThreads>
__global__ __launch_bounds__(kThreads) void logprobs_backward_kernel(
    const typename D::raw *z, int64_t V, int64_t ld, float scale, const int64_t *targets,
    const float *saved, const float *g_logprob, const float *g_entropy, typename D::raw *dz,
    int64_t ldd) {
  const int64_t r = blockIdx.x;
  const typename D::raw *row = z + r * ld;
  typename D::raw *out = dz + r * ldd;
  const float4 sv = reinterpret_cast<const float4 *>(saved)[r];
  const int64_t y = targets ? targets[r] : -1;
  float gl = g_logprob && y >= 0 ? g_logprob[r] * scale : 0.f;
  const float gh = g_entropy ? g_entropy[r] * scale : 0.f;
  const bool none = (gl == 0.f && gh == 0.f) || (sv.x == -kInf && sv.y == 0.f);
  if (y >= V && !none) gl = __builtin_nanf("");
  const float c = scale * kLog2e;
  for (int64_t i = threadIdx.x; i < (V + 7) / 8; i += kThreads) {
    float d[8];
    if (none) {
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] = 0.f;
    } else {
      float x[8];
      load8<D>(row, i, V, -kInf, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float t = fmaf(x[j] - sv.x, c, -sv.w);  // log2 of the probability
        const float p = exp2_hw(t);
        const float own = p == 0.f ? 0.f : p * fmaf(gh, fmaf(kLn2, t, sv.z), gl);
        d[j] = (8 * i + j == y ? gl : 0.f) - own;
      }
    }
    store8<D>(out, i, V, d);
  }
}

// p (exp(-u) - 1 + u), from u = ln p - ln q.  Near 0 by its series, which
// neither cancels nor depends on the rounding of q - p.
__device__ __forceinline__ float kl_term(float p, float q, float u) {
  if (p == 0.f) return q;
  if (fabsf(u) < 0.5f) {
    float h = fmaf(-u, 1.f / 40320, 1.f / 5040);
    h = fmaf(-u, h, 1.f / 720);
    h = fmaf(-u, h, 1.f / 120);
    h = fmaf(-u, h, 1.f / 24);
    h = fmaf(-u, h, 1.f / 6);
    h = fmaf(-u, h, 0.5f);
    return p * (u * u * h);
  }
  return fmaf(p, u, q - p);
}

template <typename D, int kThreads>
__global__ __launch_bounds__(kThreads) void distill_kl_kernel(
    const typename D::raw *zs, const typename D::raw *zt, int64_t V, int64_t ld_s, int64_t ld_t,
    float scale, const float *weight, float *kl, typename D::raw *ds, int64_t ldd) {
  __shared__ Stat sh[kThreads / 64];
  __shared__ float part[kThreads / 64];
  const int64_t r = blockIdx.x;
  const typename D::raw *s = zs + r * ld_s, *t = zt + r * ld_t;
  const float c = scale * kLog2e;
  const int64_t chunks = (V + 7) / 8;
  Stat a = no_logits(), b = no_logits();
  for (int64_t i = threadIdx.x; i < chunks; i += kThreads) {
    float x[8];
    load8<D>(s, i, V, -kInf, x);
    add8(a, x, c);
    load8<D>(t, i, V, -kInf, x);
    add8(b, x, c);
  }
  a = block_join<kThreads>(a, c, sh);
  b = block_join<kThreads>(b, c, sh);
  const float g = (weight ? weight[r] : 1.f) * scale;
  const bool none = empty(a) || empty(b);
  const bool zero = none || g == 0.f;
  const float la = log2f(a.Z), lb = log2f(b.Z);
  float sum = 0.f;
  for (int64_t i = threadIdx.x; i < chunks; i += kThreads) {
    float x[8], w[8], d[8];
    load8<D>(s, i, V, -kInf, x);
    load8<D>(t, i, V, -kInf, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float tq = fmaf(x[j] - a.m, c, -la), tp = fmaf(w[j] - b.m, c, -lb);
      const float q = exp2_hw(tq), p = exp2_hw(tp);
      sum += kl_term(p, q, kLn2 * (tp - tq));
      d[j] = zero ? 0.f : g * (q - p);
    }
    if (ds) store8<D>(ds + r * ldd, i, V, d);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 64; ++w) sum += part[w];
    if (none) {
      // teacher masked: nothing to match; student masked: no finite code
      const bool bad = !(a.Z == a.Z) || !(b.Z == b.Z);
      sum = bad ? __builtin_nanf("") : empty(b) ? 0.f : kInf;
    }
    kl[r] = sum;
  }
}

constexpr int kRowThreads = 256;

template <typename F>
auto with_type(int dtype, F &&f) {
  if (dtype == AF1_SRC_F32) return f(F32{});
  if (dtype == AF1_SRC_BF16) return f(BF16{});
  return f(F16{});
}

}  // namespace

size_t token_logprobs_workspace_bytes(int64_t, int64_t, int) { return 0; }

hipError_t launch_token_logprobs(const Rows &z, float scale, const int64_t *targets,
                                 float *logprob, float *entropy, float *lse, int k,
                                 float *top_logprob, int64_t *top_index, float *saved, void *,
                                 hipStream_t s) {
  const RowOut o{targets, logprob, entropy, lse, saved, k, top_logprob, top_index, scale};
  return with_type(z.dtype, [&](auto d) {
    using D = decltype(d);
    logprobs_kernel<D, kRowThreads><<<(unsigned)z.T, kRowThreads, 0, s>>>(
        static_cast<const typename D::raw *>(z.p), z.V, z.ld, scale * kLog2e, o);
    return hipGetLastError();
  });
}

hipError_t launch_token_logprobs_backward(const Rows &z, float scale, const int64_t *targets,
                                          const float *saved, const float *g_logprob,
                                          const float *g_entropy, void *dlogits, int64_t ldd,
                                          hipStream_t s) {
  return with_type(z.dtype, [&](auto d) {
    using D = decltype(d);
    logprobs_backward_kernel<D, kRowThreads><<<(unsigned)z.T, kRowThreads, 0, s>>>(
        static_cast<const typename D::raw *>(z.p), z.V, z.ld, scale, targets, saved, g_logprob,
        g_entropy, static_cast<typename D::raw *>(dlogits), ldd);
    return hipGetLastError();
  });
}

size_t distill_kl_workspace_bytes(int64_t, int64_t) { return 0; }

hipError_t launch_distill_kl(const Rows &z, const void *teacher, int64_t ld_t, float scale,
                             const float *weight, float *kl, void *dstudent, int64_t ldd, void *,
                             hipStream_t s) {
  return with_type(z.dtype, [&](auto d) {
    using D = decltype(d);
    distill_kl_kernel<D, kRowThreads><<<(unsigned)z.T, kRowThreads, 0, s>>>(
        static_cast<const typename D::raw *>(z.p), static_cast<const typename D::raw *>(teacher),
        z.V, z.ld, ld_t, scale, weight, kl, static_cast<typename D::raw *>(dstudent), ldd);
    return hipGetLastError();
  });
}

}  // namespace af1h
