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
//
// Work is cut into parts of a row (plan_parts): whole rows when there are
// enough of them to fill the device, parts of at least 2048 logits when there
// are few, whose statistics a second launch joins in the parts' order.
#include <math.h>

#include "af1_head_device.h"
#include "af1_head_internal.h"

// Products and sums are fused only where it is written: a student equal to its
// teacher goes through the same roundings, so their divergence is exactly 0.
#pragma clang fp contract(off)

namespace af1h {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ float exp2_hw(float t) { return __builtin_amdgcn_exp2f(t); }

// Running softmax statistics.  NaN logits leave m alone and make Z NaN, and so
// does +infinity (infinity less itself).
struct Stat {
  float m, Z, W;
};
__device__ __forceinline__ Stat no_logits() { return Stat{-kInf, 0.f, 0.f}; }

template <int kN>
__device__ __forceinline__ void add(Stat &s, const float (&x)[kN], float c) {
  float m = s.m;
#pragma unroll
  for (int i = 0; i < kN; ++i) m = fmaxf(m, x[i]);
  // nothing but masked entries so far: any finite base gives them 2^-inf = 0
  const float base = m == -kInf ? 0.f : m;
  const float step = s.m == -kInf ? 0.f : (s.m - base) * c;
  const float f = exp2_hw(step);
  // a step of -infinity empties both sums
  s.W = f == 0.f ? 0.f : f * fmaf(step, s.Z, s.W);
  s.Z *= f;
  s.m = m;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
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
template <int kN>
__device__ __forceinline__ Stat block_join(Stat s, float c, Stat *sh) {
  s = wave_join(s, c);
  if constexpr (kN > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
    __syncthreads();
    s = sh[0];
#pragma unroll
    for (int w = 1; w < kN / 64; ++w) s = join(s, sh[w], c);
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

constexpr int kThreads = 256;  // of every kernel here
constexpr int kWaves = kThreads / 64;

// A row's parts: `size` chunks of eight logits each (the last may be short).
struct Parts {
  int count;
  int64_t size;
};

// The chunks of one part; calls f(chunk, x) for each of this thread's, whose
// chunks lie kThreads apart, four loads in flight.
template <typename D, typename F>
__device__ __forceinline__ void each_chunk(const typename D::raw *row, int64_t c0, int64_t c1,
                                           int64_t V, F &&f) {
  constexpr int kAhead = 4;
  const int64_t whole = min(c1, V / 8);
  int64_t i = c0 + threadIdx.x;
  for (; i + (kAhead - 1) * kThreads < whole; i += kAhead * kThreads) {
    Eight<typename D::raw> e[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) e[a] = load_raw<D>(row, i + a * kThreads);
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      float x[8];
      widen<D>(e[a], x);
      f(i + a * kThreads, x);
    }
  }
  for (; i < c1; i += kThreads) {
    float x[8];
    load8<D>(row, i, V, -kInf, x);
    f(i, x);
  }
}

// ---------------------------------------------------------------------------
// Alternatives.  Every thread remembers the first of its chunks that holds its
// largest logit.  The k-th best of the threads' keys bounds the k-th best
// logit from below, and only the threads at or above it, at most k, can hold
// one of the best: their chunks are read again (from the caches), what reaches
// the bound is collected and sorted.  Keys are distinct, so equal logits need
// no special case.
// ---------------------------------------------------------------------------

constexpr int kMaxFound = 512;  // collected logits; beyond it, one at a time

struct TopLds {
  uint64_t sorted[kWaves][64];
  uint64_t found[kMaxFound];
  uint64_t bound;
  int holders[AF1_HEAD_MAX_TOP];
  int n_holders, n_found;
};

__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int mask) {
  return (uint64_t)__shfl_xor((unsigned long long)v, mask, 64);
}

__device__ __forceinline__ uint64_t exchange(uint64_t v, int mask, bool larger) {
  const uint64_t o = shfl_xor64(v, mask);
  return (v > o) == larger ? v : o;
}

// Keys of a wave, the largest in lane 0 (bitonic).
__device__ __forceinline__ uint64_t sort64(uint64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 2; k <= 64; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1)
      v = exchange(v, j, ((lane & j) == 0) == ((lane & k) == 0));
  return v;
}

// The largest 64 of two sorted lists, sorted.
__device__ __forceinline__ uint64_t merge64(uint64_t a, const uint64_t *b) {
  const int lane = threadIdx.x & 63;
  uint64_t v = max64(a, b[63 - lane]);
#pragma unroll
  for (int j = 32; j > 0; j >>= 1) v = exchange(v, j, (lane & j) == 0);
  return v;
}

// In wave 0, lane i gets the i-th largest (i < 64) of the block's keys; the
// other waves' value means nothing.
__device__ __forceinline__ uint64_t block_sort(uint64_t v, TopLds &l) {
  const int wave = threadIdx.x >> 6;
  v = sort64(v);
  l.sorted[wave][threadIdx.x & 63] = v;
  __syncthreads();
  if (wave == 0)
    for (int w = 1; w < kWaves; ++w) v = merge64(v, l.sorted[w]);
  return v;
}

// In wave 0, lane i gets the i-th largest of the n collected keys.
__device__ __forceinline__ uint64_t sort_found(const TopLds &l, uint64_t *scratch) {
  const int lane = threadIdx.x & 63, n = l.n_found;
  uint64_t v = sort64(lane < n ? l.found[lane] : 0);
  for (int at = 64; at < n; at += 64) {
    scratch[lane] = sort64(at + lane < n ? l.found[at + lane] : 0);
    __builtin_amdgcn_wave_barrier();
    v = merge64(v, scratch);
    __builtin_amdgcn_wave_barrier();
  }
  return v;
}

__device__ __forceinline__ void collect(TopLds &l, uint64_t key) {
  if (key < l.bound || key == 0) return;
  const int at = atomicAdd(&l.n_found, 1);  // the order in the list does not matter
  if (at < kMaxFound) l.found[at] = key;
}

// The k largest of `next(after)`, the block's largest key below `after` (0:
// none left); in wave 0, lane i gets the i-th.
template <typename F>
__device__ __forceinline__ uint64_t one_by_one(int k, TopLds &l, F &&next) {
  uint64_t mine = 0, last = ~0ull;
  for (int j = 0; j < k && last; ++j) {
    uint64_t b = next(last);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) b = max64(b, shfl_xor64(b, off));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) l.sorted[0][threadIdx.x >> 6] = b;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) b = max64(b, l.sorted[0][w]);
    if ((int)threadIdx.x == j) mine = b;
    last = b;
  }
  return mine;
}

// In wave 0, lane i gets the i-th largest key of the chunks c0 .. c1 - 1 (i <
// k).  best, chunk: this thread's largest logit and the first chunk with it
// (chunk < 0: the thread has none).
template <typename D>
__device__ uint64_t part_top(const typename D::raw *row, int64_t c0, int64_t c1, int64_t V, int k,
                             float best, int64_t chunk, TopLds &l) {
  const uint64_t mine = chunk < 0 ? 0 : order_key(best, 8 * chunk + 7);
  uint64_t v = block_sort(mine, l);
  if (threadIdx.x == (unsigned)(k - 1)) l.bound = v;
  if (threadIdx.x == 0) l.n_holders = l.n_found = 0;
  __syncthreads();
  if (mine != 0 && mine >= l.bound) l.holders[atomicAdd(&l.n_holders, 1)] = threadIdx.x;
  __syncthreads();
  const int64_t each = (c1 - c0 + kThreads - 1) / kThreads;
  for (int64_t i = threadIdx.x; i < l.n_holders * each; i += kThreads) {
    const int64_t c = c0 + l.holders[i / each] + i % each * kThreads;
    if (c >= c1) continue;
    float x[8];
    load8<D>(row, c, V, -kInf, x);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (8 * c + e < V) collect(l, order_key(x[e], 8 * c + e));
  }
  __syncthreads();
  if (l.n_found > kMaxFound)
    return one_by_one(k, l, [&](uint64_t after) {
      uint64_t b = 0;
      for (int64_t i = 8 * c0 + threadIdx.x; i < min(8 * c1, V); i += kThreads) {
        const uint64_t key = order_key(D::get(row[i]), i);
        if (key < after) b = max64(b, key);
      }
      return b;
    });
  return threadIdx.x < 64 ? sort_found(l, l.sorted[1]) : 0;
}

template <typename D>
__device__ __forceinline__ void write_top(const RowOut &o, const typename D::raw *row, int64_t r,
                                          const Stat &s, uint64_t key) {
  if ((int)threadIdx.x >= o.k) return;
  const bool there = key != 0;
  o.top_index[r * o.k + threadIdx.x] = there ? (int64_t)key_index(key) : -1;
  o.top_logprob[r * o.k + threadIdx.x] =
      there ? log_prob(D::get(row[key_index(key)]), s, logf(s.Z), o.scale) : -kInf;
}

// What the parts of a row leave for the launch that joins them.
struct PartOut {
  Stat *stats;     // [T, parts]
  uint64_t *keys;  // [T, parts, k], sorted
};

template <typename D, bool kTop>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(const typename D::raw *z, int64_t V,
                                                            int64_t ld, float c, Parts parts,
                                                            PartOut po, RowOut o) {
  __shared__ Stat sh[kWaves];
  __shared__ TopLds top;
  const int64_t r = blockIdx.x / parts.count;
  const int part = blockIdx.x % parts.count;
  const typename D::raw *row = z + r * ld;
  const int64_t c0 = part * parts.size, c1 = min(c0 + parts.size, (V + 7) / 8);
  Stat s = no_logits();
  float best = -kInf;
  int64_t chunk = -1;
  each_chunk<D>(row, c0, c1, V, [&](int64_t i, const float(&x)[8]) {
    if constexpr (kTop) {
      float m = x[0];
      bool nan = x[0] != x[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) m = fmaxf(m, x[e]), nan |= x[e] != x[e];
      if (nan) m = __builtin_nanf("");
      // NaN comes first
      if (chunk < 0 || m > best || (m != m && best == best)) best = m, chunk = i;
    }
    add(s, x, c);
  });
  s = block_join<kThreads>(s, c, sh);
  uint64_t key = 0;
  if constexpr (kTop) key = part_top<D>(row, c0, c1, V, o.k, best, chunk, top);
  if (parts.count == 1) {
    if (threadIdx.x == 0) write_row<D>(o, row, r, V, s);
    if constexpr (kTop) write_top<D>(o, row, r, s, key);
  } else {
    if (threadIdx.x == 0) po.stats[blockIdx.x] = s;
    if (kTop && (int)threadIdx.x < o.k) po.keys[(int64_t)blockIdx.x * o.k + threadIdx.x] = key;
  }
}

// Statistics of a row's parts (at most 64), joined in a fixed order; called by
// a whole wave.
__device__ __forceinline__ Stat join_parts(const Stat *stats, int parts, float c) {
  const int lane = threadIdx.x & 63;
  return wave_join(lane < parts ? stats[lane] : no_logits(), c);
}

// One block a row.  The parts' best keys bound the k-th best from below.
template <typename D, bool kTop>
__global__ __launch_bounds__(kThreads) void logprobs_join_kernel(const typename D::raw *z,
                                                                 int64_t V, int64_t ld, float c,
                                                                 int parts, PartOut po, RowOut o) {
  __shared__ TopLds l;
  const int64_t r = blockIdx.x;
  const typename D::raw *row = z + r * ld;
  const Stat s = join_parts(po.stats + r * parts, parts, c);
  if (threadIdx.x == 0) write_row<D>(o, row, r, V, s);
  if constexpr (kTop) {
    const uint64_t *keys = po.keys + r * parts * o.k;
    if (threadIdx.x < 64) {
      const uint64_t v = sort64((int)threadIdx.x < parts ? keys[threadIdx.x * o.k] : 0);
      // the list of a part with fewer than k logits ends in zeros
      if ((int)threadIdx.x == o.k - 1) l.bound = v;
      if (threadIdx.x == 0) l.n_found = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < parts * o.k; i += kThreads) collect(l, keys[i]);
    __syncthreads();
    uint64_t key;
    if (l.n_found > kMaxFound)
      key = one_by_one(o.k, l, [&](uint64_t after) {
        uint64_t b = 0;
        for (int i = threadIdx.x; i < parts * o.k; i += kThreads)
          if (keys[i] < after) b = max64(b, keys[i]);
        return b;
      });
    else
      key = threadIdx.x < 64 ? sort_found(l, l.sorted[1]) : 0;
    write_top<D>(o, row, r, s, key);
  }
}

template <typename D>
__global__ __launch_bounds__(kThreads) void logprobs_backward_kernel(
    const typename D::raw *z, int64_t V, int64_t ld, float scale, Parts parts,
    const int64_t *targets, const float *saved, const float *g_logprob, const float *g_entropy,
    typename D::raw *dz, int64_t ldd) {
  const int64_t r = blockIdx.x / parts.count;
  const int64_t c0 = blockIdx.x % parts.count * parts.size;
  const int64_t c1 = min(c0 + parts.size, (V + 7) / 8);
  typename D::raw *out = dz + r * ldd;
  const float4 sv = reinterpret_cast<const float4 *>(saved)[r];
  const int64_t y = targets ? targets[r] : -1;
  float gl = g_logprob && y >= 0 ? g_logprob[r] * scale : 0.f;
  const float gh = g_entropy ? g_entropy[r] * scale : 0.f;
  if ((gl == 0.f && gh == 0.f) || (sv.x == -kInf && sv.y == 0.f)) {
    const float none[8] = {};
    for (int64_t i = c0 + threadIdx.x; i < c1; i += kThreads) store8<D>(out, i, V, none);
    return;
  }
  if (y >= V) gl = __builtin_nanf("");
  const float c = scale * kLog2e;
  each_chunk<D>(z + r * ld, c0, c1, V, [&](int64_t i, const float(&x)[8]) {
    float d[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float t = fmaf(x[j] - sv.x, c, -sv.w);  // log2 of the probability
      const float p = exp2_hw(t);
      d[j] = p == 0.f ? 0.f : -p * fmaf(gh, fmaf(kLn2, t, sv.z), gl);
    }
    if (y >= 8 * i && y < 8 * i + 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (8 * i + j == y) d[j] += gl;
    }
    store8<D>(out, i, V, d);
  });
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

// Both rows' statistics and what the second pass needs of them.
struct KlRow {
  float ms, ls, mt, lt;  // largest logit and log2 Z of the student and the teacher
  float g;               // the gradient's factor
  bool none, bad;        // a row that masks everything; NaN
  float instead;         // kl where none
};

__device__ __forceinline__ KlRow kl_row(const Stat &a, const Stat &b, float g) {
  KlRow k{a.m, log2f(a.Z), b.m, log2f(b.Z), g, empty(a) || empty(b), false, 0.f};
  // teacher masked: nothing to match; student masked: no finite code for it
  if (k.none)
    k.instead = a.Z != a.Z || b.Z != b.Z ? __builtin_nanf("") : empty(b) ? 0.f : kInf;
  return k;
}

// The chunks of both rows, two loads of each in flight.
template <typename D, typename F>
__device__ __forceinline__ void each_pair(const typename D::raw *s, const typename D::raw *t,
                                          int64_t c0, int64_t c1, int64_t V, F &&f) {
  constexpr int kAhead = 2;
  const int64_t whole = min(c1, V / 8);
  int64_t i = c0 + threadIdx.x;
  for (; i + (kAhead - 1) * kThreads < whole; i += kAhead * kThreads) {
    Eight<typename D::raw> a[kAhead], b[kAhead];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      a[q] = load_raw<D>(s, i + q * kThreads);
      b[q] = load_raw<D>(t, i + q * kThreads);
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      float x[8], w[8];
      widen<D>(a[q], x);
      widen<D>(b[q], w);
      f(i + q * kThreads, x, w);
    }
  }
  for (; i < c1; i += kThreads) {
    float x[8], w[8];
    load8<D>(s, i, V, -kInf, x);
    load8<D>(t, i, V, -kInf, w);
    f(i, x, w);
  }
}

struct KlArgs {
  int64_t V, ld_s, ld_t, ldd;
  float scale;
  const float *weight;
  float *kl;
  Parts parts;
  Stat *stats;      // [2, T, parts]: the student's, then the teacher's
  float *sums;      // [T, parts]
};

// One part of the second pass: gradient written, the terms' sum returned (in
// every thread).
template <typename D>
__device__ float kl_part(const KlRow &k, const typename D::raw *s, const typename D::raw *t,
                         typename D::raw *ds, int64_t c0, int64_t c1, const KlArgs &g, float *sh) {
  const float c = g.scale * kLog2e;
  const bool zero = k.none || k.g == 0.f;
  float sum = 0.f;
  each_pair<D>(s, t, c0, c1, g.V, [&](int64_t i, const float(&x)[8], const float(&w)[8]) {
    float d[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float tq = fmaf(x[j] - k.ms, c, -k.ls), tp = fmaf(w[j] - k.mt, c, -k.lt);
      const float q = exp2_hw(tq), p = exp2_hw(tp);
      sum += kl_term(p, q, kLn2 * (tp - tq));
      d[j] = zero ? 0.f : k.g * (q - p);
    }
    if (ds) store8<D>(ds, i, g.V, d);
  });
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = sum;
  __syncthreads();
  sum = sh[0];
  for (int w = 1; w < kWaves; ++w) sum += sh[w];
  return sum;
}

template <typename D>
__device__ __forceinline__ void pair_stats(const typename D::raw *s, const typename D::raw *t,
                                           int64_t c0, int64_t c1, int64_t V, float c, Stat *sh,
                                           Stat &a, Stat &b) {
  a = b = no_logits();
  each_pair<D>(s, t, c0, c1, V, [&](int64_t, const float(&x)[8], const float(&w)[8]) {
    add(a, x, c);
    add(b, w, c);
  });
  a = block_join<kThreads>(a, c, sh);
  b = block_join<kThreads>(b, c, sh);
}

// A row a block, both passes: the second finds the row in the caches.
template <typename D>
__global__ __launch_bounds__(kThreads) void kl_rows_kernel(const typename D::raw *zs,
                                                           const typename D::raw *zt,
                                                           typename D::raw *ds, KlArgs g) {
  __shared__ Stat sh[kWaves];
  __shared__ float part[kWaves];
  const int64_t r = blockIdx.x, chunks = (g.V + 7) / 8;
  const typename D::raw *s = zs + r * g.ld_s, *t = zt + r * g.ld_t;
  Stat a, b;
  pair_stats<D>(s, t, 0, chunks, g.V, g.scale * kLog2e, sh, a, b);
  const KlRow k = kl_row(a, b, (g.weight ? g.weight[r] : 1.f) * g.scale);
  const float sum = kl_part<D>(k, s, t, ds ? ds + r * g.ldd : nullptr, 0, chunks, g, part);
  if (threadIdx.x == 0) g.kl[r] = k.none ? k.instead : sum;
}

// The same in parts: statistics, then terms and gradient, then the terms' sum.
template <typename D>
__global__ __launch_bounds__(kThreads) void kl_stats_kernel(const typename D::raw *zs,
                                                            const typename D::raw *zt, int64_t T,
                                                            KlArgs g) {
  __shared__ Stat sh[kWaves];
  const int64_t r = blockIdx.x / g.parts.count;
  const int64_t c0 = blockIdx.x % g.parts.count * g.parts.size;
  Stat a, b;
  pair_stats<D>(zs + r * g.ld_s, zt + r * g.ld_t, c0, min(c0 + g.parts.size, (g.V + 7) / 8), g.V,
                g.scale * kLog2e, sh, a, b);
  if (threadIdx.x == 0) {
    g.stats[blockIdx.x] = a;
    g.stats[T * g.parts.count + blockIdx.x] = b;
  }
}

__device__ __forceinline__ KlRow kl_join(int64_t r, int64_t T, const KlArgs &g) {
  const Stat *st = g.stats + r * g.parts.count;
  const float c = g.scale * kLog2e;
  const Stat a = join_parts(st, g.parts.count, c);
  const Stat b = join_parts(st + T * g.parts.count, g.parts.count, c);
  return kl_row(a, b, (g.weight ? g.weight[r] : 1.f) * g.scale);
}

template <typename D>
__global__ __launch_bounds__(kThreads) void kl_parts_kernel(const typename D::raw *zs,
                                                            const typename D::raw *zt,
                                                            typename D::raw *ds, int64_t T,
                                                            KlArgs g) {
  __shared__ float part[kWaves];
  const int64_t r = blockIdx.x / g.parts.count;
  const int64_t c0 = blockIdx.x % g.parts.count * g.parts.size;
  const float sum = kl_part<D>(kl_join(r, T, g), zs + r * g.ld_s, zt + r * g.ld_t,
                               ds ? ds + r * g.ldd : nullptr, c0,
                               min(c0 + g.parts.size, (g.V + 7) / 8), g, part);
  if (threadIdx.x == 0) g.sums[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kThreads) void kl_sum_kernel(int64_t T, KlArgs g) {
  const int64_t r = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (r >= T) return;
  const int lane = threadIdx.x & 63;
  float sum = lane < g.parts.count ? g.sums[r * g.parts.count + lane] : 0.f;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
  const KlRow k = kl_join(r, T, g);
  if (lane == 0) g.kl[r] = k.none ? k.instead : sum;
}

// Parts of a row for T rows: as many as give the device kWant blocks, of at
// least one chunk a thread, at most one for each lane of the joining wave.
constexpr int64_t kWant = 2048;

Parts plan_parts(int64_t T, int64_t V, int most) {
  const int64_t chunks = (V + 7) / 8;
  int64_t n = T >= kWant / 2 ? 1 : (kWant + T - 1) / T;
  const int64_t fit = (chunks + kThreads - 1) / kThreads;
  n = n < fit ? n : fit;
  n = n < most ? n : most;
  const int64_t size = ((chunks + n - 1) / n + kThreads - 1) / kThreads * kThreads;
  return Parts{(int)((chunks + size - 1) / size), size};
}
constexpr int kMaxParts = 64;

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

}  // namespace

size_t token_logprobs_workspace_bytes(int64_t T, int64_t V, int k) {
  const Parts p = plan_parts(T, V, kMaxParts);
  if (p.count == 1) return 0;
  return up16((size_t)T * p.count * sizeof(Stat)) + (size_t)T * p.count * k * 8;
}

hipError_t launch_token_logprobs(const Rows &z, float scale, const int64_t *targets,
                                 float *logprob, float *entropy, float *lse, int k,
                                 float *top_logprob, int64_t *top_index, float *saved, void *ws,
                                 hipStream_t s) {
  const RowOut o{targets, logprob, entropy, lse, saved, k, top_logprob, top_index, scale};
  const Parts p = plan_parts(z.T, z.V, kMaxParts);
  const PartOut po{static_cast<Stat *>(ws),
                   reinterpret_cast<uint64_t *>(static_cast<uint8_t *>(ws) +
                                                up16((size_t)z.T * p.count * sizeof(Stat)))};
  const float c = scale * kLog2e;
  return with_type(z.dtype, [&](auto d) {
    using D = decltype(d);
    const auto *in = static_cast<const typename D::raw *>(z.p);
    const unsigned blocks = (unsigned)(z.T * p.count);
    if (k > 0)
      logprobs_kernel<D, true><<<blocks, kThreads, 0, s>>>(in, z.V, z.ld, c, p, po, o);
    else
      logprobs_kernel<D, false><<<blocks, kThreads, 0, s>>>(in, z.V, z.ld, c, p, po, o);
    if (p.count > 1) {
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      if (k > 0)
        logprobs_join_kernel<D, true>
            <<<(unsigned)z.T, kThreads, 0, s>>>(in, z.V, z.ld, c, p.count, po, o);
      else
        logprobs_join_kernel<D, false>
            <<<(unsigned)z.T, 64, 0, s>>>(in, z.V, z.ld, c, p.count, po, o);
    }
    return hipGetLastError();
  });
}

hipError_t launch_token_logprobs_backward(const Rows &z, float scale, const int64_t *targets,
                                          const float *saved, const float *g_logprob,
                                          const float *g_entropy, void *dlogits, int64_t ldd,
                                          hipStream_t s) {
  const Parts p = plan_parts(z.T, z.V, 1 << 12);
  return with_type(z.dtype, [&](auto d) {
    using D = decltype(d);
    logprobs_backward_kernel<D><<<(unsigned)(z.T * p.count), kThreads, 0, s>>>(
        static_cast<const typename D::raw *>(z.p), z.V, z.ld, scale, p, targets, saved, g_logprob,
        g_entropy, static_cast<typename D::raw *>(dlogits), ldd);
    return hipGetLastError();
  });
}

size_t distill_kl_workspace_bytes(int64_t T, int64_t V) {
  const Parts p = plan_parts(T, V, kMaxParts);
  return p.count == 1 ? 0 : up16((size_t)2 * T * p.count * sizeof(Stat)) + (size_t)T * p.count * 4;
}

hipError_t launch_distill_kl(const Rows &z, const void *teacher, int64_t ld_t, float scale,
                             const float *weight, float *kl, void *dstudent, int64_t ldd, void *ws,
                             hipStream_t s) {
  const Parts p = plan_parts(z.T, z.V, kMaxParts);
  const KlArgs g{z.V, z.ld, ld_t, ldd, scale, weight, kl, p, static_cast<Stat *>(ws),
                 reinterpret_cast<float *>(static_cast<uint8_t *>(ws) +
                                           up16((size_t)2 * z.T * p.count * sizeof(Stat)))};
  return with_type(z.dtype, [&](auto d) {
    using D = decltype(d);
    const auto *a = static_cast<const typename D::raw *>(z.p);
    const auto *b = static_cast<const typename D::raw *>(teacher);
    auto *out = static_cast<typename D::raw *>(dstudent);
    if (p.count == 1) {
      kl_rows_kernel<D><<<(unsigned)z.T, kThreads, 0, s>>>(a, b, out, g);
      return hipGetLastError();
    }
    const unsigned blocks = (unsigned)(z.T * p.count);
    kl_stats_kernel<D><<<blocks, kThreads, 0, s>>>(a, b, z.T, g);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    kl_parts_kernel<D><<<blocks, kThreads, 0, s>>>(a, b, out, z.T, g);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    kl_sum_kernel<<<(unsigned)((z.T + kWaves - 1) / kWaves), kThreads, 0, s>>>(z.T, g);
    return hipGetLastError();
  });
}

}  // namespace af1h
