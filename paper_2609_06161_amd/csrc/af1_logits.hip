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
// Work is cut into parts of a row: whole rows when there are enough of them to
// fill the device, parts of at least 2048 logits when there are few.  Parts'
// results are joined in the parts' order.
//
// All of it is bound by memory where there are rows enough.  Log probabilities of
// 1500 rows of 50257 bf16: 29.6 us, the rate of a copy; with 5 alternatives 35.5,
// with 20 39.6: the selection comes at the end of rows that are all resident at
// once, so none hides another's.  One row of 128256 fp32 with 20: 11 us in two
// launches (one workgroup and a search for every
// alternative: 1672).  2048 rows of 32000 bf16: 26 us.
//
// Gradients are stored past the caches, which then still hold the logits of the
// forward: forward and backward of 2048 rows of 32000 bf16 76 us, stored plainly
// 89; 2048 rows of 128256 bf16 of the KL 321 and 328.  The product that reads the
// gradient next is not slower for it (45 to 2048 rows, 32000 to 128256 wide).
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

// One value a lane combined over the 64 lanes in a fixed order, in every lane:
// four DPP steps within rows of 16, then the four rows.
template <int kCtrl>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kCtrl, 0xF, 0xF, false));
}
template <typename Op>
__device__ __forceinline__ float wave_all(float v, Op op) {
  v = op(v, dpp<0xB1>(v));   // lane ^ 1
  v = op(v, dpp<0x4E>(v));   // lane ^ 2
  v = op(v, dpp<0x124>(v));  // row rotated by 4
  v = op(v, dpp<0x128>(v));  // and by 8
  const int i = __float_as_int(v);
  const float r0 = __int_as_float(__builtin_amdgcn_readlane(i, 0));
  const float r1 = __int_as_float(__builtin_amdgcn_readlane(i, 16));
  const float r2 = __int_as_float(__builtin_amdgcn_readlane(i, 32));
  const float r3 = __int_as_float(__builtin_amdgcn_readlane(i, 48));
  return op(op(r0, r1), op(r2, r3));
}
__device__ __forceinline__ float wave_add(float v) {
  return wave_all(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_all(v, [](float a, float b) { return fmaxf(a, b); });
}

__device__ __forceinline__ float max8(const float (&x)[8]) {
  return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
               fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
}

// Running softmax statistics (W where kEntropy).  NaN logits leave m alone and
// make Z NaN, and so does +infinity (infinity less itself).
struct Stat {
  float m, Z, W;
};
__device__ __forceinline__ Stat no_logits() { return Stat{-kInf, 0.f, 0.f}; }

// The statistics about `m`, at least s.m.
template <bool kEntropy>
__device__ __forceinline__ void rebase(Stat &s, float m, float c) {
  // nothing but masked entries so far: any finite base gives them 2^-inf = 0
  const float step = s.m == -kInf ? 0.f : (s.m - m) * c;
  const float f = exp2_hw(step);
  // a step of -infinity empties both sums
  if constexpr (kEntropy) s.W = f == 0.f ? 0.f : f * fmaf(step, s.Z, s.W);
  s.Z *= f;
  s.m = m;
}

// kN times eight logits, the largest of which is `top`.
template <bool kEntropy, int kN>
__device__ __forceinline__ void add(Stat &s, const float (&x)[kN][8], float top, float c) {
  rebase<kEntropy>(s, fmaxf(s.m, top), c);
  const float base = s.m == -kInf ? 0.f : s.m;
#pragma unroll
  for (int n = 0; n < kN; ++n)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = (x[n][i] - base) * c;
      const float e = exp2_hw(t);
      s.Z += e;
      // 2^-200 is 0 in fp32: masked entries add 0
      if constexpr (kEntropy) s.W = fmaf(e, fmaxf(t, -200.f), s.W);
    }
}

template <bool kEntropy>
__device__ __forceinline__ Stat wave_join(Stat s, float c) {
  rebase<kEntropy>(s, wave_max(s.m), c);
  s.Z = wave_add(s.Z);
  if constexpr (kEntropy) s.W = wave_add(s.W);
  return s;
}

// The statistics (without entropy) of two sets of logits together.
__device__ __forceinline__ Stat join2(Stat a, Stat b, float c) {
  const float m = fmaxf(a.m, b.m);
  rebase<false>(a, m, c);
  rebase<false>(b, m, c);
  return Stat{m, a.Z + b.Z, 0.f};
}

constexpr int kThreads = 256;  // of every kernel here
constexpr int kWaves = kThreads / 64;

// The block's statistics, in every thread; sh holds one entry a wave.
template <bool kEntropy>
__device__ __forceinline__ Stat block_join(Stat s, float c, Stat *sh) {
  s = wave_join<kEntropy>(s, c);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  Stat w[kWaves];
  float m = -kInf;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) w[i] = sh[i], m = fmaxf(m, w[i].m);
  s = Stat{m, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    rebase<kEntropy>(w[i], m, c);
    s.Z += w[i].Z;
    s.W += w[i].W;
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
// The logit itself (0 for -0).
__device__ __forceinline__ float key_logit(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

template <int kV>
struct Int {
  static constexpr int value = kV;
};

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

// A row's target and its logit, read before the statistics are there.
struct Target {
  int64_t index = -1;
  float logit = 0.f;
};
template <typename D>
__device__ __forceinline__ Target target_of(const RowOut &o, const typename D::raw *row, int64_t r,
                                            int64_t V) {
  Target t;
  if (o.logprob && threadIdx.x == 0) {
    t.index = o.targets[r];
    if (t.index >= 0 && t.index < V) t.logit = D::get(row[t.index]);
  }
  return t;
}

__device__ void write_row(const RowOut &o, const Target &t, int64_t r, int64_t V, const Stat &s) {
  const float lnZ = logf(s.Z);
  const float H = empty(s) ? 0.f : lnZ - kLn2 * (s.W / s.Z);
  if (o.entropy) o.entropy[r] = H;
  if (o.lse) o.lse[r] = empty(s) ? -kInf : s.m * o.scale + lnZ;
  if (o.saved)
    reinterpret_cast<float4 *>(o.saved)[r] = make_float4(s.m, s.Z, H, log2f(s.Z));
  if (o.logprob)
    o.logprob[r] = t.index < 0    ? 0.f
                   : t.index >= V ? __builtin_nanf("")
                                  : log_prob(t.logit, s, lnZ, o.scale);
}

constexpr int kMaxParts = 64;  // of a row: one for each lane of the joining wave

// A row's parts: `size` chunks of eight logits each (the last may be short).
struct Parts {
  int count;
  int64_t size;
};

// The chunks of one part; calls f(chunk, x) for this thread's, which lie
// kThreads apart: two at a time (chunk and the next, x[2][8]) where there are
// whole groups of four, with four loaded while four are worked on, and single
// ones (x[1][8]) behind them.
template <typename D, typename F>
__device__ __forceinline__ void each_chunk(const typename D::raw *row, int64_t c0, int64_t c1,
                                           int64_t V, F &&f) {
  constexpr int kAhead = 4, kTurn = kAhead * kThreads;
  const int whole = (int)min(c1, V / 8), end = (int)c1;
  int i = (int)c0 + threadIdx.x;
  Eight<D> e[kAhead];
  const auto load = [&](int at) {
#pragma unroll
    for (int a = 0; a < kAhead; ++a) e[a] = load_raw<D>(row, at + a * kThreads);
  };
  if (i + (kAhead - 1) * kThreads < whole) load(i);
  for (; i + (kAhead - 1) * kThreads < whole; i += kTurn) {
    Eight<D> now[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) now[a] = e[a];
    if (i + kTurn + (kAhead - 1) * kThreads < whole) load(i + kTurn);
#pragma unroll
    for (int a = 0; a < kAhead; a += 2) {
      float x[2][8];
      widen<D>(now[a], x[0]);
      widen<D>(now[a + 1], x[1]);
      f(i + a * kThreads, x);
    }
  }
  for (; i < end; i += kThreads) {
    float x[1][8];
    load8<D>(row, i, V, -kInf, x[0]);
    f(i, x);
  }
}

// ---------------------------------------------------------------------------
// Alternatives.  Every thread remembers the first of its chunks that holds its
// largest logit.  The k-th best of a wave's keys bounds the k-th best logit
// from below, and so does the largest of the waves' bounds; only the threads at
// or above it, at most k a wave, can hold one of the best: that chunk, or all of
// a thread's if its second best reaches the bound too, is read again (from the
// caches; a thread's chunks lie in different lines, and reading all of every
// thread's took 52 us instead of 39.6 for 1500 rows of 50257 bf16 with 20), and
// what reaches the bound is collected and sorted.
// Keys are distinct, so equal logits need no special case.  Rows with NaN, which
// the threads' largest logits do not see, and rows with more to collect than
// there is room for are searched once for every alternative.
// ---------------------------------------------------------------------------

constexpr int kMaxFound = 512;  // collected logits; beyond it, one at a time

struct TopLds {
  uint64_t waves[kWaves], scratch[64];
  uint64_t found[kMaxFound];
  uint64_t bound;
  int holders[kWaves * AF1_HEAD_MAX_TOP], chunks[kWaves * AF1_HEAD_MAX_TOP];
  int n_holders, n_chunks, n_found;
};

__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int mask) {
  return (uint64_t)__shfl_xor((unsigned long long)v, mask, 64);
}

// The value of lane ^ kMask, by register moves.
template <int kMask>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  const auto move = [](uint32_t u, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, decltype(ctrl)::value, 0xF, 0xF, false);
  };
  if constexpr (kMask == 1) return move(v, Int<0xB1>{});
  if constexpr (kMask == 2) return move(v, Int<0x4E>{});
  // the lanes of eight mirrored (^ 7), then of four (^ 3)
  if constexpr (kMask == 4) return move(move(v, Int<0x141>{}), Int<0x1B>{});
  if constexpr (kMask == 8) return move(v, Int<0x128>{});  // the row rotated by 8
  if constexpr (kMask == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  }
  if constexpr (kMask == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  }
}

template <int kMask>
__device__ __forceinline__ uint64_t exchange(uint64_t v, bool larger) {
  const uint64_t o = (uint64_t)lane_xor<kMask>((uint32_t)(v >> 32)) << 32 | lane_xor<kMask>((uint32_t)v);
  return (v > o) == larger ? v : o;
}

// The steps of a bitonic merge of runs of 2 kMask keys, descending where `down`.
template <int kMask>
__device__ __forceinline__ uint64_t merge_steps(uint64_t v, bool down) {
  v = exchange<kMask>(v, ((threadIdx.x & kMask) == 0) == down);
  if constexpr (kMask > 1) v = merge_steps<kMask / 2>(v, down);
  return v;
}

// Keys of a wave, the largest in lane 0 (bitonic).
__device__ __forceinline__ uint64_t sort64(uint64_t v) {
  const int lane = threadIdx.x & 63;
  v = merge_steps<1>(v, (lane & 2) == 0);
  v = merge_steps<2>(v, (lane & 4) == 0);
  v = merge_steps<4>(v, (lane & 8) == 0);
  v = merge_steps<8>(v, (lane & 16) == 0);
  v = merge_steps<16>(v, (lane & 32) == 0);
  return merge_steps<32>(v, true);
}

// The largest 64 of two sorted lists, sorted.
__device__ __forceinline__ uint64_t merge64(uint64_t a, const uint64_t *b) {
  return merge_steps<32>(max64(a, b[63 - (threadIdx.x & 63)]), true);
}

// In wave 0, lane i gets the i-th largest of the n collected keys.
__device__ __forceinline__ uint64_t sort_found(TopLds &l) {
  const int lane = threadIdx.x & 63, n = l.n_found;
  uint64_t v = sort64(lane < n ? l.found[lane] : 0);
  for (int at = 64; at < n; at += 64) {
    l.scratch[lane] = sort64(at + lane < n ? l.found[at + lane] : 0);
    __builtin_amdgcn_wave_barrier();
    v = merge64(v, l.scratch);
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
    if ((threadIdx.x & 63) == 0) l.waves[threadIdx.x >> 6] = b;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) b = max64(b, l.waves[w]);
    if ((int)threadIdx.x == j) mine = b;
    last = b;
  }
  return mine;
}

// In wave 0, lane i gets the i-th largest key of the chunks c0 .. c1 - 1 (i <
// k).  best, chunk: this thread's largest logit and the first chunk with it
// (chunk < 0: the thread has none); second: the largest of its other chunks.
// odd: there may be NaN.
template <typename D>
__device__ uint64_t part_top(const typename D::raw *row, int64_t c0, int64_t c1, int64_t V, int k,
                             float best, float second, int chunk, bool odd, TopLds &l) {
  const uint64_t mine = chunk < 0 ? 0 : order_key(best, 8 * (int64_t)chunk + 7);
  const uint64_t v = sort64(mine);
  if ((int)(threadIdx.x & 63) == k - 1) l.waves[threadIdx.x >> 6] = v;
  if (threadIdx.x == 0) l.n_holders = l.n_chunks = l.n_found = 0;
  __syncthreads();
  uint64_t bound = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) bound = max64(bound, l.waves[w]);
  if (threadIdx.x == 0) l.bound = bound;
  if (mine != 0 && mine >= bound) {
    // no bound has the logit NaN, and all chunks count
    if (second < key_logit(bound))
      l.chunks[atomicAdd(&l.n_chunks, 1)] = chunk;
    else
      l.holders[atomicAdd(&l.n_holders, 1)] = threadIdx.x;
  }
  __syncthreads();
  // at most 128 of both, and 2^13 chunks each
  const unsigned each = (unsigned)(c1 - c0 + kThreads - 1) / kThreads, ones = l.n_chunks;
  for (unsigned i = threadIdx.x; i < ones + l.n_holders * each; i += kThreads) {
    const unsigned j = i - ones;
    const int64_t c = i < ones ? l.chunks[i] : c0 + l.holders[j / each] + j % each * kThreads;
    if (c >= c1) continue;
    float x[8];
    load8<D>(row, c, V, -kInf, x);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (8 * c + e < V) collect(l, order_key(x[e], 8 * c + e));
  }
  __syncthreads();
  if (odd || l.n_found > kMaxFound)
    return one_by_one(k, l, [&](uint64_t after) {
      uint64_t b = 0;
      for (int64_t i = 8 * c0 + threadIdx.x; i < min(8 * c1, V); i += kThreads) {
        const uint64_t key = order_key(D::get(row[i]), i);
        if (key < after) b = max64(b, key);
      }
      return b;
    });
  return threadIdx.x < 64 ? sort_found(l) : 0;
}

__device__ __forceinline__ void write_top(const RowOut &o, int64_t r, const Stat &s, uint64_t key) {
  if ((int)threadIdx.x >= o.k) return;
  const bool there = key != 0;
  o.top_index[r * o.k + threadIdx.x] = there ? (int64_t)key_index(key) : -1;
  o.top_logprob[r * o.k + threadIdx.x] =
      there ? log_prob(key_logit(key), s, logf(s.Z), o.scale) : -kInf;
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
  const Target target = parts.count == 1 ? target_of<D>(o, row, r, V) : Target{};
  Stat s = no_logits();
  float best = -kInf, second = -kInf;
  int chunk = -1;
  each_chunk<D>(row, c0, c1, V, [&](int i, const auto &x) {
    constexpr int kN = sizeof(x) / 32;
    float top = -kInf;
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      const float m = max8(x[n]);
      if constexpr (kTop)
      {
        second = __builtin_amdgcn_fmed3f(m, best, second);
        if (chunk < 0 || m > best) best = m, chunk = i + n * kThreads;
      }
      top = fmaxf(top, m);
    }
    add<true>(s, x, top, c);
  });
  s = block_join<true>(s, c, sh);
  uint64_t key = 0;
  if constexpr (kTop) key = part_top<D>(row, c0, c1, V, o.k, best, second, chunk, s.Z != s.Z, top);
  if (parts.count == 1) {
    if (threadIdx.x == 0) write_row(o, target, r, V, s);
    if constexpr (kTop) write_top(o, r, s, key);
  } else {
    if (threadIdx.x == 0) po.stats[blockIdx.x] = s;
    if (kTop && (int)threadIdx.x < o.k) po.keys[(int64_t)blockIdx.x * o.k + threadIdx.x] = key;
  }
}

// Statistics of a row's parts (at most 64), joined in a fixed order; called by
// a whole wave.
template <bool kEntropy>
__device__ __forceinline__ Stat join_parts(const Stat *stats, int parts, float c) {
  const int lane = threadIdx.x & 63;
  return wave_join<kEntropy>(lane < parts ? stats[lane] : no_logits(), c);
}

// One block a row.  The parts' best keys bound the k-th best from below.
template <typename D, bool kTop>
__global__ __launch_bounds__(kThreads) void logprobs_join_kernel(const typename D::raw *z,
                                                                 int64_t V, int64_t ld, float c,
                                                                 int parts, PartOut po, RowOut o) {
  __shared__ TopLds l;
  const int64_t r = blockIdx.x;
  const typename D::raw *row = z + r * ld;
  // everything is asked for at once
  const uint64_t *keys = po.keys + r * parts * o.k;
  constexpr int kEach = kTop ? kMaxParts * AF1_HEAD_MAX_TOP / kThreads : 1;
  uint64_t mine[kEach], first = 0;
  if constexpr (kTop) {
    if ((int)threadIdx.x < parts) first = keys[threadIdx.x * o.k];
#pragma unroll
    for (int a = 0; a < kEach; ++a) {
      const int i = threadIdx.x + a * kThreads;
      mine[a] = i < parts * o.k ? keys[i] : 0;
    }
  }
  const Target target = target_of<D>(o, row, r, V);
  const Stat s = join_parts<true>(po.stats + r * parts, parts, c);
  if (threadIdx.x == 0) write_row(o, target, r, V, s);
  if constexpr (kTop) {
    if (threadIdx.x < 64) {
      const uint64_t v = sort64(first);
      // the list of a part with fewer than k logits ends in zeros
      if ((int)threadIdx.x == o.k - 1) l.bound = v;
      if (threadIdx.x == 0) l.n_found = 0;
    }
    __syncthreads();
#pragma unroll
    for (int a = 0; a < kEach; ++a) collect(l, mine[a]);
    __syncthreads();
    uint64_t key;
    if (l.n_found > kMaxFound)
      key = one_by_one(o.k, l, [&](uint64_t after) {
        uint64_t b = 0;
#pragma unroll
        for (int a = 0; a < kEach; ++a)
          if (mine[a] < after) b = max64(b, mine[a]);
        return b;
      });
    else
      key = threadIdx.x < 64 ? sort_found(l) : 0;
    write_top(o, r, s, key);
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
  const auto fill = [&](float v) {
    const float all[8] = {v, v, v, v, v, v, v, v};
    for (int64_t i = c0 + threadIdx.x; i < c1; i += kThreads) store8<D>(out, i, V, all);
  };
  if ((gl == 0.f && gh == 0.f) || (sv.x == -kInf && sv.y == 0.f)) return fill(0.f);
  if (y >= V && gl != 0.f) gl = __builtin_nanf("");
  if (gl != gl || gh != gh) return fill(__builtin_nanf(""));  // masked entries too
  const float c = scale * kLog2e;
  each_chunk<D>(z + r * ld, c0, c1, V, [&](int first, const auto &x) {
#pragma unroll
    for (int n = 0; n < (int)(sizeof(x) / 32); ++n) {
      const int64_t i = first + n * kThreads;
      float d[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float t = fmaf(x[n][j] - sv.x, c, -sv.w);  // log2 of the probability
        const float p = exp2_hw(t);
        d[j] = p == 0.f ? 0.f : -p * fmaf(gh, fmaf(kLn2, t, sv.z), gl);
      }
      if (y >= 8 * i && y < 8 * i + 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (8 * i + j == y) d[j] += gl;
      }
      store8<D, true>(out, i, V, d);
    }
  });
}

// ---------------------------------------------------------------------------
// KL divergence.  With p and q the teacher's and the student's softmax and
// u = log2 p - log2 q,
//   kl = ln2 A + ln(1 + B),   A = sum p u,   B = sum (p 2^-u - p) = sum (q - p).
// B is 0 but for rounding.  What the fp32 statistics are off by shifts all u
// alike, by s say; A then changes by s and ln2 A + ln(1 + B) only by its square,
// so a divergence that is small beside the logarithms errs by some 1e-8.  u is
// taken from the difference of the two logits, and q - p = p (2^-u - 1), the
// gradient's factor, from u.
//
// A block holds its part of both rows in registers from the first pass
// (statistics) to the second (terms and gradient), so that memory is read
// once.  A row of several parts is several blocks' work: each publishes its
// statistics, waits for the others' and joins them all in the parts' order.
// Waiting is bounded: statistics that do not arrive (their block has found no
// place on the device yet) are computed by the block that misses them, from the
// logits, with the same operations.  Rows of more parts than the device holds at
// once get their statistics from a launch of their own.  2048 rows of 128256 bf16
// with the gradient: 321 us, 4.9 TB/s (reading both rows again for the second
// pass: 517); 45 rows of 50257 fp32 15 us.
// ---------------------------------------------------------------------------

struct KlArgs {
  int64_t V, ld_s, ld_t, ldd;
  float scale;
  const float *weight;
  float *kl;
  Parts parts;
  // where a row has several parts:
  uint64_t *stats;  // [2, T, parts]: m and Z of the student, then of the teacher
  uint64_t *sums;   // [T, parts]: A and B
  int *done;        // [T]
};

constexpr uint64_t kNotYet = ~0ull;  // m is never NaN, so no statistics look so
#ifdef AF1_TEST_BUILD
// The test build waits for nothing, and every other part publishes some 60 us
// late: blocks compute the statistics that they miss.
constexpr int kPolls = 1, kLate = 16;
#else
constexpr int kPolls = 4096, kLate = 0;
#endif

__device__ __forceinline__ uint64_t pack2(float a, float b) {
  return (uint64_t)__float_as_uint(a) << 32 | __float_as_uint(b);
}
__device__ __forceinline__ float first_of(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ float second_of(uint64_t v) { return __uint_as_float((uint32_t)v); }

__device__ __forceinline__ uint64_t peek(const uint64_t *p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Stores v where every part of the chip sees it, and returns when it is there.
__device__ __forceinline__ void publish(uint64_t *p, uint64_t v) {
  const uint64_t old = __hip_atomic_exchange(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  asm volatile("" ::"v"(old) : "memory");
}

__global__ __launch_bounds__(kThreads) void kl_clear_kernel(uint64_t *words, int64_t n, int *done,
                                                            int64_t T) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i < n) words[i] = kNotYet;
  if (i < T) done[i] = 0;
}

struct KlLds {
  Stat wave[2 * kWaves];
  Stat part[2][64];
  Stat row[2];
  float sum[2 * kWaves];
  uint64_t missing;
};

// Statistics of a part whose block has not delivered.
template <typename D>
__device__ __forceinline__ void part_stats(const typename D::raw *s, const typename D::raw *t,
                                           int64_t c0, int64_t c1, int64_t V, float c, KlLds &l,
                                           Stat &a, Stat &b) {
  a = b = no_logits();
  for (int64_t i = c0 + threadIdx.x; i < c1; i += kThreads) {
    float x[1][8], w[1][8];
    load8<D>(s, i, V, -kInf, x[0]);
    load8<D>(t, i, V, -kInf, w[0]);
    add<false>(a, x, max8(x[0]), c);
    add<false>(b, w, max8(w[0]), c);
  }
  __syncthreads();
  a = block_join<false>(a, c, l.wave);
  b = block_join<false>(b, c, l.wave + kWaves);
}

// Statistics of every part, for rows whose parts do not all fit the device at
// once: those that run would wait for the others in vain and compute each of
// them themselves.
template <typename D>
__global__ __launch_bounds__(kThreads) void kl_stats_kernel(const typename D::raw *zs,
                                                            const typename D::raw *zt, int64_t T,
                                                            KlArgs g) {
  __shared__ KlLds l;
  const int64_t r = blockIdx.x / g.parts.count;
  const int64_t c0 = blockIdx.x % g.parts.count * g.parts.size;
  Stat a, b;
  part_stats<D>(zs + r * g.ld_s, zt + r * g.ld_t, c0, min(c0 + g.parts.size, (g.V + 7) / 8), g.V,
                g.scale * kLog2e, l, a, b);
  if (threadIdx.x == 0) {
    g.stats[blockIdx.x] = pack2(a.m, a.Z);
    g.stats[T * g.parts.count + blockIdx.x] = pack2(b.m, b.Z);
  }
}

// The rows' statistics from all parts'; every thread of the block calls it.
template <typename D>
__device__ void join_rows(const typename D::raw *s, const typename D::raw *t, int64_t r, int64_t T,
                          const KlArgs &g, float c, KlLds &l, Stat &a, Stat &b) {
  const int n = g.parts.count;
  const uint64_t *sa = g.stats + r * n, *sb = g.stats + (T + r) * n;
  for (int base = 0; base < n; base += 64) {
    const int here = min(64, n - base);
    if (threadIdx.x < 64) {
      const int lane = threadIdx.x;
      uint64_t va = 0, vb = 0;
      bool have = lane >= here;
      for (int poll = 0; poll < kPolls; ++poll) {
        if (!have) {
          va = peek(sa + base + lane);
          vb = peek(sb + base + lane);
          have = va != kNotYet && vb != kNotYet;
        }
        if (__all(have)) break;
        __builtin_amdgcn_s_sleep(2);
      }
      if (have && lane < here) {
        l.part[0][lane] = Stat{first_of(va), second_of(va), 0.f};
        l.part[1][lane] = Stat{first_of(vb), second_of(vb), 0.f};
      }
      const uint64_t missing = __ballot(!have);
      if (lane == 0) l.missing = missing;
    }
    __syncthreads();
    for (uint64_t missing = l.missing; missing; missing &= missing - 1) {
      const int p = __builtin_ctzll(missing);
      const int64_t c0 = (base + p) * g.parts.size;
      Stat x, y;
      part_stats<D>(s, t, c0, min(c0 + g.parts.size, (g.V + 7) / 8), g.V, c, l, x, y);
      if (threadIdx.x == 0) {
        // The part's block writes its gradient, maybe over these logits, only
        // after it has published: what it published by now goes first.
        const uint64_t va = peek(sa + base + p), vb = peek(sb + base + p);
        if (va != kNotYet && vb != kNotYet) {
          x = Stat{first_of(va), second_of(va), 0.f};
          y = Stat{first_of(vb), second_of(vb), 0.f};
        }
        l.part[0][p] = x;
        l.part[1][p] = y;
      }
      __syncthreads();
    }
    if (threadIdx.x < 64) {
      const int lane = threadIdx.x;
      Stat x = lane < here ? l.part[0][lane] : no_logits();
      Stat y = lane < here ? l.part[1][lane] : no_logits();
      x = wave_join<false>(x, c);
      y = wave_join<false>(y, c);
      if (base > 0) {
        x = join2(l.row[0], x, c);
        y = join2(l.row[1], y, c);
      }
      if (lane == 0) l.row[0] = x, l.row[1] = y;
    }
    __syncthreads();
  }
  a = l.row[0];
  b = l.row[1];
}

template <typename D, int kChunks>
__global__ __launch_bounds__(kThreads, 4) void kl_kernel(const typename D::raw *zs,
                                                         const typename D::raw *zt,
                                                         typename D::raw *ds, int64_t T, KlArgs g) {
  using R = typename D::raw;
  __shared__ KlLds l;
  const int parts = g.parts.count;
  const int64_t r = blockIdx.x / parts, V = g.V;
  const int64_t c0 = blockIdx.x % parts * g.parts.size;
  const int64_t c1 = min(c0 + g.parts.size, (V + 7) / 8);
  const R *s = zs + r * g.ld_s, *t = zt + r * g.ld_t;
  const float c = g.scale * kLog2e;

  Eight<D> xs[kChunks], xt[kChunks];
  const int whole = (int)(V / 8), first = (int)c0 + threadIdx.x, end = (int)c1;
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    // chunks that are not there read another one and look masked
    const int i = first + j * kThreads;
    const uint32_t at = (uint32_t)min(i, whole - 1) * (uint32_t)sizeof(Eight<D>);
    if (whole > 0) {
      xs[j] = *reinterpret_cast<const Eight<D> *>(reinterpret_cast<const char *>(s) + at);
      xt[j] = *reinterpret_cast<const Eight<D> *>(reinterpret_cast<const char *>(t) + at);
    }
  }
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    const int i = first + j * kThreads;
    if (i >= whole || i >= end) {
      const int64_t some = i < end ? V : 0;
      xs[j] = load_raw_to<D>(s, i, some, -kInf);
      xt[j] = load_raw_to<D>(t, i, some, -kInf);
    }
  }
  Stat a = no_logits(), b = no_logits();
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    if (c0 + j * kThreads >= c1) break;
    float x[1][8];
    widen<D>(xs[j], x[0]);
    add<false>(a, x, max8(x[0]), c);
    widen<D>(xt[j], x[0]);
    add<false>(b, x, max8(x[0]), c);
  }
  a = block_join<false>(a, c, l.wave);
  b = block_join<false>(b, c, l.wave + kWaves);
  if (parts > 1) {
    if (kLate > 0 && (blockIdx.x % parts & 1))
      for (int i = 0; i < kLate; ++i) __builtin_amdgcn_s_sleep(127);
    if (threadIdx.x == 0) {
      publish(g.stats + blockIdx.x, pack2(a.m, a.Z));
      publish(g.stats + T * parts + blockIdx.x, pack2(b.m, b.Z));
    }
    join_rows<D>(s, t, r, T, g, c, l, a, b);
  }

  const float gf = (g.weight ? g.weight[r] : 1.f) * g.scale;
  const bool none = empty(a) || empty(b), zero = none || gf == 0.f;
  const float la = log2f(a.Z), lb = log2f(b.Z);
  const float K = fmaf(b.m - a.m, c, lb - la);
  float A = 0.f, B = 0.f;
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    if (c0 + j * kThreads >= c1) break;
    float x[8], w[8], d[8];
    widen<D>(xs[j], x);
    widen<D>(xt[j], w);
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
      float p[4], e[4], u[4], least = kInf, most = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        p[k] = exp2_hw(fmaf(w[h + k] - b.m, c, -lb));
        u[k] = fmaf(w[h + k] - x[h + k], c, -K);
        e[k] = exp2_hw(-u[k]);
        least = fminf(least, p[k]);
        most = fmaxf(most, e[k]);
      }
      if (least > 0.f && most < kInf) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          d[h + k] = fmaf(p[k], e[k], -p[k]);
          A = fmaf(p[k], u[k], A);
        }
      } else {
        // masked entries, or ones below fp32: q on its own; 0 log 0 is 0
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          d[h + k] = exp2_hw(fmaf(x[h + k] - a.m, c, -la)) - p[k];
          A = fmaf(p[k], p[k] == 0.f ? 0.f : u[k], A);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        B += d[h + k];
        d[h + k] = zero ? 0.f : d[h + k] * gf;
      }
    }
    const int64_t i = c0 + threadIdx.x + j * kThreads;
    if (ds && i < c1) store8<D, true>(ds + r * g.ldd, i, V, d);
  }
  A = wave_add(A);
  B = wave_add(B);
  if ((threadIdx.x & 63) == 0) {
    l.sum[threadIdx.x >> 6] = A;
    l.sum[kWaves + (threadIdx.x >> 6)] = B;
  }
  __syncthreads();
  if (threadIdx.x >= 64) return;
  A = l.sum[0];
  B = l.sum[kWaves];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) A += l.sum[w], B += l.sum[kWaves + w];
  const int lane = threadIdx.x;
  if (parts > 1) {
    // the block that finishes the row adds the parts' sums
    int last = 0;
    if (lane == 0) {
      publish(g.sums + blockIdx.x, pack2(A, B));
      last = __hip_atomic_fetch_add(g.done + r, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
             parts - 1;
    }
    if (!__builtin_amdgcn_readfirstlane(last)) return;
    A = B = 0.f;
    for (int base = 0; base < parts; base += 64) {
      const uint64_t v = base + lane < parts ? peek(g.sums + r * parts + base + lane) : 0;
      A += wave_add(first_of(v));
      B += wave_add(second_of(v));
    }
  }
  if (lane == 0) {
    float kl = fmaf(kLn2, A, log1pf(B));
    kl = kl < 0.f ? 0.f : kl;  // the divergence is not: 0 is nearer to it
    // teacher masked: nothing to match; student masked: no finite code for it
    if (none) kl = a.Z != a.Z || b.Z != b.Z ? __builtin_nanf("") : empty(b) ? 0.f : kInf;
    g.kl[r] = kl;
  }
}

// Parts of a row for T rows: as many as give the device `want` blocks (whole rows
// from half of that), of at least one chunk a thread, at most `most`.
//
// Forward: 1024, four blocks a compute unit; a part costs a selection of its own
// and the join.  600 rows of 50257 bf16 with 5 alternatives 22.8 us, with 2048
// blocks 28.0; 64 of 128256 14.1 and 16.9.  Backward: 2048, which has neither to
// pay for: 600 rows of 128256 bf16 53.5 us, with 1024 blocks 63.
constexpr int64_t kForwardBlocks = 1024, kBackwardBlocks = 2048;

Parts plan_parts(int64_t T, int64_t V, int64_t want, int most) {
  const int64_t chunks = (V + 7) / 8;
  int64_t n = T >= want / 2 ? 1 : (want + T - 1) / T;
  const int64_t fit = (chunks + kThreads - 1) / kThreads;
  n = n < fit ? n : fit;
  n = n < most ? n : most;
  const int64_t size = ((chunks + n - 1) / n + kThreads - 1) / kThreads * kThreads;
  return Parts{(int)((chunks + size - 1) / size), size};
}

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

}  // namespace

size_t token_logprobs_workspace_bytes(int64_t T, int64_t V, int k) {
  const Parts p = plan_parts(T, V, kForwardBlocks, kMaxParts);
  if (p.count == 1) return 0;
  return up16((size_t)T * p.count * sizeof(Stat)) + (size_t)T * p.count * k * 8;
}

hipError_t launch_token_logprobs(const Rows &z, float scale, const int64_t *targets,
                                 float *logprob, float *entropy, float *lse, int k,
                                 float *top_logprob, int64_t *top_index, float *saved, void *ws,
                                 hipStream_t s) {
  const RowOut o{targets, logprob, entropy, lse, saved, k, top_logprob, top_index, scale};
  const Parts p = plan_parts(z.T, z.V, kForwardBlocks, kMaxParts);
  PartOut po{nullptr, nullptr};
  if (p.count > 1)
    po = PartOut{static_cast<Stat *>(ws),
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
  const Parts p = plan_parts(z.T, z.V, kBackwardBlocks, 1 << 12);
  return with_type(z.dtype, [&](auto d) {
    using D = decltype(d);
    logprobs_backward_kernel<D><<<(unsigned)(z.T * p.count), kThreads, 0, s>>>(
        static_cast<const typename D::raw *>(z.p), z.V, z.ld, scale, p, targets, saved, g_logprob,
        g_entropy, static_cast<typename D::raw *>(dlogits), ldd);
    return hipGetLastError();
  });
}

// Chunks of eight that a thread of the KL kernel holds of each row: 64
// registers, or 32 bytes when there are few rows to fill the device with.
template <typename D>
constexpr int kl_chunks(bool few) {
  return few ? (sizeof(typename D::raw) == 4 ? 1 : 2) : (sizeof(typename D::raw) == 4 ? 4 : 8);
}

constexpr int64_t kKlBlocks = 256;

struct KlPlan {
  bool few;
  Parts parts;
  // a row's parts are more than half of the workgroups that the device holds at
  // once (four a compute unit): their statistics take a launch of their own.
  // From 4.2 million fp32 or 8.4 million 16-bit logits; one row of 2^24 fp32 with
  // the gradient: 134 us.
  bool stats_first() const { return parts.count > 2 * device_cus(); }
};

KlPlan plan_kl(int dtype, int64_t T, int64_t V) {
  return with_type(dtype, [&](auto d) {
    using D = decltype(d);
    const int64_t chunks = (V + 7) / 8;
    KlPlan p{};
    for (bool few : {false, true}) {
      const int64_t most = (int64_t)kl_chunks<D>(few) * kThreads, n = (chunks + most - 1) / most;
      // as even as whole turns of the block allow
      const int64_t size = ((chunks + n - 1) / n + kThreads - 1) / kThreads * kThreads;
      p = KlPlan{few, Parts{(int)((chunks + size - 1) / size), size}};
      // a workgroup for every compute unit: 64 rows of 128256 bf16 in 21 us with
      // eight parts a row, 28 with thirty-two
      if (T * p.parts.count >= kKlBlocks) break;
    }
    return p;
  });
}

size_t distill_kl_workspace_bytes(int64_t T, int64_t V) {
  // of whatever type the logits are
  size_t most = 0;
  for (int dtype : {AF1_SRC_F32, AF1_SRC_BF16, AF1_SRC_F16}) {
    const size_t n = plan_kl(dtype, T, V).parts.count;
    const size_t need = n == 1 ? 0 : (size_t)T * (n * 24 + 4);
    most = need > most ? need : most;
  }
  return most;
}

hipError_t launch_distill_kl(const Rows &z, const void *teacher, int64_t ld_t, float scale,
                             const float *weight, float *kl, void *dstudent, int64_t ldd, void *ws,
                             hipStream_t s) {
  const KlPlan plan = plan_kl(z.dtype, z.T, z.V);
  KlArgs g{z.V, z.ld, ld_t, ldd, scale, weight, kl, plan.parts, nullptr, nullptr, nullptr};
  const int64_t blocks = z.T * plan.parts.count;
  if (plan.parts.count > 1) {
    g.stats = static_cast<uint64_t *>(ws);
    g.sums = g.stats + 2 * blocks;
    g.done = reinterpret_cast<int *>(g.sums + blocks);
    kl_clear_kernel<<<(unsigned)((2 * blocks + kThreads - 1) / kThreads), kThreads, 0, s>>>(
        g.stats, 2 * blocks, g.done, z.T);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && plan.stats_first())
      e = with_type(z.dtype, [&](auto d) {
        using D = decltype(d);
        kl_stats_kernel<D><<<(unsigned)blocks, kThreads, 0, s>>>(
            static_cast<const typename D::raw *>(z.p), static_cast<const typename D::raw *>(teacher),
            z.T, g);
        return hipGetLastError();
      });
    if (e != hipSuccess) return e;
  }
  return with_type(z.dtype, [&](auto d) {
    using D = decltype(d);
    const auto *a = static_cast<const typename D::raw *>(z.p);
    const auto *b = static_cast<const typename D::raw *>(teacher);
    auto *out = static_cast<typename D::raw *>(dstudent);
    if (plan.few)
      kl_kernel<D, kl_chunks<D>(true)><<<(unsigned)blocks, kThreads, 0, s>>>(a, b, out, z.T, g);
    else
      kl_kernel<D, kl_chunks<D>(false)><<<(unsigned)blocks, kThreads, 0, s>>>(a, b, out, z.T, g);
    return hipGetLastError();
  });
}

}  // namespace af1h

#ifdef AF1_TEST_BUILD
// Parts of a KL row, and whether their statistics take a launch of their own.
extern "C" AF1_API int af1_test_kl_plan(int32_t dtype, int64_t T, int64_t V, int32_t *out) {
  const af1h::KlPlan p = af1h::plan_kl(dtype, T, V);
  out[0] = p.parts.count;
  out[1] = p.stats_first();
  return 0;
}

// Parts of a row of log probabilities.
extern "C" AF1_API int af1_test_logprobs_plan(int64_t T, int64_t V, int32_t *out) {
  out[0] = af1h::plan_parts(T, V, af1h::kForwardBlocks, af1h::kMaxParts).count;
  return 0;
}
#endif
