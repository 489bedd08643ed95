// soma_sample.hip -- the next token of every row of logits: temperature, top-k, top-p
// and min-p, from given random numbers.
//
// A block takes one row, which it reads once into LDS (or again and again, if it is too
// long).  Nothing is sorted: what the filters keep is every token from a border on in
// the order of (logit, -index), and the border is found from a histogram of the
// distances from the largest logit, its bins as fine as the row's range allows, and from
// the few tokens of the bin that holds it, compared with one another.  (A bin of more
// tokens than lanes, as equal logits make it: the border is found bit by bit.)  Weights
// are integers, fp64 exponentials times 2^s, so that their sums do not depend on the
// order in which LDS's atomics add them up.  Then the waves sum what is kept in
// consecutive pieces of the row, and the one whose piece holds the token looks for it.
//
// 256 rows of 50,257 in bf16, all filters: 70 us, a row a compute unit, the slowest row's
// time: 3 for the largest, 4 for the histogram, 4 to 18 for the weights (fp64, and LDS's
// atomics), 10 to 17 for two borders, 4 to 12 for the sums.  The rows are 26 MB, 5 us.
//
// An exponential is 2^(k/256) from a table times a polynomial of degree 4: the remainder
// is at most ln 2 / 512, its fifth power over 5! 3.8e-17.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "soma.h"
#include "soma_host.hpp"
#include "soma_types.hpp"
#include "soma_wave.hpp"

namespace soma {
namespace {

typedef unsigned long long u64;

struct Sample {
  const void* logits;
  int64_t stride;
  const float *u, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* tokens;
  float* logprob;
  int vocab, shift;           // weights are multiples of 2^-shift
};

// A logit's bits in the order of the values, 0 for -infinity and NaN.
template <class T>
__device__ __forceinline__ uint32_t key_of(float x) {
  if (!(x > -__builtin_huge_valf())) return 0;
  if (x == 0.0f) x = 0.0f;                  // both zeros are equal
  const uint32_t b = __float_as_uint(x), k = b & 0x80000000u ? ~b : b | 0x80000000u;
  return sizeof(T) == 2 ? k >> 16 : k;
}
template <class T>
__device__ __forceinline__ float value_of(uint32_t k) {
  if (sizeof(T) == 2) k = k << 16 | (k & 0x8000u ? 0u : 0xFFFFu);
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

// Sum over the lanes in front of this one, and over all of them.
template <class V>
__device__ __forceinline__ V wave_before(V v, V* all) {
  const int lane = threadIdx.x & 63;
  V sum = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const V x = __shfl_up(sum, d);
    if (lane >= d) sum += x;
  }
  *all = __shfl(sum, 63);
  return sum - v;
}

constexpr int kIndexBits = 20;              // of a vocabulary
constexpr size_t kLds = 160 * 1024;         // of a compute unit: more than that must not be asked for

// kBins bins; kInLds: the row is held in LDS.
template <class T, int kThreads, int kBins, bool kInLds>
struct Row {
  static constexpr int kWaves = kThreads / 64, kMine = kBins / kThreads;
  static constexpr int kOrderBits = (sizeof(T) == 2 ? 16 : 32) + kIndexBits;
  struct Shared {
    u64 weight[kBins];
    u64 order[kThreads], own[kThreads];     // tokens of the bin that holds a border
    double table[256];
    float line[kWaves][128];
    u64 wave_weight[kWaves];
    u64 wave_count[kWaves];
    u64 border;
    uint32_t count[kBins];
    uint32_t listed, found_bin;
    u64 found_weight;
  };
  Shared& s;
  const T* x;                 // in memory
  const T* held;              // in LDS, `lead` elements from 16 bytes
  int lead, vocab, shift;
  float top, low, fine;       // the largest logit; below which weights are 0; bins per distance
  float edge;                 // the border's logit, and
  int edge_to;                // the last of those equal to it that is kept
  double per;                 // 256 log2(e) / temperature

  // Tokens that a lane works on side by side: eight in a row of LDS, whose ends are filled
  // up with -infinity, or eight that lie 64 apart in memory.
  static constexpr int kAhead = 8;
  template <class F>
  static __device__ __forceinline__ void each(F f) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) f(k);
  }
  __device__ __forceinline__ int groups() const { return kInLds ? (lead + vocab + 7) / 8 : (vocab + 511) / 512 * 64; }
  // Token k of group v; of consecutive groups of 64 the tokens are consecutive.
  __device__ __forceinline__ int token(int v, int k) const { return kInLds ? 8 * v + k - lead : (v >> 6) * 512 + (v & 63) + 64 * k; }
  __device__ __forceinline__ int first_token(int v) const { return max(0, kInLds ? 8 * v - lead : (v >> 6) * 512); }
  __device__ __forceinline__ void eight(int v, float (&l)[kAhead]) const {
    if constexpr (kInLds) {
      if constexpr (sizeof(T) == 2) {
        const uint4 u = *reinterpret_cast<const uint4*>(held - lead + 8 * v);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        each([&](int k) { l[k] = __uint_as_float(k & 1 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16); });
      } else {
        const float4 a = load_four(held - lead + 8 * v), b = load_four(held - lead + 8 * v + 4);
        l[0] = a.x, l[1] = a.y, l[2] = a.z, l[3] = a.w, l[4] = b.x, l[5] = b.y, l[6] = b.z, l[7] = b.w;
      }
    } else {
      each([&](int k) { l[k] = token(v, k) < vocab ? load_value(x + token(v, k)) : -__builtin_huge_valf(); });
    }
  }

  __device__ __forceinline__ float at(int i) const { return kInLds ? load_value(held + i) : load_value(x + i); }

  // Position in the ranking: the larger, the earlier; 0: never drawn.
  __device__ __forceinline__ u64 order_of(float l, int i) const {
    return l >= low ? static_cast<u64>(key_of<T>(l)) << kIndexBits | static_cast<uint32_t>((1 << kIndexBits) - 1 - i) : 0;
  }
  // Whether a token lies at the border or in front of it in the ranking.
  __device__ __forceinline__ bool in(float l, int i) const { return l >= edge && (l > edge || i <= edge_to); }

  // Lets f see what is in, closed up: 64 logits at a time, one a lane, and once what is
  // left.  Groups first, first + 64, .. of a wave.
  template <class F>
  __device__ __forceinline__ void closed(int first, int end, F f) {
    const int lane = threadIdx.x & 63;
    float* const line = s.line[threadIdx.x >> 6];
    int listed = 0;
    for (int v0 = first; v0 < end; v0 += 64) {
      const int v = v0 + lane;
      float l[kAhead];
      bool mine[kAhead], any = false;
      if (v < end) eight(v, l);
      each([&](int k) { any |= mine[k] = v < end && l[k] >= edge; });
      if (__builtin_amdgcn_ballot_w64(any) == 0) continue;
      each([&](int k) {
        mine[k] = mine[k] && (l[k] > edge || token(v, k) <= edge_to);
        const u64 here = __builtin_amdgcn_ballot_w64(mine[k]);
        if (mine[k]) line[listed + __builtin_amdgcn_mbcnt_hi(here >> 32, __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(here), 0))] = l[k];
        listed += __popcll(here);
        if (listed >= 64) {
          wave_lds_sync();
          f(line[lane], true);
          listed -= 64;
          const float rest = line[64 + lane];
          wave_lds_sync();
          line[lane] = rest;
        }
      });
    }
    wave_lds_sync();
    f(lane < listed ? line[lane] : top, lane < listed);
  }

  // exp((l - top) / temperature) = 2^(k / 256) 2^r, k + 256 r = y: the first as the power
  // *n and a factor in [1, 2) from the table, the product with the second.  The rounding
  // to k is an addition's, whose sum holds k in its lower half.
  __device__ __forceinline__ double share(float l, int* n) const {
    constexpr double kRound = 6755399441055744.0;       // 1.5 2^52
    double y = (static_cast<double>(l) - static_cast<double>(top)) * per;
    y = l >= top ? 0.0 : fmax(y, -1e6);
    const double z = y + kRound, r = y - (z - kRound);
    constexpr double c1 = 0.69314718055994530942 / 256, c2 = c1 * c1 / 2, c3 = c2 * c1 / 3, c4 = c3 * c1 / 4;
    const double p = fma(fma(fma(fma(c4, r, c3), r, c2), r, c1), r, 1.0);
    const int k = static_cast<int>(__double_as_longlong(z));
    *n = k >> 8;
    return s.table[k & 255] * p;
  }
  __device__ __forceinline__ double share(float l) const {
    int n;
    const double w = share(l, &n);
    return ldexp(w, n);
  }
  // As a multiple of 2^-shift, rounded down: the fraction's bits, moved.
  __device__ __forceinline__ u64 weight_of(float l) const {
    int n;
    const uint64_t b = __double_as_longlong(share(l, &n));
    const int right = 62 - shift - n - (static_cast<int>(b >> 52) - 1023);
    const u64 m = (b << 10 & 0x3FFFFFFFFFFFFFFFull) | 0x4000000000000000ull;
    return right < 64 ? m >> right : 0;
  }

  // (distances that are no number, of infinities and NaN, in the last)
  __device__ __forceinline__ int bin_of(float l) const { return static_cast<int>(fminf((top - l) * fine, kBins - 1)); }

  template <class V>
  __device__ V over_block(V v) {
    V all;
    wave_before(v, &all);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.wave_weight[threadIdx.x >> 6] = all;
    __syncthreads();
    V sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += static_cast<V>(s.wave_weight[w]);
    return sum;
  }

  // Number and weight of the tokens of every bin: of all of them (their number alone, or
  // both), or of those that are in.
  __device__ __forceinline__ void histogram(bool all, bool weights) {
    for (int i = threadIdx.x; i < kBins; i += kThreads) s.weight[i] = 0, s.count[i] = 0;
    __syncthreads();
    if (all) {
      for (int v = threadIdx.x; v < groups(); v += kThreads) {
        float l[kAhead];
        eight(v, l);
        u64 w[kAhead];
        // (of what does not count, any number)
        if (weights) each([&](int k) { w[k] = weight_of(l[k]); });
        each([&](int k) {
          if (!(l[k] >= low)) return;
          const int bin = bin_of(l[k]);
          atomicAdd(&s.count[bin], 1u);
          if (weights) atomicAdd(&s.weight[bin], w[k]);
        });
      }
    } else {
      const int piece = (groups() + kWaves * 64 - 1) / (kWaves * 64) * 64, first = static_cast<int>(threadIdx.x >> 6) * piece;
      closed(first, min(first + piece, groups()), [&](float l, bool mine) {
        const u64 w = weight_of(l);
        if (!mine) return;
        atomicAdd(&s.count[bin_of(l)], 1u);
        atomicAdd(&s.weight[bin_of(l)], w);
      });
    }
    __syncthreads();
  }

  // The border where the tokens up to it become `goal` in number (by_count) or weight,
  // which it puts in place of the one that the histogram went by; not if all of them do
  // not.
  template <bool by_count>
  __device__ __forceinline__ void find(u64 goal) {
    // bins in the order of their distances
    u64 c[kMine], mine = 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int bin = threadIdx.x * kMine + i;
      c[i] = by_count ? s.count[bin] : s.weight[bin];
      mine += c[i];
    }
    u64 all;
    u64 before = wave_before(mine, &all);
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.wave_count[wave] = all;
    if (threadIdx.x == 0) s.listed = 0, s.border = ~0ull, s.found_bin = kBins;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) before += w < wave ? s.wave_count[w] : 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      if (before < goal && before + c[i] >= goal) {
        s.found_bin = threadIdx.x * kMine + i;
        s.found_weight = before;
      }
      before += c[i];
    }
    __syncthreads();
    const int bin = s.found_bin;
    if (bin >= kBins) return;
    const u64 front = s.found_weight;
    const uint32_t n = s.count[bin];
    if (n > kThreads) {
      // bit by bit: the largest position up to which there is enough
      u64 b = 0;
      for (int bit = kOrderBits - 1; bit >= 0; --bit) {
        const u64 trial = b | 1ull << bit;
        u64 v = 0;
        for (int i = threadIdx.x; i < vocab; i += kThreads) {
          const float l = at(i);
          if (order_of(l, i) >= trial) v += by_count ? 1 : weight_of(l);
        }
        if (over_block(v) >= goal) b = trial;
      }
      set_border(b);
      return;
    }
    for (int v = threadIdx.x; v < groups(); v += kThreads) {
      float l[kAhead];
      eight(v, l);
      bool any = false;
      each([&](int k) { any |= bin_of(l[k]) == bin; });
      if (!any) continue;
      each([&](int k) {
        if (bin_of(l[k]) != bin) return;
        const u64 o = order_of(l[k], token(v, k));
        if (o == 0 || !in(l[k], token(v, k))) return;
        const uint32_t to = atomicAdd(&s.listed, 1u);
        s.order[to] = o;
        s.own[to] = weight_of(l[k]);
      });
    }
    const uint32_t eights = (n + 7) / 8 * 8;
    if (threadIdx.x >= n && threadIdx.x < eights) s.order[threadIdx.x] = 0;
    __syncthreads();
    if (threadIdx.x < n) {
      const u64 o = s.order[threadIdx.x];
      u64 up = front;                       // in front of this one
      for (uint32_t j = 0; j < eights; j += 8) {
        u64 theirs[8], own[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) theirs[k] = s.order[j + k], own[k] = by_count ? 1 : s.own[j + k];
#pragma unroll
        for (int k = 0; k < 8; ++k) up += theirs[k] > o ? own[k] : 0;
      }
      if (up < goal) atomicMin(&s.border, o);
    }
    __syncthreads();
    const u64 border = s.border;
    __syncthreads();
    set_border(border);
  }

  __device__ __forceinline__ void set_border(u64 order) {
    edge = value_of<T>(static_cast<uint32_t>(order >> kIndexBits));
    edge_to = (1 << kIndexBits) - 1 - static_cast<int>(order & ((1 << kIndexBits) - 1));
  }
};

template <class T, int kThreads, int kBins, bool kInLds>
__global__ __launch_bounds__(kThreads) void k_sample(const Sample a) {
  typedef Row<T, kThreads, kBins, kInLds> R;
  __shared__ typename R::Shared shared;
  extern __shared__ __align__(16) unsigned char memory[];
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T* const x = static_cast<const T*>(a.logits) + row * a.stride;
  R r{shared, x, nullptr, 0, a.vocab, a.shift};

  // the largest logit, and the smallest (of some) that is a number: how far bins have to reach
  float highest = -__builtin_huge_valf(), lowest = __builtin_huge_valf();
  if constexpr (kInLds) {
    // 16 bytes at a time where the row's address allows, at the same place in 16 bytes of LDS
    constexpr int kEight = 16 / sizeof(T);
    const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(x) % 16 / sizeof(T));
    T* const held = reinterpret_cast<T*>(memory) + lead;
    r.held = held, r.lead = lead;
    if (threadIdx.x < 16) {
      const int i = threadIdx.x < 8 ? static_cast<int>(threadIdx.x) - lead : a.vocab + static_cast<int>(threadIdx.x) - 8;
      if (threadIdx.x < 8 ? i < 0 : (i + lead) / 8 == (a.vocab + lead - 1) / 8) store_value(held + i, -__builtin_huge_valf());
    }
    const int first = min(lead ? kEight - lead : 0, a.vocab), wide = (a.vocab - first) / kEight;
    constexpr int kBatch = 4;
    for (int i0 = threadIdx.x; i0 < wide; i0 += kThreads * kBatch) {
      uint4 u[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (i0 + kThreads * k < wide) u[k] = *reinterpret_cast<const uint4*>(x + first + (i0 + kThreads * k) * kEight);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int i = first + (i0 + kThreads * k) * kEight;
        if (i0 + kThreads * k >= wide) break;
        *reinterpret_cast<uint4*>(held + i) = u[k];
        const uint32_t w[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // (fmaxf leaves NaN out)
          highest = fmaxf(highest, __uint_as_float(sizeof(T) == 2 ? w[e] & 0xFFFF0000u : w[e]));
          if constexpr (sizeof(T) == 2) highest = fmaxf(highest, __uint_as_float(w[e] << 16));
        }
        const float some = __uint_as_float(sizeof(T) == 2 ? w[0] << 16 : w[0]);
        lowest = fminf(lowest, some > -__builtin_huge_valf() ? some : lowest);
      }
    }
    const int rest = a.vocab - wide * kEight;           // at both ends
    if (static_cast<int>(threadIdx.x) < rest) {
      const int i = static_cast<int>(threadIdx.x) < first ? threadIdx.x : threadIdx.x + wide * kEight;
      held[i] = x[i];
      highest = fmaxf(highest, load_value(x + i));
    }
  } else {
    for (int v = threadIdx.x; v < r.groups(); v += kThreads) {
      float l[R::kAhead];
      r.eight(v, l);
      R::each([&](int k) { highest = fmaxf(highest, l[k]); });
      lowest = fminf(lowest, l[0] > -__builtin_huge_valf() ? l[0] : lowest);
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    highest = fmaxf(highest, __shfl_xor(highest, d));
    lowest = fminf(lowest, __shfl_xor(lowest, d));
  }
  if (lane == 0) shared.line[0][wave] = highest, shared.line[0][64 + wave] = lowest;
  if (threadIdx.x < 256) shared.table[threadIdx.x] = exp2(threadIdx.x * 0.00390625);
  if (threadIdx.x == 0) shared.found_bin = ~0u;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < R::kWaves; ++w) {
    highest = fmaxf(highest, shared.line[0][w]);
    lowest = fminf(lowest, shared.line[0][64 + w]);
  }
  __syncthreads();
  const float temperature = a.temperature ? a.temperature[row] : 1.0f;
  if (!(highest > -__builtin_huge_valf()) || !(temperature > 0.0f)) {
    // none, or the first of the likeliest
    uint32_t first = ~0u;
    if (highest > -__builtin_huge_valf())
      for (int i = threadIdx.x; i < a.vocab; i += kThreads)
        if (r.at(i) == highest) first = min(first, static_cast<uint32_t>(i));
    if (first != ~0u) atomicMin(&shared.found_bin, first);
    __syncthreads();
    if (threadIdx.x == 0) {
      a.tokens[row] = static_cast<int32_t>(shared.found_bin);
      if (a.logprob) a.logprob[row] = shared.found_bin != ~0u ? 0.0f : -__builtin_huge_valf();
    }
    return;
  }
  r.top = highest == 0.0f ? 0.0f : highest;
  r.per = 369.32993046757463 / static_cast<double>(temperature);
  // weights below a unit are 0; an infinite logit leaves no other
  const float reach = r.top == __builtin_huge_valf() ? 0.0f : (a.shift + 0.02f) * 0.6931472f * temperature;
  r.low = r.top == __builtin_huge_valf() ? r.top : fmaxf(r.top - reach, -3.402823466e38f);
  const float range = lowest < r.top ? fminf(reach, r.top - lowest) : reach;
  r.fine = range > 0.0f ? fminf(kBins / range, 1e30f) : 0.0f;
  r.edge = r.low, r.edge_to = a.vocab;

  const int32_t top_k = a.top_k ? a.top_k[row] : 0;
  const float top_p = a.top_p ? a.top_p[row] : 1.0f;
  const float least = a.min_p ? a.min_p[row] : 0.0f;
  const double min_p = least > 0.0f ? fmin(static_cast<double>(least), 1.0) : 0.0;
  const bool by_k = top_k > 0 && top_k < a.vocab, by_p = top_p < 1.0f;
  if (by_k) {
    r.histogram(true, false);
    r.template find<true>(top_k);
  }
  if (by_p) {
    r.histogram(!by_k, true);
    u64 total = 0;
    for (int i = threadIdx.x; i < kBins; i += kThreads) total += shared.weight[i];
    total = r.over_block(total);
    const double p = fmax(static_cast<double>(top_p), 0.0);
    r.template find<false>(min(max(static_cast<u64>(ceil(p * static_cast<double>(total))), u64{1}), total));
  }
  const auto weight_of = [&](float l) { return min_p > 0.0 && r.share(l) < min_p ? 0 : r.weight_of(l); };

  // The row in consecutive pieces, a wave each; then the piece that holds the token, the
  // same way, until one wave can go through it.
  int from = 0, to = a.vocab;
  u64 sum = 0, all;
  const int piece0 = (r.groups() + R::kWaves * 64 - 1) / (R::kWaves * 64) * 64;
  r.closed(wave * piece0, min((wave + 1) * piece0, r.groups()), [&](float l, bool mine) {
    const u64 w = weight_of(l);
    sum += mine ? w : 0;
  });
  wave_before(sum, &all);
  __syncthreads();
  if (lane == 0) shared.wave_weight[wave] = all;
  __syncthreads();
  u64 total = 0;
#pragma unroll
  for (int w = 0; w < R::kWaves; ++w) total += shared.wave_weight[w];
  const double target = fmin(fmax(static_cast<double>(a.u[row]), 0.0), 1.0) * static_cast<double>(total);
  u64 goal = min(static_cast<u64>(target), total - 1);
  // the piece that holds the token: the waves whose pieces end in front of it
  const auto choose = [&]() {
    u64 end = 0, front = 0;
    int w = 0;
#pragma unroll
    for (int i = 0; i < R::kWaves; ++i) {
      end += shared.wave_weight[i];
      if (goal >= end) front = end, w = i + 1;
    }
    goal -= front;
    return w;
  };
  int w = choose();
  from = r.first_token(w * piece0), to = min(r.first_token((w + 1) * piece0), a.vocab);
  while (to - from > 256) {
    const int piece = (to - from + R::kWaves * 64 - 1) / (R::kWaves * 64) * 64;
    const int lo = min(from + wave * piece, to), hi = min(lo + piece, to);
    sum = 0;
    for (int i = lo + lane; i < hi; i += 64) {
      const float l = r.at(i);
      if (r.in(l, i)) sum += weight_of(l);
    }
    wave_before(sum, &all);
    __syncthreads();
    if (lane == 0) shared.wave_weight[wave] = all;
    __syncthreads();
    w = choose();
    from = min(from + w * piece, to), to = min(from + piece, to);
  }
  if (wave != 0) return;
  for (int i = from; i < to; i += 64) {
    const float l = i + lane < to ? r.at(i + lane) : -__builtin_huge_valf();
    const u64 own = r.in(l, i + lane) ? weight_of(l) : 0;
    u64 here;
    const u64 front = wave_before(own, &here);
    if (goal < here) {
      if (own && front <= goal && goal < front + own) {
        a.tokens[row] = i + lane;
        if (a.logprob)
          a.logprob[row] = static_cast<float>(log(r.share(l) / ldexp(static_cast<double>(total), -a.shift)));
      }
      break;
    }
    goal -= here;
  }
}

// Up to 256 tokens, one a lane: each compares itself with all others, which gives its
// rank and the weight in front of it at once.  One pass without histograms, a few block
// sums: latency alone counts (64 rows of 256 in fp32: 8.6 us, with histograms 13.8).
constexpr int kFew = 256;

template <class T>
__global__ __launch_bounds__(kFew) void k_sample_few(const Sample a) {
  constexpr int kWaves = kFew / 64;
  __shared__ u64 order[kFew], weight[kFew], sums[3][kWaves];
  __shared__ float tops[kWaves];
  const int64_t row = blockIdx.x;
  const int i = threadIdx.x, lane = i & 63, wave = i >> 6;
  const float inf = __builtin_huge_valf();
  const float x = i < a.vocab ? load_value(static_cast<const T*>(a.logits) + row * a.stride + i) : -inf;
  const float l = x > -inf ? x : -inf;      // (NaN as well)
  float top = wave_max(l);
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  const float temperature = a.temperature ? a.temperature[row] : 1.0f;
  const bool greedy = !(temperature > 0.0f);
  double w = 0.0;
  if (l > -inf) w = l == top ? 1.0 : top == inf || greedy ? 0.0 : exp((static_cast<double>(l) - static_cast<double>(top)) / static_cast<double>(temperature));
  const double v = ldexp(w, a.shift - 32);
  const uint32_t high = static_cast<uint32_t>(v);
  const u64 own = static_cast<u64>(high) << 32 | static_cast<uint32_t>((v - static_cast<double>(high)) * 4294967296.0);
  const u64 mine = own ? static_cast<u64>(key_of<T>(l)) << 32 | static_cast<uint32_t>(kFew - i) : 0;
  order[i] = mine, weight[i] = own;
  __syncthreads();
  int rank = 0;
  u64 front = 0;
  for (int j = 0; j < a.vocab; j += 8) {
    u64 o[8], u[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = order[j + k], u[k] = weight[j + k];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      rank += o[k] > mine;
      front += o[k] > mine ? u[k] : 0;
    }
  }
  const int32_t top_k = greedy ? 1 : a.top_k ? a.top_k[row] : 0;
  const float top_p = a.top_p ? a.top_p[row] : 1.0f, least = a.min_p ? a.min_p[row] : 0.0f;
  bool in = own && (top_k <= 0 || rank < top_k);
  u64 all;
  if (!greedy && top_p < 1.0f) {
    wave_before(in ? own : 0, &all);
    if (lane == 0) sums[0][wave] = all;
    __syncthreads();
    const u64 total = sums[0][0] + sums[0][1] + sums[0][2] + sums[0][3];
    const u64 goal = min(max(static_cast<u64>(ceil(fmax(static_cast<double>(top_p), 0.0) * static_cast<double>(total))), u64{1}), total);
    in = in && front < goal;
  }
  if (!greedy && least > 0.0f) in = in && w >= fmin(static_cast<double>(least), 1.0);
  u64 before = wave_before(in ? own : 0, &all);
  if (lane == 0) sums[1][wave] = all;
  __syncthreads();
  u64 total = 0;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    before += k < wave ? sums[1][k] : 0;
    total += sums[1][k];
  }
  if (total == 0) {
    if (i == 0) {
      a.tokens[row] = -1;
      if (a.logprob) a.logprob[row] = -inf;
    }
    return;
  }
  const u64 goal = min(static_cast<u64>(fmin(fmax(static_cast<double>(a.u[row]), 0.0), 1.0) * static_cast<double>(total)), total - 1);
  if (in && before <= goal && goal < before + own) {
    a.tokens[row] = i;
    if (a.logprob) a.logprob[row] = static_cast<float>(log(w / ldexp(static_cast<double>(total), -a.shift)));
  }
}

// The instance that holds a row in LDS beside what it shares, if there is room.
template <class T, int kThreads, int kBins>
int sample_held(const Sample& a, int rows, hipStream_t st, bool* fits) {
  // from the 16 bytes that it begins in, in whole groups of eight
  const size_t lds = (static_cast<size_t>(a.vocab) + (16 / sizeof(T) - 1) + 7) / 8 * 8 * sizeof(T);
  *fits = sizeof(typename Row<T, kThreads, kBins, true>::Shared) + lds <= kLds;
  if (!*fits) return SOMA_OK;
  return launch("k_sample", k_sample<T, kThreads, kBins, true>, dim3(rows), dim3(kThreads), static_cast<unsigned>(lds), st, a);
}

template <class T>
int sample_as(const Sample& a, int rows, hipStream_t st) {
  if (a.vocab <= kFew) return launch("k_sample_few", k_sample_few<T>, dim3(rows), dim3(kFew), 0, st, a);
  bool fits = false;
  const int rc = a.vocab <= 4096 ? sample_held<T, 256, 512>(a, rows, st, &fits) : sample_held<T, 1024, 2048>(a, rows, st, &fits);
  if (fits) return rc;
  return launch("k_sample", k_sample<T, 1024, 2048, false>, dim3(rows), dim3(1024), 0, st, a);
}

}  // namespace
}  // namespace soma

using namespace soma;

extern "C" {

int soma_sample(const soma_sample_config* cfg, const void* logits, const float* u, const float* temperature,
                const int32_t* top_k, const float* top_p, const float* min_p, int32_t* tokens, float* logprob, void* stream) {
  if (!cfg) return set_error(SOMA_EINVAL, "cfg is NULL");
  const soma_sample_config& c = *cfg;
  if (c.reserved) return set_error(SOMA_EINVAL, "reserved must be 0");
  if (!is_type(c.type)) return set_error(SOMA_EINVAL, "type %d is none of enum soma_type", c.type);
  if (c.rows < 0 || c.rows > (1 << 20)) return set_error(SOMA_ESHAPE, "rows %d is out of range", c.rows);
  if (c.vocab < 1 || c.vocab > (1 << 20)) return set_error(SOMA_ESHAPE, "vocab %d is out of range", c.vocab);
  if (c.logit_stride < c.vocab || c.logit_stride > (int64_t{1} << 32)) return set_error(SOMA_ESHAPE, "logit_stride is out of range");
  if (c.rows > 0 && (!logits || !u || !tokens)) return set_error(SOMA_EINVAL, "NULL device pointer");
  if (!is_aligned(logits, type_size(c.type)) || !is_aligned(u, 4) || !is_aligned(temperature, 4) || !is_aligned(top_k, 4) ||
      !is_aligned(top_p, 4) || !is_aligned(min_p, 4) || !is_aligned(tokens, 4) || !is_aligned(logprob, 4))
    return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  const auto of_rows = [&](const void* p) { return span_of(p, c.rows, 1, 1, 4); };
  if (!are_apart({of_rows(tokens), of_rows(logprob)},
                 {span_of(logits, c.rows, c.vocab, c.logit_stride, type_size(c.type)), of_rows(u), of_rows(temperature),
                  of_rows(top_k), of_rows(top_p), of_rows(min_p)}))
    return set_error(SOMA_EINVAL, "an output overlaps another array");
  if (c.rows == 0) return set_ok();
  int bits = 0;
  while ((1 << bits) < c.vocab) ++bits;
  const Sample a{logits, c.logit_stride, u, temperature, top_p, min_p, top_k, tokens, logprob, c.vocab, 62 - bits};
  if (int rc = c.type == SOMA_FLOAT ? sample_as<float>(a, c.rows, stream_of(stream)) : sample_as<bf16>(a, c.rows, stream_of(stream)))
    return rc;
  return set_ok();
}

}  // extern "C"
