// soma_sample.hip -- the next token of every row of logits: temperature, top-k, top-p
// and min-p, from given random numbers.
//
// A block takes one row.  Nothing is sorted: what the filters keep is every token whose
// logit is above a threshold and, of those equal to it, the first few by index.  The
// thresholds come from histograms of the logits' bits, in the order of their values,
// of the number and the weight of tokens: 11 bits at a time, each time in the bin that
// holds the border.  Weights are integers (fp64 exponentials times 2^s), so that their
// sums do not depend on the order in which LDS's atomics add them up.  Then the waves
// sum what is kept in consecutive pieces of the row, and the one whose piece holds the
// token looks for it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "soma.h"
#include "soma_host.hpp"
#include "soma_types.hpp"

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

constexpr int kBins = 2048;

template <class T, int kThreads>
struct Row {
  static constexpr int kWaves = kThreads / 64, kMine = kBins / kThreads;
  const T* x;
  int vocab, shift;
  float top;                  // the largest logit
  double per;                 // 1 / temperature

  struct Shared {
    u64 weight[kBins];
    uint32_t count[kBins];
    u64 wave_weight[kWaves];
    u64 wave_count[kWaves];
    u64 found_weight, found_own;
    uint32_t found_count, found_key;
    int found;
  };
  Shared& s;

  __device__ __forceinline__ double share(float l) const {
    if (top == __builtin_huge_valf()) return l == top ? 1.0 : 0.0;
    return l == top ? 1.0 : exp((static_cast<double>(l) - static_cast<double>(top)) * per);
  }
  __device__ __forceinline__ u64 weight(double w) const { return static_cast<u64>(ldexp(w, shift) + 0.5); }

  // Tokens in front of the bin, in descending order, that crosses a border.
  struct Border {
    uint32_t bin, count, own;           // in front of it, in it
    u64 weight;                         // in front of it
    bool there;
  };

  // Histogram of bits [at, at + kBits) of the keys whose upper bits are `prefix`.
  __device__ void histogram(int at, int bits, uint32_t prefix, bool all) {
    for (int i = threadIdx.x; i < kBins; i += kThreads) s.weight[i] = 0, s.count[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < vocab; i += kThreads) {
      const float l = load_value(x + i);
      const uint32_t k = key_of<T>(l);
      if (!k || (!all && k >> (at + bits) != prefix)) continue;
      const uint32_t bin = (k >> at) & ((1u << bits) - 1);
      atomicAdd(&s.count[bin], 1u);
      atomicAdd(&s.weight[bin], weight(share(l)));
    }
    __syncthreads();
  }

  // The bin where the tokens in front become `k` or more (by_count), or their weight
  // `limit`; count0 and weight0 lie in front of all bins.  total: all bins' weight.
  __device__ Border find(bool by_count, u64 k, u64 limit, uint32_t count0, u64 weight0, u64* total) {
    u64 c[kMine], w[kMine], cs = 0, ws = 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int bin = kBins - 1 - (static_cast<int>(threadIdx.x) * kMine + i);
      c[i] = s.count[bin], w[i] = s.weight[bin];
      cs += c[i], ws += w[i];
    }
    u64 call, wall;
    u64 cb = wave_before(cs, &call), wb = wave_before(ws, &wall);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) s.wave_count[wave] = call, s.wave_weight[wave] = wall;
    if (threadIdx.x == 0) s.found = 0;
    __syncthreads();
    u64 sum = 0;
    for (int i = 0; i < kWaves; ++i) {
      if (i < wave) cb += s.wave_count[i], wb += s.wave_weight[i];
      sum += s.wave_weight[i];
    }
    if (total) *total = sum;
    cb += count0, wb += weight0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const bool here = c[i] && (by_count ? cb < k && cb + c[i] >= k : wb < limit && wb + w[i] >= limit);
      if (here) {
        s.found = 1;
        s.found_key = kBins - 1 - (threadIdx.x * kMine + i);
        s.found_count = static_cast<uint32_t>(cb), s.found_own = c[i], s.found_weight = wb;
      }
      cb += c[i], wb += w[i];
    }
    __syncthreads();
    Border b{s.found_key, s.found_count, static_cast<uint32_t>(s.found_own), s.found_weight, s.found != 0};
    __syncthreads();
    return b;
  }

  static constexpr int kKeyBits = sizeof(T) == 2 ? 16 : 32;

  // Goes on from a bin of the first histogram to a single key.
  __device__ Border refine(Border b, bool by_count, u64 k, u64 limit, uint32_t* key) {
    uint32_t prefix = b.bin;
    int at = kKeyBits - 11;
    while (at > 0) {
      const int bits = min(at, 11);
      at -= bits;
      histogram(at, bits, prefix, false);
      b = find(by_count, k, limit, b.count, b.weight, nullptr);
      prefix = prefix << bits | b.bin;
    }
    *key = prefix;
    return b;
  }
};

template <class T, int kThreads>
__global__ __launch_bounds__(kThreads) void k_sample(const Sample a) {
  typedef Row<T, kThreads> R;
  __shared__ typename R::Shared shared;
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  R r{static_cast<const T*>(a.logits) + row * a.stride, a.vocab, a.shift, 0.0f, 1.0, shared};

  // the likeliest token
  u64 best = 0;
  for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
    const uint32_t k = key_of<T>(load_value(r.x + i));
    if (k) best = max(best, static_cast<u64>(k) << 32 | static_cast<uint32_t>(~i));
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) best = max(best, static_cast<u64>(__shfl_xor(best, d)));
  if (lane == 0) shared.wave_weight[wave] = best;
  __syncthreads();
  for (int w = 0; w < R::kWaves; ++w) best = max(best, shared.wave_weight[w]);
  __syncthreads();
  const float temperature = a.temperature ? a.temperature[row] : 1.0f;
  if (best == 0 || !(temperature > 0.0f)) {
    if (threadIdx.x == 0) {
      a.tokens[row] = best ? static_cast<int32_t>(~static_cast<uint32_t>(best)) : -1;
      if (a.logprob) a.logprob[row] = best ? 0.0f : -__builtin_huge_valf();
    }
    return;
  }
  r.top = value_of<T>(static_cast<uint32_t>(best >> 32));
  r.per = 1.0 / static_cast<double>(temperature);

  const int32_t top_k = a.top_k ? a.top_k[row] : 0;
  const float top_p = a.top_p ? a.top_p[row] : 1.0f;
  const float least = a.min_p ? a.min_p[row] : 0.0f;
  const double min_p = least > 0.0f ? fmin(static_cast<double>(least), 1.0) : 0.0;
  const bool by_k = top_k > 0 && top_k < a.vocab, by_p = top_p < 1.0f;
  // kept: keys above `key`, and the first `ties` of those equal to it
  uint32_t key = 0, ties = 0;
  bool all_ties = true;
  if (by_k || by_p) {
    r.histogram(R::kKeyBits - 11, 11, 0, true);
    u64 total = 0;
    typename R::Border b{};
    if (by_k) {
      b = r.find(true, top_k, 0, 0, 0, &total);
      if (b.there) {
        b = r.refine(b, true, top_k, 0, &key);
        ties = top_k - b.count;
        all_ties = ties >= b.own;
        total = b.weight + ties * r.weight(r.share(value_of<T>(key)));
        if (by_p) r.histogram(R::kKeyBits - 11, 11, 0, true);
      }
    }
    if (by_p) {
      u64 sum = 0;
      if (!by_k) {
        r.find(false, 0, ~0ull, 0, 0, &sum);
        total = sum;
      }
      const double p = fmax(static_cast<double>(top_p), 0.0);
      const u64 limit = min(max(static_cast<u64>(ceil(p * static_cast<double>(total))), u64{1}), total);
      b = r.find(false, 0, limit, 0, 0, nullptr);
      if (b.there) {
        b = r.refine(b, false, 0, limit, &key);
        const u64 own = r.weight(r.share(value_of<T>(key)));
        ties = static_cast<uint32_t>((limit - b.weight + own - 1) / own);
        all_ties = ties >= b.own;
      }
    }
  }

  // consecutive pieces of the row, a wave each
  const int piece = (a.vocab + R::kWaves * 64 - 1) / (R::kWaves * 64) * 64;
  const int from = min(wave * piece, a.vocab), to = min(from + piece, a.vocab);
  int last = a.vocab;                       // ties are kept up to here
  if (!all_ties) {
    uint32_t n = 0;
    for (int i = from; i < to; i += 64)
      n += __popcll(__builtin_amdgcn_ballot_w64(i + lane < to && key_of<T>(load_value(r.x + i + lane)) == key));
    if (lane == 0) shared.wave_count[wave] = n;
    __syncthreads();
    u64 before = 0;
    for (int w = 0; w < wave; ++w) before += shared.wave_count[w];
    if (before < ties && before + n >= ties) {
      uint32_t left = ties - static_cast<uint32_t>(before);
      for (int i = from; i < to; i += 64) {
        const u64 here = __builtin_amdgcn_ballot_w64(i + lane < to && key_of<T>(load_value(r.x + i + lane)) == key);
        const uint32_t m = __popcll(here);
        if (m >= left) {
          // the lane with left - 1 ties in front of it
          const bool mine = (here >> lane & 1) && __popcll(here & ((1ull << lane) - 1)) + 1 == left;
          if (mine) shared.found = i + lane;
          break;
        }
        left -= m;
      }
    }
    __syncthreads();
    last = shared.found;
    __syncthreads();
  }
  const auto kept = [&](int i) -> u64 {
    if (i >= to) return 0;
    const float l = load_value(r.x + i);
    const uint32_t k = key_of<T>(l);
    if (!k || k < key || (k == key && i > last)) return 0;
    const double w = r.share(l);
    return w >= min_p ? r.weight(w) : 0;
  };
  u64 sum = 0, all;
  for (int i = from; i < to; i += 64) sum += kept(i + lane);
  wave_before(sum, &all);
  if (lane == 0) shared.wave_weight[wave] = all;
  __syncthreads();
  u64 before = 0, total = 0;
  for (int w = 0; w < R::kWaves; ++w) {
    if (w < wave) before += shared.wave_weight[w];
    total += shared.wave_weight[w];
  }
  const float u = a.u[row];
  const double target = fmin(fmax(static_cast<double>(u), 0.0), 1.0) * static_cast<double>(total);
  u64 goal = min(static_cast<u64>(target), total - 1);
  if (before <= goal && goal < before + all) {
    goal -= before;
    for (int i = from; i < to; i += 64) {
      const u64 w = kept(i + lane);
      u64 here;
      const u64 front = wave_before(w, &here);
      if (goal < here) {
        if (w && front <= goal && goal < front + w) {
          a.tokens[row] = i + lane;
          if (a.logprob)
            a.logprob[row] = static_cast<float>(log(r.share(load_value(r.x + i + lane)) / ldexp(static_cast<double>(total), -a.shift)));
        }
        break;
      }
      goal -= here;
    }
  }
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
  const bool small = c.vocab <= 4096;
  const auto kernel = c.type == SOMA_FLOAT ? (small ? k_sample<float, 256> : k_sample<float, 1024>)
                                           : (small ? k_sample<bf16, 256> : k_sample<bf16, 1024>);
  if (int rc = launch("k_sample", kernel, dim3(c.rows), dim3(small ? 256 : 1024), 0, stream_of(stream), a)) return rc;
  return set_ok();
}

}  // extern "C"
