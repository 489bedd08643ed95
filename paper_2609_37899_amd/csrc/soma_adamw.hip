// soma_adamw.hip -- one AdamW step over many tensors in one launch.
//
//   g = scale * grad;  m <- beta1 m + (1 - beta1) g;  v <- beta2 v + (1 - beta2) g^2
//   p <- (1 - lr decay) p - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + delta)
//
// in fp32 whatever the tensors' types, one rounding for every operation (no
// contraction; but see adamw_ordinary), p rounded once to its own type.
//
// Moments in 8 bits.  256 consecutive elements share two fp32 scales.  m is an
// e4m3 code times (largest |m| / 448).  v is kept as its square root, which
// halves the range of exponents: 4 bits of exponent and 4 of mantissa, code k
// in 1 .. 255 standing for (16 + k % 16) 2^(k / 16 - 19), code 0 for 0, times
// (largest root / 1.9375).  Both are rounded to nearest even.  A root that is
// not 0 keeps at least code 1 (3.4e-5 of the block's largest), so that no
// element's step is divided by delta alone; a first moment below 2^-10 of
// e4m3's unit (2.2e-6 of the block's largest) becomes 0.  The update of p uses
// the new moments before their rounding.
//
// To nearest, an update of less than half a code is lost, at every step again: with
// beta2 = 0.999 v moves by a thousandth of its distance to g^2, its codes lie 6 to
// 12% apart, so that an element falls only as its block's largest does.  (One element
// of 256 keeps its gradient, the others' fall tenfold: their root is 7.8 times too
// large after 5,000 updates.)  Random rounding (random_codes) keeps either neighbour
// with the probability that makes the expected value the exact one, so the average of
// many steps is followed; a word of Philox for each element serves it, drawn from the
// element, its tensor and the number of the update.
//
// The step is bound by memory: every element is read and written once.  A
// block takes 4096 consecutive elements of one tensor (a table of blocks, made
// once with the plan, names the tensor), a wave 256 of them at a time, four a
// lane: 16-byte accesses to fp32, and the 256 elements that share a scale are
// one wave's, whose two maxima never leave its registers.  With 8-bit moments
// the operations would bound it (387 us where the bytes take 234): blocks of
// ordinary values go a way of their own, with half of them.
//
// Measured: 24 tensors of 40 M fp32 elements in all, moments of 32 bits: 217 us,
// 5.2 TB/s, as fast as a copy.  400 tensors of 120 M bf16 elements, moments of 8
// bits: 238 us (5.0 TB/s), their values in fp32 240 us (5.0 TB/s).  Steps of the same
// back to back take 272 us, rounded at random 343 (operations bound it: Philox is 40
// multiplications for four elements); with fp32 parameters and gradients 365 and 389.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "soma.h"
#include "soma_host.hpp"
#include "soma_rng.hpp"
#include "soma_types.hpp"

namespace soma {
namespace {

constexpr int kStateBlock = 256;      // elements that share the scales of 8-bit moments
constexpr int kChunk = 4096;          // elements of one block
// The same where such blocks would be fewer than four for each compute unit: a wave
// has 256 elements then, and waits for memory once (131,000 elements: 3.9 us, with
// blocks of 4096 6.8).
constexpr int kSmallChunk = 1024, kSmallBlocks = 1024;
constexpr int kThreadsAdamw = 256;
constexpr int kRounds = kChunk / (4 * kThreadsAdamw);
constexpr float kTopM = 448.0f;       // the largest e4m3 value
constexpr float kTopRoot = 1.9375f;   // the largest value of a root's code
constexpr int kRootBias = 112 << 4;   // code + kRootBias: the upper 12 bits of the fp32 value's magnitude

struct Tensor {
  void* param;
  const void* grad;
  void *m, *v;
  float *m_scale, *v_scale;
  void* copy;
  int64_t count;
  double decay;
  int32_t kind;      // 4 (param is bf16) + 2 (grad is bf16) + 1 (moments in 8 bits)
  int32_t wide;      // every pointer allows accesses to four elements at once
};

struct Block {
  int32_t tensor, chunk;
};

struct Rates {
  float beta1, omb1, beta2, omb2, size, root, delta;
  int32_t ordinary;  // root and delta are at most 2^30
  int32_t chunk;     // elements of one block
  double lr;
};

// Random rounding: Philox's key and the update's part of its counter, the tensor.
struct Draw {
  uint2 key;
  uint32_t t, tensor;
};

// A block's scale from its largest magnitude, and the factor that brings its
// values onto the code's range (0 for a block of zeros, or one whose largest
// has no finite factor).
__device__ __forceinline__ float code_factor(float top, float largest) {
  return top > 1e-35f ? largest * (1.0f / top) : 0.0f;
}

__device__ __forceinline__ uint32_t root_code(float y) {
  const uint32_t b = __float_as_uint(y) & 0x7FFFFFFFu;   // NaN may have a sign, which the sum would carry past 2^32
  int k = static_cast<int>((b + 0x3FFFFu + ((b >> 19) & 1u)) >> 19) - kRootBias;
  k = k < 1 ? 1 : (k > 255 ? 255 : k);    // NaN and infinity: 255
  return y == 0.0f ? 0u : static_cast<uint32_t>(k);
}

__device__ __forceinline__ float root_value(uint32_t k) {
  return k ? __uint_as_float((k + kRootBias) << 19) : 0.0f;
}

// e4m3 code of y, |y| <= 448 up to a rounding; NaN for what is not finite.
__device__ __forceinline__ uint32_t e4m3_four(const float (&y)[4]) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  uint32_t u = static_cast<uint32_t>(w);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (!(__builtin_fabsf(y[i]) < 1e30f)) u |= 0x7Fu << (8 * i);
  return u;
}

template <int kByte>
__device__ __forceinline__ float e4m3_value(uint32_t w) {
  return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(w), kByte);
}

// Random rounding of four elements from element `at` on, a multiple of four.  Each has a
// word of Philox4x32-10 with key stream_key(seed, t), counter (lo32(at / 4), tensor,
// lo32(t), hi32(at / 4)): its upper 20 bits are v's draw, the lower 12 m's, both at the
// middle of their interval, (draw + 1/2) 2^-20 and 2^-12.

// y, |y| <= 448 up to a rounding, to one of the two e4m3 values beside it, away from 0
// if the draw is below (|y| - lower) / (upper - lower).  Below 2^-6 the steps are
// 2^-9, as they are in [2^-6, 2^-5): the value is moved there and back.
__device__ __forceinline__ float random_e4m3(float y, uint32_t draw) {
  const float a = __builtin_fabsf(y), shift = a < 0x1p-6f ? 0x1p-6f : 0.0f;
  const uint32_t b = (__float_as_uint(a + shift) + 0xFFFFFu - (draw * 256u + 128u)) & ~0xFFFFFu;
  return __builtin_copysignf(fminf(__uint_as_float(b) - shift, kTopM), y);
}

// The code of one of the two roots beside y, the larger one if the draw is below
// (y^2 - lower^2) / (larger^2 - lower^2): it is v, the square, whose expected value
// stays.  As to nearest, what is not 0 keeps code 1, and NaN and infinity have 255.
__device__ __forceinline__ uint32_t random_root_code(float y, uint32_t draw) {
  const uint32_t b = __float_as_uint(y) & 0x7FFFFFFFu, low = b & ~0x7FFFFu;
  const float y0 = __uint_as_float(low), y1 = __uint_as_float(low + 0x80000u);
  const float u = static_cast<float>(2u * draw + 1u) * 0x1p-21f;
  int k = static_cast<int>(b >> 19) - kRootBias + (u * ((y1 - y0) * (y1 + y0)) < (y - y0) * (y + y0) ? 1 : 0);
  k = k < 1 ? 1 : (k > 255 ? 255 : k);
  return y == 0.0f ? 0u : static_cast<uint32_t>(k);
}

// ym: m over its scale, left rounded to e4m3's values; yr: the roots over theirs.
// Returns the roots' codes.
__device__ __forceinline__ uint32_t random_codes(const Draw& d, int64_t at, float (&ym)[4], const float (&yr)[4]) {
  const uint64_t q = static_cast<uint64_t>(at) >> 2;
  const uint4 x = philox4x32_10(make_uint4(static_cast<uint32_t>(q), d.tensor, d.t, static_cast<uint32_t>(q >> 32)), d.key);
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float r = random_e4m3(ym[i], w[i] & 0xFFFu);
    ym[i] = __builtin_fabsf(ym[i]) < 1e30f ? r : ym[i];
    codes |= random_root_code(yr[i], w[i] >> 12) << (8 * i);
  }
  return codes;
}

// Largest finite magnitude of four.
__device__ __forceinline__ float finite_max(const float (&x)[4]) {
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = __builtin_fabsf(x[i]);
    top = a <= 3.402823466e38f && a > top ? a : top;
  }
  return top;
}

// sqrt(x) for x in [2^-96, 2^90], to nearest but for about one in a million, off by
// one last bit there: x rsq(x) and one step towards x.
__device__ __forceinline__ float ordinary_root(float x) {
  const float y = __builtin_amdgcn_rsqf(x), s = x * y;
  return __builtin_fmaf(__builtin_fmaf(-s, s, x), 0.5f * y, s);
}

// 1 / x, to nearest but for as few, x well inside the range.
__device__ __forceinline__ float ordinary_inverse(float x) {
  const float y = __builtin_amdgcn_rcpf(x);
  return __builtin_fmaf(__builtin_fmaf(-x, y, 1.0f), y, y);
}

// Four consecutive values as they lie in memory.
template <class T>
struct Four;
template <>
struct Four<float> {
  typedef float4 Raw;
  static __device__ __forceinline__ Raw load(const float* p) { return *reinterpret_cast<const float4*>(p); }
  static __device__ __forceinline__ void values(const Raw& u, float (&x)[4]) { x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w; }
};
template <>
struct Four<bf16> {
  typedef uint2 Raw;
  static __device__ __forceinline__ Raw load(const bf16* p) { return *reinterpret_cast<const uint2*>(p); }
  static __device__ __forceinline__ void values(const Raw& u, float (&x)[4]) {
    x[0] = __uint_as_float(u.x << 16), x[1] = __uint_as_float(u.x & 0xFFFF0000u);
    x[2] = __uint_as_float(u.y << 16), x[3] = __uint_as_float(u.y & 0xFFFF0000u);
  }
};

template <class T>
__device__ __forceinline__ void load_lane(const T* p, int64_t at, int n, bool wide, float (&x)[4]) {
  if (wide && n >= 4) {
    const float4 v = load_four(p + at);
    x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < n ? load_value(p + at + i) : 0.0f;
  }
}

template <class T>
__device__ __forceinline__ void store_lane(T* p, int64_t at, int n, bool wide, const float (&x)[4]) {
  if (wide && n >= 4) {
    store_four(p + at, make_float4(x[0], x[1], x[2], x[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) store_value(p + at + i, x[i]);
  }
}

__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int64_t at, int n, bool wide) {
  if (wide && n >= 4) return *reinterpret_cast<const uint32_t*>(p + at);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < n) w |= static_cast<uint32_t>(p[at + i]) << (8 * i);
  return w;
}

__device__ __forceinline__ void store_codes(uint8_t* p, int64_t at, int n, bool wide, uint32_t w) {
  if (wide && n >= 4) {
    *reinterpret_cast<uint32_t*>(p + at) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[at + i] = static_cast<uint8_t>(w >> (8 * i));
  }
}

__device__ __forceinline__ void decode(uint32_t mw, uint32_t vw, float ms, float vs, float (&m)[4], float (&v)[4]) {
  m[0] = e4m3_value<0>(mw) * ms, m[1] = e4m3_value<1>(mw) * ms, m[2] = e4m3_value<2>(mw) * ms,
  m[3] = e4m3_value<3>(mw) * ms;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float r = root_value((vw >> (8 * i)) & 255u) * vs;
    v[i] = r * r;
  }
}

// The wave's 256 elements from `block` on, any length and alignment.
template <class P, class G, bool kBytes, bool kRandom>
__device__ __forceinline__ void adamw_round(const Tensor& t, int64_t block, const Rates& r, const Draw& d, float scale,
                                            float keep) {
  const int lane = threadIdx.x & 63;
  const bool wide = t.wide != 0;
  P* const param = static_cast<P*>(t.param);
  const int64_t at = block + lane * 4;
  const int64_t left = t.count - at;
  const int n = left < 4 ? static_cast<int>(left) : 4;          // may be negative
  float p[4], g[4], m[4], v[4];
  load_lane(param, at, n, wide, p);
  load_lane(static_cast<const G*>(t.grad), at, n, wide, g);
  if constexpr (kBytes) {
    const int64_t s = block / kStateBlock;
    decode(load_codes(static_cast<const uint8_t*>(t.m), at, n, wide),
           load_codes(static_cast<const uint8_t*>(t.v), at, n, wide), t.m_scale[s], t.v_scale[s], m, v);
  } else {
    load_lane(static_cast<const float*>(t.m), at, n, wide, m);
    load_lane(static_cast<const float*>(t.v), at, n, wide, v);
  }
  float root[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float gi = g[i] * scale;
    m[i] = r.beta1 * m[i] + r.omb1 * gi;
    v[i] = r.beta2 * v[i] + r.omb2 * (gi * gi);
    root[i] = sqrtf(v[i]);
    p[i] = p[i] * keep - r.size * (m[i] / (root[i] * r.root + r.delta));
  }
  store_lane(param, at, n, wide, p);
  if (t.copy) store_lane(static_cast<bf16*>(t.copy), at, n, wide, p);
  if constexpr (kBytes) {
    if (n < 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i >= n) m[i] = 0.0f, root[i] = 0.0f;
    }
    const float top_m = wave_max(finite_max(m)), top_r = wave_max(finite_max(root));
    const float fm = code_factor(top_m, kTopM), fr = code_factor(top_r, kTopRoot);
    float y[4];
    uint32_t vw = 0;
    if constexpr (kRandom) {
      float yr[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = m[i] * fm, yr[i] = root[i] * fr;
      vw = random_codes(d, at, y, yr);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[i] = m[i] * fm;
        vw |= root_code(root[i] * fr) << (8 * i);
      }
    }
    store_codes(static_cast<uint8_t*>(t.m), at, n, wide, e4m3_four(y));
    store_codes(static_cast<uint8_t*>(t.v), at, n, wide, vw);
    if (lane == 0) {
      const int64_t s = block / kStateBlock;
      t.m_scale[s] = top_m * (1.0f / kTopM);
      t.v_scale[s] = top_r * (1.0f / kTopRoot);
    }
  } else {
    store_lane(static_cast<float*>(t.m), at, n, wide, m);
    store_lane(static_cast<float*>(t.v), at, n, wide, v);
  }
}

// 256 whole, aligned elements with moments in 8 bits, as they were loaded.
template <class P, class G>
struct RawBytes {
  typename Four<P>::Raw p;
  typename Four<G>::Raw g;
  uint32_t m, v;
  float m_scale, v_scale;

  __device__ __forceinline__ void load(const Tensor& t, int64_t block) {
    const int64_t at = block + (threadIdx.x & 63) * 4, s = block / kStateBlock;
    p = Four<P>::load(static_cast<const P*>(t.param) + at);
    g = Four<G>::load(static_cast<const G*>(t.grad) + at);
    m = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.m) + at);
    v = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.v) + at);
    m_scale = t.m_scale[s], v_scale = t.v_scale[s];
  }
};

// The same results as adamw_round's (p's to 3 roundings of its step) where the
// values are ordinary, and false, with nothing written, where they are not: a code
// or a value of 0 in v, v outside [2^-96, 2^90], m not finite or above 2^100 in
// any of the 256.  In those ranges nothing is subnormal, infinite or NaN, so the
// root, the quotients and the codes need none of the steps that look for it: 54
// operations for each element where there were 100.
template <class P, class G, bool kRandom>
__device__ __forceinline__ bool adamw_ordinary(const Tensor& t, int64_t block, const Rates& r, const Draw& d, float scale,
                                               float keep, const RawBytes<P, G>& raw) {
  const int lane = threadIdx.x & 63;
  float p[4], g[4], m[4], v[4];
  Four<P>::values(raw.p, p);
  Four<G>::values(raw.g, g);
  m[0] = e4m3_value<0>(raw.m) * raw.m_scale, m[1] = e4m3_value<1>(raw.m) * raw.m_scale;
  m[2] = e4m3_value<2>(raw.m) * raw.m_scale, m[3] = e4m3_value<3>(raw.m) * raw.m_scale;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float root = __uint_as_float((((raw.v >> (8 * i)) & 255u) + kRootBias) << 19) * raw.v_scale;
    v[i] = root * root;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float gi = g[i] * scale;
    m[i] = r.beta1 * m[i] + r.omb1 * gi;
    v[i] = r.beta2 * v[i] + r.omb2 * (gi * gi);
  }
  // A sum is NaN if one of its terms is.
  const float sum_m = __builtin_fabsf(m[0]) + __builtin_fabsf(m[1]) + __builtin_fabsf(m[2]) + __builtin_fabsf(m[3]);
  const float sum_v = v[0] + v[1] + v[2] + v[3], low = fminf(fminf(v[0], v[1]), fminf(v[2], v[3]));
  const bool zero = ((raw.v - 0x01010101u) & ~raw.v & 0x80808080u) != 0;
  const float top_m = wave_max(fmaxf(fmaxf(__builtin_fabsf(m[0]), __builtin_fabsf(m[1])),
                                     fmaxf(__builtin_fabsf(m[2]), __builtin_fabsf(m[3]))));
  const bool ordinary = !zero && sum_m <= 0x1p100f && sum_v <= 0x1p90f && low >= 0x1p-96f && top_m >= 0x1p-96f;
  if (__builtin_amdgcn_ballot_w64(ordinary) != ~uint64_t(0)) return false;
  float root[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    root[i] = ordinary_root(v[i]);
    p[i] = p[i] * keep - r.size * (m[i] * __builtin_amdgcn_rcpf(root[i] * r.root + r.delta));
  }
  const float top_r = wave_max(fmaxf(fmaxf(root[0], root[1]), fmaxf(root[2], root[3])));
  const float fm = kTopM * ordinary_inverse(top_m), fr = kTopRoot * ordinary_inverse(top_r);
  const int64_t at = block + lane * 4;
  float y[4];
  uint32_t vw = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = m[i] * fm;
  if constexpr (kRandom) {
    float yr[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) yr[i] = root[i] * fr;
    vw = random_codes(d, at, y, yr);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t b = __float_as_uint(root[i] * fr);
      // negative codes are wanted: what is below code 1 becomes 1
      const int k = static_cast<int>(b + ((b >> 19) & 1u) + (0x3FFFFu - (uint32_t(kRootBias) << 19))) >> 19;
      vw |= static_cast<uint32_t>(k < 1 ? 1 : k) << (8 * i);
    }
  }
  int mw = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  mw = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], mw, true);
  store_four(static_cast<P*>(t.param) + at, make_float4(p[0], p[1], p[2], p[3]));
  if (t.copy) store_four(static_cast<bf16*>(t.copy) + at, make_float4(p[0], p[1], p[2], p[3]));
  *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.m) + at) = static_cast<uint32_t>(mw);
  *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.v) + at) = vw;
  if (lane == 0) {
    const int64_t s = block / kStateBlock;
    t.m_scale[s] = top_m * (1.0f / kTopM);
    t.v_scale[s] = top_r * (1.0f / kTopRoot);
  }
  return true;
}

template <class P, class G, bool kBytes, bool kRandom>
__device__ __forceinline__ void adamw_chunk(const Tensor& t, int64_t first, const Rates& r, const Draw& d, float scale) {
  const int wave = threadIdx.x >> 6;
  const float keep = static_cast<float>(1.0 - r.lr * t.decay);
  first += wave * kStateBlock;
  if constexpr (kBytes) {
    // Whole chunks: the loads of all four rounds are on their way at once.
    if (t.wide && r.ordinary && r.chunk == kChunk && first - wave * kStateBlock + kChunk <= t.count) {
      RawBytes<P, G> raw[kRounds];
#pragma unroll
      for (int k = 0; k < kRounds; ++k) raw[k].load(t, first + k * 4 * kStateBlock);
#pragma unroll
      for (int k = 0; k < kRounds; ++k)
        if (!adamw_ordinary<P, G, kRandom>(t, first + k * 4 * kStateBlock, r, d, scale, keep, raw[k]))
          adamw_round<P, G, true, kRandom>(t, first + k * 4 * kStateBlock, r, d, scale, keep);
      return;
    }
  }
  const int64_t end = min(t.count, first + r.chunk);
#pragma unroll 2
  for (int k = 0; k < kRounds; ++k) {
    const int64_t block = first + k * 4 * kStateBlock;            // the wave's 256 elements
    if (block >= end) break;                                      // wave-uniform
    adamw_round<P, G, kBytes, kBytes && kRandom>(t, block, r, d, scale, keep);
  }
}

template <bool kRandom>
__global__ __launch_bounds__(kThreadsAdamw) void k_adamw(const Tensor* tensors, const Block* blocks, Rates r, Draw d,
                                                         const float* grad_scale) {
  const Block b = blocks[blockIdx.x];
  const Tensor t = tensors[b.tensor];
  const float scale = grad_scale ? *grad_scale : 1.0f;
  const int64_t first = int64_t(b.chunk) * r.chunk;
  d.tensor = b.tensor;
  switch (t.kind) {
    case 0: adamw_chunk<float, float, false, kRandom>(t, first, r, d, scale); break;
    case 1: adamw_chunk<float, float, true, kRandom>(t, first, r, d, scale); break;
    case 2: adamw_chunk<float, bf16, false, kRandom>(t, first, r, d, scale); break;
    case 3: adamw_chunk<float, bf16, true, kRandom>(t, first, r, d, scale); break;
    case 4: adamw_chunk<bf16, float, false, kRandom>(t, first, r, d, scale); break;
    case 5: adamw_chunk<bf16, float, true, kRandom>(t, first, r, d, scale); break;
    case 6: adamw_chunk<bf16, bf16, false, kRandom>(t, first, r, d, scale); break;
    default: adamw_chunk<bf16, bf16, true, kRandom>(t, first, r, d, scale); break;
  }
}

// The moments' values, in fp32.  The outputs' addresses travel with the
// launch, kOutputs tensors at a time.
constexpr int kOutputs = 200;
struct Outputs {
  float *m[kOutputs], *v[kOutputs];
};

__global__ __launch_bounds__(kThreadsAdamw) void k_adamw_moments(const Tensor* tensors, const Block* blocks, int first_tensor,
                                                                 int chunk, Outputs out) {
  const Block b = blocks[blockIdx.x];
  const Tensor t = tensors[b.tensor];
  float* const mo = out.m[b.tensor - first_tensor];
  float* const vo = out.v[b.tensor - first_tensor];
  const bool wide = t.wide && reinterpret_cast<uintptr_t>(mo) % 16 == 0 && reinterpret_cast<uintptr_t>(vo) % 16 == 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t first = int64_t(b.chunk) * chunk + wave * kStateBlock;
  if (wide && (t.kind & 1) && chunk == kChunk && first - wave * kStateBlock + kChunk <= t.count) {
    // Whole chunks: the loads of all four rounds are on their way at once.
    uint32_t mw[kRounds], vw[kRounds];
    float ms[kRounds], vs[kRounds];
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
      const int64_t block = first + k * 4 * kStateBlock, s = block / kStateBlock;
      mw[k] = reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.m) + block)[lane];
      vw[k] = reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.v) + block)[lane];
      ms[k] = t.m_scale[s], vs[k] = t.v_scale[s];
    }
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
      const int64_t at = first + k * 4 * kStateBlock + lane * 4;
      float m[4], v[4];
      decode(mw[k], vw[k], ms[k], vs[k], m, v);
      store_four(mo + at, make_float4(m[0], m[1], m[2], m[3]));
      store_four(vo + at, make_float4(v[0], v[1], v[2], v[3]));
    }
    return;
  }
  const int64_t end = min(t.count, first + chunk);
#pragma unroll 2
  for (int k = 0; k < kRounds; ++k) {
    const int64_t block = first + k * 4 * kStateBlock;
    if (block >= end) break;
    const int64_t at = block + lane * 4, left = t.count - at;
    const int n = left < 4 ? static_cast<int>(left) : 4;
    float m[4], v[4];
    if (t.kind & 1) {
      const int64_t s = block / kStateBlock;
      decode(load_codes(static_cast<const uint8_t*>(t.m), at, n, wide),
             load_codes(static_cast<const uint8_t*>(t.v), at, n, wide), t.m_scale[s], t.v_scale[s], m, v);
    } else {
      load_lane(static_cast<const float*>(t.m), at, n, wide, m);
      load_lane(static_cast<const float*>(t.v), at, n, wide, v);
    }
    store_lane(mo, at, n, wide, m);
    store_lane(vo, at, n, wide, v);
  }
}

int64_t chunks_of(int64_t count, int chunk) { return (count + chunk - 1) / chunk; }

int check_tensors(const soma_adamw_tensor* x, int32_t n, int* chunk, int64_t* chunks) {
  if (!x || n < 1) return set_error(SOMA_EINVAL, "no tensors");
  *chunks = 0;
  for (int32_t i = 0; i < n; ++i) {
    const soma_adamw_tensor& t = x[i];
    if (t.count < 0 || t.count > (int64_t(1) << 42)) return set_error(SOMA_ESHAPE, "tensor %d: bad count", i);
    if (!is_type(t.param_type) || !is_type(t.grad_type)) return set_error(SOMA_EINVAL, "tensor %d: unknown type", i);
    if (t.state_bits != 8 && t.state_bits != 32)
      return set_error(SOMA_EINVAL, "tensor %d: moments are held in 32 or in 8 bits", i);
    if (!std::isfinite(t.weight_decay)) return set_error(SOMA_EINVAL, "tensor %d: weight_decay must be finite", i);
    if (t.count > 0) {
      if (!t.param || !t.grad || !t.m || !t.v || (t.state_bits == 8 && (!t.m_scale || !t.v_scale)))
        return set_error(SOMA_EINVAL, "tensor %d: NULL device pointer", i);
      const size_t state = t.state_bits == 8 ? 1 : 4;
      if (!is_aligned(t.param, type_size(t.param_type)) || !is_aligned(t.grad, type_size(t.grad_type)) ||
          !is_aligned(t.m, state) || !is_aligned(t.v, state) || !is_aligned(t.m_scale, 4) ||
          !is_aligned(t.v_scale, 4) || !is_aligned(t.copy, 2))
        return set_error(SOMA_EINVAL, "tensor %d: a pointer is not aligned to its elements", i);
    }
    *chunks += chunks_of(t.count, kChunk);
  }
  *chunk = kChunk;
  if (*chunks < kSmallBlocks) {
    *chunk = kSmallChunk, *chunks = 0;
    for (int32_t i = 0; i < n; ++i) *chunks += chunks_of(x[i].count, kSmallChunk);
  }
  if (*chunks > (int64_t(1) << 30)) return set_error(SOMA_ESHAPE, "more than 2^42 elements");
  return SOMA_OK;
}

struct Range {
  uintptr_t at, end;
  bool written;
};

// Whether an array that the step writes overlaps another (two tensors' blocks run
// at the same time).
int check_apart(const soma_adamw_tensor* x, int32_t n) {
  Range* const r = new (std::nothrow) Range[7 * size_t(n)];
  if (!r) return set_error(SOMA_EINVAL, "out of host memory");
  size_t k = 0;
  for (int32_t i = 0; i < n; ++i) {
    const soma_adamw_tensor& t = x[i];
    if (t.count == 0) continue;
    const size_t count = size_t(t.count), blocks = (count + kStateBlock - 1) / kStateBlock;
    const bool bytes = t.state_bits == 8;
    const auto add = [&](const void* p, size_t n_bytes, bool written) {
      if (p) r[k++] = Range{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + n_bytes, written};
    };
    add(t.param, count * type_size(t.param_type), true);
    add(t.grad, count * type_size(t.grad_type), false);
    add(t.m, count * (bytes ? 1 : 4), true);
    add(t.v, count * (bytes ? 1 : 4), true);
    if (bytes) add(t.m_scale, blocks * 4, true), add(t.v_scale, blocks * 4, true);
    add(t.copy, count * 2, true);
  }
  std::sort(r, r + k, [](const Range& a, const Range& b) { return a.at < b.at; });
  uintptr_t read_end = 0, written_end = 0;
  bool apart = true;
  for (size_t i = 0; i < k; ++i) {
    apart = apart && r[i].at >= written_end && (!r[i].written || r[i].at >= read_end);
    uintptr_t& end = r[i].written ? written_end : read_end;
    end = std::max(end, r[i].end);
  }
  delete[] r;
  return apart ? SOMA_OK : set_error(SOMA_EINVAL, "two arrays of the plan overlap");
}

size_t table_bytes(int32_t n) { return up256(size_t(n) * sizeof(Tensor)); }

}  // namespace
}  // namespace soma

struct soma_adamw {
  int32_t n, chunk;
  int64_t chunks;
  const soma::Tensor* tensors;       // device
  const soma::Block* blocks;         // device
  int64_t* first_chunk;              // host, [n + 1]
  int32_t rounding;                  // enum soma_rounding
  uint64_t seed;
};

using namespace soma;

extern "C" {

int soma_adamw_workspace_size(const soma_adamw_tensor* tensors, int32_t n, size_t* bytes) {
  int chunk = 0;
  int64_t chunks = 0;
  if (int rc = check_tensors(tensors, n, &chunk, &chunks)) return rc;
  if (!bytes) return set_error(SOMA_EINVAL, "bytes is NULL");
  *bytes = table_bytes(n) + up256(size_t(chunks) * sizeof(Block));
  return set_ok();
}

int soma_adamw_create(const soma_adamw_tensor* tensors, int32_t n, void* workspace, size_t ws_bytes, void* stream,
                      soma_adamw** out) {
  int chunk = 0;
  int64_t chunks = 0;
  if (int rc = check_tensors(tensors, n, &chunk, &chunks)) return rc;
  if (!out) return set_error(SOMA_EINVAL, "out is NULL");
  if (int rc = check_apart(tensors, n)) return rc;
  const size_t need = table_bytes(n) + up256(size_t(chunks) * sizeof(Block));
  if (int rc = check_workspace(workspace, ws_bytes, need)) return rc;
  const hipStream_t st = stream_of(stream);
  // Waiting for a stream that records a graph would end the recording.
  hipStreamCaptureStatus recording = hipStreamCaptureStatusNone;
  hipError_t e = hipStreamIsCapturing(st, &recording);
  if (e != hipSuccess) return device_error("hipStreamIsCapturing", e);
  if (recording != hipStreamCaptureStatusNone) return set_error(SOMA_EINVAL, "a plan cannot be made on a stream that is captured");
  char* host = new (std::nothrow) char[need]();
  int64_t* first = new (std::nothrow) int64_t[size_t(n) + 1];
  soma_adamw* plan = new (std::nothrow) soma_adamw;
  if (!host || !first || !plan) {
    delete[] host;
    delete[] first;
    delete plan;
    return set_error(SOMA_EINVAL, "out of host memory");
  }
  Tensor* tt = reinterpret_cast<Tensor*>(host);
  Block* bb = reinterpret_cast<Block*>(host + table_bytes(n));
  int64_t at = 0;
  for (int32_t i = 0; i < n; ++i) {
    const soma_adamw_tensor& x = tensors[i];
    const size_t state = x.state_bits == 8 ? 4 : 16;
    first[i] = at;
    tt[i] = Tensor{x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, x.copy, x.count, x.weight_decay,
                   4 * (x.param_type == SOMA_BFLOAT) + 2 * (x.grad_type == SOMA_BFLOAT) + (x.state_bits == 8),
                   is_aligned(x.param, 4 * type_size(x.param_type)) && is_aligned(x.grad, 4 * type_size(x.grad_type)) &&
                       is_aligned(x.m, state) && is_aligned(x.v, state) && is_aligned(x.copy, 8)};
    for (int64_t c = 0; c < chunks_of(x.count, chunk); ++c) bb[at++] = Block{i, int32_t(c)};
  }
  first[n] = at;
  e = hipMemcpyAsync(workspace, host, need, hipMemcpyHostToDevice, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  delete[] host;
  if (e != hipSuccess) {
    delete[] first;
    delete plan;
    return device_error("copying the tensors' table", e);
  }
  *plan = soma_adamw{n, chunk, chunks, static_cast<const Tensor*>(workspace),
                     reinterpret_cast<const Block*>(static_cast<char*>(workspace) + table_bytes(n)), first,
                     SOMA_ROUND_NEAREST, 0};
  *out = plan;
  return set_ok();
}

void soma_adamw_destroy(soma_adamw* plan) {
  if (!plan) return;
  delete[] plan->first_chunk;
  delete plan;
}

int soma_adamw_set_rounding(soma_adamw* plan, int32_t rounding, uint64_t seed) {
  if (!plan) return set_error(SOMA_EINVAL, "plan is NULL");
  if (rounding != SOMA_ROUND_NEAREST && rounding != SOMA_ROUND_RANDOM)
    return set_error(SOMA_EINVAL, "unknown rounding %d", rounding);
  plan->rounding = rounding;
  plan->seed = seed;
  return set_ok();
}

int soma_adamw_step(soma_adamw* plan, int64_t t, double lr, double beta1, double beta2, double delta,
                    const float* grad_scale, void* stream) {
  if (!plan) return set_error(SOMA_EINVAL, "plan is NULL");
  if (t < 1) return set_error(SOMA_EINVAL, "the update number t must be >= 1");
  if (!std::isfinite(lr)) return set_error(SOMA_EINVAL, "lr must be finite");
  if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0))
    return set_error(SOMA_EINVAL, "beta1 and beta2 must be in [0, 1)");
  if (!(std::isfinite(float(delta)) && float(delta) > 0.0f)) return set_error(SOMA_EINVAL, "delta must be finite and > 0 in fp32");
  if (!is_aligned(grad_scale, 4)) return set_error(SOMA_EINVAL, "grad_scale must be 4-byte aligned");
  if (plan->chunks == 0) return set_ok();
  const double bc1 = 1.0 - std::pow(beta1, double(t)), bc2 = 1.0 - std::pow(beta2, double(t));
  if (!std::isfinite(float(lr / bc1))) return set_error(SOMA_EINVAL, "lr / (1 - beta1^t) must be finite in fp32");
  const Rates r{float(beta1), float(1.0 - beta1), float(beta2), float(1.0 - beta2), float(lr / bc1),
                float(1.0 / std::sqrt(bc2)), float(delta), 1.0 / std::sqrt(bc2) <= 0x1p30 && delta <= 0x1p30, plan->chunk, lr};
  // stream_key(seed, t)
  const Draw d{make_uint2(uint32_t(plan->seed), uint32_t(plan->seed >> 32) ^ uint32_t(uint64_t(t) >> 32)), uint32_t(t), 0};
  const dim3 grid(unsigned(plan->chunks)), block(kThreadsAdamw);
  const auto kernel = plan->rounding == SOMA_ROUND_RANDOM ? k_adamw<true> : k_adamw<false>;
  if (int rc = launch("k_adamw", kernel, grid, block, 0, stream_of(stream), plan->tensors, plan->blocks, r, d, grad_scale))
    return rc;
  return set_ok();
}

int soma_adamw_moments(soma_adamw* plan, float* const* m_out, float* const* v_out, void* stream) {
  if (!plan) return set_error(SOMA_EINVAL, "plan is NULL");
  if (!m_out || !v_out) return set_error(SOMA_EINVAL, "m_out or v_out is NULL");
  for (int32_t i = 0; i < plan->n; ++i)
    if (plan->first_chunk[i + 1] > plan->first_chunk[i] &&
        (!m_out[i] || !v_out[i] || !is_aligned(m_out[i], 4) || !is_aligned(v_out[i], 4)))
      return set_error(SOMA_EINVAL, "tensor %d: outputs must be 4-byte aligned device pointers", i);
  for (int32_t i = 0; i < plan->n; i += kOutputs) {
    const int32_t end = i + kOutputs < plan->n ? i + kOutputs : plan->n;
    const int64_t chunks = plan->first_chunk[end] - plan->first_chunk[i];
    if (chunks == 0) continue;
    Outputs o{};
    for (int32_t k = i; k < end; ++k) o.m[k - i] = m_out[k], o.v[k - i] = v_out[k];
    if (int rc = launch("k_adamw_moments", k_adamw_moments, dim3(unsigned(chunks)), dim3(kThreadsAdamw), 0,
                        stream_of(stream), plan->tensors, plan->blocks + plan->first_chunk[i], i, plan->chunk, o))
      return rc;
  }
  return set_ok();
}

}  // extern "C"
