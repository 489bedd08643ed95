// soma_la.hip -- linear attention with a decay a_h for each head,
//   S_t = a S_{t-1} + k_t v_t^T,   o_t = scale q_t^T S_t,
// over packed sequences, forward, backward and for single tokens.
//
// One walk serves all of it.  For arrays X, Y, Z of rows
//   out_i = X_i (sum_{j <= i} a^(i-j) Y_j (x) Z_j  +  a^(i+e) R),
// i counted from the row where the walk begins and R what it begins with:
//   o     X = q,  Y = k,  Z = v,   R = s0,   from the first row on;
//   dq    X = do, Y = v,  Z = k,   R = s0^T, from the first row on;
//   dk    X = v,  Y = do, Z = q,   R = dsT^T, from the last row back;
//   dv    X = k,  Y = q,  Z = do,  R = dsT,  from the last row back,
// with e = 1 from the front (a row sees the state in front of it decayed once) and
// e = 0 from the back (D_T = scale q_T do_T^T + dsT); what a walk back ends with,
// R = a D_1, is ds0.
//
// A block walks one head's rows in chunks of C (bf16 64, fp32 32), its four waves
// side by side over the columns of Z.  In a chunk
//   P = X Y^T with a^(i-j) below its diagonal (16 x 16 tiles dealt out to the waves,
//       exchanged through LDS),
//   out = P Z + a^(i+e) X R,   R <- a^m R + sum_j a^(m-j-e) Y_j (x) Z_j.
// R stays in registers, in the MFMA's own layout: the four values that a lane holds
// of a result are four of the k that it feeds as an operand, and the order of k is
// free, so R goes from result to operand without a move; the rows of Y^T are dealt
// out to suit.
//
// bf16 operands enter the matrix cores as they are.  P and R enter as two bf16 parts
// (2^-16 of a value; out is rounded to bf16 behind it), Z times its weight in the
// state's update as three, which hold all 24 bits: states stay fp32.  fp32 goes
// through the fp32 MFMA.  Weights in a chunk are products of a^((i-j) mod 16 + 15)
// and a^(16 k - 15), both powers of nonnegative exponent: nothing overflows.
//
// Where the diagonal's tiles meet values of Z that are not finite, zeros of P would
// make NaN of them for rows in front of theirs: such a chunk forms P Z without them
// and adds their terms one by one.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "soma.h"
#include "soma_host.hpp"
#include "soma_types.hpp"

namespace soma {
namespace {

constexpr float kL2e = 1.4426950408889634f;
constexpr int kThreads = 256;

typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));

// How a type feeds the matrix cores: kEl values of k a lane and fragment, of which
// a fragment has kKw = 4 kEl; kC rows a chunk; kPad elements between rows in LDS.
template <class T>
struct Kind;
template <>
struct Kind<bf16> {
  typedef uint16_t Word;
  typedef b8 Frag;
  static constexpr int kEl = 8, kKw = 32, kC = 64, kPad = 8, kParts = 2;
};
template <>
struct Kind<float> {
  typedef float Word;
  typedef f4 Frag;
  static constexpr int kEl = 4, kKw = 16, kC = 32, kPad = 4, kParts = 1;
};

__device__ __forceinline__ f4 mfma(const b8& a, const b8& b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f4 mfma(const f4& a, const f4& b, f4 c) {
#pragma unroll
  for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], c, 0, 0, 0);
  return c;
}

// Eight fp32 values as bf16 parts: all but the last truncated, so that no part
// overflows and what is left is exact; the last rounded.
template <int kN>
__device__ __forceinline__ void split(float (&x)[8], b8 (&part)[kN]) {
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (n == kN - 1) {
        w[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
      } else {
        const uint32_t lo = __float_as_uint(x[2 * i]), hi = __float_as_uint(x[2 * i + 1]);
        w[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
        x[2 * i] -= __uint_as_float(lo & 0xFFFF0000u);
        x[2 * i + 1] -= __uint_as_float(hi & 0xFFFF0000u);
      }
    }
    part[n] = __builtin_bit_cast(b8, make_uint4(w[0], w[1], w[2], w[3]));
  }
}

struct Walk {
  const void *x, *y, *z;
  int64_t x_stride, y_stride, z_stride;     // elements between rows
  int x_share, y_share, z_share;            // heads that share one of x's, y's or z's
  int inner, outer;                         // columns of a head of x and y; of z and out
  int x_vec, y_vec, z_vec;                  // 16-byte loads
  void* out;                                // [rows][heads outer] of T, or fp32
  int out_float, out_vec;
  const float *begin, *log_decay;           // states [sequences][heads][..], or NULL: zeros
  float* end;                               // the same, or NULL: not wanted
  int64_t row_stride, col_stride;           // of begin and end, an inner and an outer index
  const int32_t* offsets;                   // [sequences + 1], or NULL: `length` rows each
  int rows, length, sequences, heads, slices;
  int back;                                 // from the last row to the first
  float p_scale, in_scale, front_scale;     // of P, of the state's update, of what R gives
  int piece, pieces;                        // rows a piece (0: a block a sequence), pieces
  float* slots;                             // [pieces][heads][slices][a block's state]
  int2* info;                               // [pieces]: rows of a piece's map, sequence it begins in (-1: in front of it)
};

__device__ __forceinline__ int first_row(const Walk& a, int s) {
  if (!a.offsets) return s * a.length;
  const int b = a.offsets[s];
  return min(max(b, 0), a.rows);
}

// First sequence that has rows from `row` on, or begins (empty) there or later.
__device__ __forceinline__ int sequence_from(const Walk& a, int row) {
  int lo = 0, hi = a.sequences;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (first_row(a, mid + 1) > row || first_row(a, mid) >= row) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// Last sequence that begins in front of `row`, or -1.
__device__ __forceinline__ int sequence_before(const Walk& a, int row) {
  int lo = 0, hi = a.sequences;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (first_row(a, mid) < row) lo = mid + 1;
    else hi = mid;
  }
  return lo - 1;
}

// kEl elements of a row of T from column c on, zeros from `width` on.
template <class T>
__device__ __forceinline__ uint4 load_unit(const T* row, int c, int width, bool there, int vec) {
  uint4 u = make_uint4(0, 0, 0, 0);
  if (!there) return u;
  if (vec) {
    if (c < width) u = *reinterpret_cast<const uint4*>(row + c);
    return u;
  }
  uint32_t w[4] = {0, 0, 0, 0};
  if constexpr (sizeof(T) == 2) {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < width) w[i / 2] |= static_cast<uint32_t>(p[c + i]) << (16 * (i & 1));
  } else {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(row);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < width) w[i] = p[c + i];
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A value that is not finite, told by its exponent's carry into the bit above.
template <class T>
__device__ __forceinline__ uint32_t not_finite(const uint4& u) {
  constexpr uint32_t e = sizeof(T) == 2 ? 0x7F807F80u : 0x7F800000u, one = sizeof(T) == 2 ? 0x00800080u : 0x00800000u,
                     top = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
  return (((u.x & e) + one) | ((u.y & e) + one) | ((u.z & e) + one) | ((u.w & e) + one)) & top;
}

// A fragment with zeros in the place of what is not finite.
__device__ __forceinline__ b8 finite_part(const b8& f) {
  const uint4 u = __builtin_bit_cast(uint4, f);
  uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((w[i] & 0x7F80u) == 0x7F80u) w[i] &= 0xFFFF0000u;
    if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] &= 0xFFFFu;
  }
  return __builtin_bit_cast(b8, make_uint4(w[0], w[1], w[2], w[3]));
}
__device__ __forceinline__ f4 finite_part(const f4& f) {
  f4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (__float_as_uint(f[i]) & 0x7F800000u) == 0x7F800000u ? 0.0f : f[i];
  return r;
}

// Rows of one array on their way to LDS: kRows x kCols, kThreads lanes side by side.
template <class T, int kRows, int kCols>
struct Tile {
  typedef Kind<T> K;
  static constexpr int kUnits = kCols / K::kEl, kMine = kRows * kUnits / kThreads, kStride = kCols + K::kPad;
  static_assert(kMine * kThreads == kRows * kUnits, "every lane has as many units");
  uint4 u[kMine];

  __device__ __forceinline__ void load(const T* base, int64_t stride, int row0, int dir, int m, int c0, int width, int vec) {
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
      const int at = threadIdx.x + kThreads * k, r = at / kUnits, c = c0 + at % kUnits * K::kEl;
      u[k] = load_unit(base + static_cast<int64_t>(row0 + (r < m ? dir * r : 0)) * stride, c, width, r < m, vec);
    }
  }
  __device__ __forceinline__ uint32_t store(typename K::Word* lds) const {
    uint32_t bad = 0;
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
      const int at = threadIdx.x + kThreads * k, r = at / kUnits, c = at % kUnits * K::kEl;
      *reinterpret_cast<uint4*>(lds + r * kStride + c) = u[k];
      bad |= not_finite<T>(u[k]);
    }
    return bad;
  }
};

// Fragment of an operand whose k lie side by side in a row: row l % 16, kEl values.
template <class T>
__device__ __forceinline__ typename Kind<T>::Frag along(const typename Kind<T>::Word* lds, int stride, int row, int k) {
  const int l = threadIdx.x & 63;
  return *reinterpret_cast<const typename Kind<T>::Frag*>(lds + (row + (l & 15)) * stride + k + (l >> 4) * Kind<T>::kEl);
}

// Fragment of an operand whose k are rows: column col + (n / 4) step + n % 4 for lane
// n = l % 16, kEl rows from k + kEl (l / 16) on.
__device__ __forceinline__ b8 across(const uint16_t* lds, int stride, int k, int col, int step) {
  const int l = threadIdx.x & 63, row = k + 8 * (l >> 4) + ((l & 15) >> 2), c = col + (l & 3) * step;
  typedef __attribute__((address_space(3))) s4 Lds;
  const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(lds + row * stride + c));
  const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(lds + (row + 4) * stride + c));
  return __builtin_bit_cast(b8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
__device__ __forceinline__ f4 across(const float* lds, int stride, int k, int col, int step) {
  const int l = threadIdx.x & 63, c = col + ((l & 15) >> 2) * step + (l & 3);
  const float* p = lds + (k + 4 * (l >> 4)) * stride + c;
  return f4{p[0], p[stride], p[2 * stride], p[3 * stride]};
}

// kInner: columns of X and Y, filled up; kTiles: 16-column tiles of Z a wave.  kMap:
// only what a piece adds to the state behind it.
template <class T, int kInner, int kTiles, bool kMap>
struct Walker {
  typedef Kind<T> K;
  typedef typename K::Word Word;
  typedef typename K::Frag Frag;
  static constexpr int kC = K::kC, kRowTiles = kC / 16, kSteps = kInner / K::kKw, kCols = 64 * kTiles,
                       kSub = K::kKw / 16;  // 16-row tiles of R a fragment
  static constexpr int kXs = kInner + K::kPad, kZs = kCols + K::kPad, kPs = kC + K::kPad;
  static constexpr int kPWords = kC * kPs * K::kParts;
  static constexpr int kLds =
      (kMap ? kC * (kXs + kZs) : kC * (2 * kXs + kZs) + kPWords) * static_cast<int>(sizeof(Word)) + 16;
  // a block's state in a slot
  static constexpr int kState = kInner * kCols;

  f4 r[kSteps][kSub][kTiles];  // rows kKw t + (m / 4) kEl + m % 4 + 4 sub, m = 4 (l / 16) + element
  float l2;                    // log2 of the decay
  float in[kC / K::kKw][K::kEl];
  int in_for;

  __device__ __forceinline__ float power(int n) const { return __builtin_amdgcn_exp2f(l2 * static_cast<float>(n)); }

  __device__ __forceinline__ void weights(const Walk& a, int m) {
    in_for = m;
    const int g = (threadIdx.x & 63) >> 4, e = a.back ? 0 : 1;
#pragma unroll
    for (int t = 0; t < kC / K::kKw; ++t)
#pragma unroll
      for (int i = 0; i < K::kEl; ++i) {
        const int j = t * K::kKw + g * K::kEl + i;
        in[t][i] = j < m ? a.in_scale * power(m - j - e) : 0.0f;
      }
  }

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) r[t][s][n] = f4{0, 0, 0, 0};
  }

  // Inner and outer index of element 0 of r[t][s][n]; the other three follow.
  static __device__ __forceinline__ int inner_of(int t, int s, int lane) { return K::kKw * t + (lane >> 4) * K::kEl + 4 * s; }
  static __device__ __forceinline__ int outer_of(int wave, int n, int lane) { return (wave * kTiles + n) * 16 + (lane & 15); }

  __device__ __forceinline__ void read_state(const Walk& a, const float* p, int col0) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
          const int c = col0 + outer_of(wave, n, lane), d = inner_of(t, s, lane);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            r[t][s][n][i] = p && c < a.outer && d + i < a.inner ? p[(d + i) * a.row_stride + c * a.col_stride] : 0.0f;
        }
  }
  __device__ __forceinline__ void write_state(const Walk& a, float* p, int col0) const {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
          const int c = col0 + outer_of(wave, n, lane), d = inner_of(t, s, lane);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (c < a.outer && d + i < a.inner) p[(d + i) * a.row_stride + c * a.col_stride] = r[t][s][n][i];
        }
  }
  // A slot holds the registers as they lie.
  static __device__ __forceinline__ int in_slot(int t, int s, int n) { return (((t * kSub + s) * kTiles + n) * kThreads) * 4; }
  __device__ __forceinline__ void read_slot(const float* p) {
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) r[t][s][n] = *reinterpret_cast<const f4*>(p + in_slot(t, s, n) + threadIdx.x * 4);
  }
  __device__ __forceinline__ void write_slot(float* p) const {
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) *reinterpret_cast<f4*>(p + in_slot(t, s, n) + threadIdx.x * 4) = r[t][s][n];
  }

  // Rows lo .. hi - 1 of the arrays.
  __device__ void part(const Walk& a, int lo, int hi, int head, int col0, Word* lds) {
    Word* const ly = lds;
    Word* const lz = ly + kC * kXs;
    Word* const lx = lz + kC * kZs;
    Word* const lp = lx + kC * kXs;
    uint32_t* const flags = reinterpret_cast<uint32_t*>(kMap ? lx : lp + kPWords);
    const T* const x = static_cast<const T*>(a.x) + static_cast<int64_t>(head / a.x_share) * a.inner;
    const T* const y = static_cast<const T*>(a.y) + static_cast<int64_t>(head / a.y_share) * a.inner;
    const T* const z = static_cast<const T*>(a.z) + static_cast<int64_t>(head / a.z_share) * a.outer;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, li = lane & 15;
    const int dir = a.back ? -1 : 1, n = hi - lo, row0 = a.back ? hi - 1 : lo;

    // weights of a tile: below the diagonal a^(i-j) = a^(ii - jj + 15) a^(16 k - 15)
    float below[4], at[4], front[kRowTiles], far[kRowTiles];
    if constexpr (!kMap) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int d = li - (4 * g + i);
        below[i] = power(d + 15);
        at[i] = d >= 0 ? a.p_scale * power(d) : 0.0f;
      }
#pragma unroll
      for (int t = 0; t < kRowTiles; ++t) {
        front[t] = a.front_scale * power(16 * t + li + (a.back ? 0 : 1));
        far[t] = t ? a.p_scale * power(16 * t - 15) : 0.0f;
      }
    }

    Tile<T, kC, kInner> tx, ty;
    Tile<T, kC, kCols> tz;
    const auto fetch = [&](int c) {
      const int m = min(kC, n - c), row = row0 + dir * c;
      if constexpr (!kMap) tx.load(x, a.x_stride, row, dir, m, 0, a.inner, a.x_vec);
      ty.load(y, a.y_stride, row, dir, m, 0, a.inner, a.y_vec);
      tz.load(z, a.z_stride, row, dir, m, col0, a.outer, a.z_vec);
    };
    fetch(0);
    for (int c = 0; c < n; c += kC) {
      const int m = min(kC, n - c), flag = (c / kC) & 1;
      __syncthreads();  // the tiles in front have been read
      if constexpr (!kMap) tx.store(lx);
      ty.store(ly);
      const uint32_t bad = tz.store(lz);
      if constexpr (!kMap)
        if (bad) flags[flag] = 1;
      __syncthreads();
      if (c + kC < n) fetch(c + kC);
      if (in_for != m) weights(a, m);
      bool slow = false;
      if constexpr (!kMap) {
        slow = flags[flag] != 0;
        // P, tiles 0 .. below and on the diagonal in the order of their rows
#pragma unroll
        for (int k = 0; k < (kRowTiles * (kRowTiles + 1) / 2 + 3) / 4; ++k) {
          const int t = wave + 4 * k;
          const int ti = t >= 6 ? 3 : t >= 3 ? 2 : t >= 1 ? 1 : 0, tj = t - ti * (ti + 1) / 2;
          if (tj > ti || ti >= kRowTiles || 16 * ti >= m) break;
          f4 p = {0, 0, 0, 0};
#pragma unroll
          for (int s = 0; s < kSteps; ++s)
            p = mfma(along<T>(ly, kXs, 16 * tj, s * K::kKw), along<T>(lx, kXs, 16 * ti, s * K::kKw), p);
          if (ti == tj) {
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = li >= 4 * g + i ? p[i] * at[i] : 0.0f;
          } else {
            const float w = ti - tj == 1 ? far[1] : ti - tj == 2 ? far[kRowTiles > 2 ? 2 : 1] : far[kRowTiles - 1];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] *= below[i] * w;
          }
          Word* const to = lp + (16 * ti + li) * kPs + 16 * tj + 4 * g;
          if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<f4*>(to) = p;
          } else {
            const uint32_t u[4] = {__float_as_uint(p[0]), __float_as_uint(p[1]), __float_as_uint(p[2]), __float_as_uint(p[3])};
            *reinterpret_cast<uint2*>(to) =
                make_uint2(__builtin_amdgcn_perm(u[1], u[0], 0x07060302u), __builtin_amdgcn_perm(u[3], u[2], 0x07060302u));
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] -= __uint_as_float(u[i] & 0xFFFF0000u);
            *reinterpret_cast<uint2*>(to + kC * kPs) = make_uint2(bf16_pair(p[0], p[1]), bf16_pair(p[2], p[3]));
          }
        }
        __syncthreads();
        if (threadIdx.x == 0) flags[flag ^ 1] = 0;
      }

      // out^T: lane l holds row l % 16 of a row tile, columns 4 (l / 16) ..
      f4 o[kRowTiles][kTiles];
      if constexpr (!kMap) {
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i)
#pragma unroll
          for (int k = 0; k < kTiles; ++k) o[i][k] = f4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          Frag fx[kRowTiles];
#pragma unroll
          for (int i = 0; i < kRowTiles; ++i) fx[i] = along<T>(lx, kXs, 16 * i, s * K::kKw);
#pragma unroll
          for (int k = 0; k < kTiles; ++k) {
            if constexpr (sizeof(T) == 4) {
#pragma unroll
              for (int i = 0; i < kRowTiles; ++i) o[i][k] = mfma(r[s][0][k], fx[i], o[i][k]);
            } else {
              float v[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) v[i] = r[s][i / 4][k][i % 4];
              b8 part[2];
              split(v, part);
#pragma unroll
              for (int i = 0; i < kRowTiles; ++i) o[i][k] = mfma(part[1], fx[i], mfma(part[0], fx[i], o[i][k]));
            }
          }
        }
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i)
#pragma unroll
          for (int k = 0; k < kTiles; ++k) o[i][k] *= front[i];
      }

      // the state, and P Z from the same fragments of Z
      const float keep = power(m);
#pragma unroll
      for (int t = 0; t < kSteps; ++t)
#pragma unroll
        for (int s = 0; s < kSub; ++s)
#pragma unroll
          for (int k = 0; k < kTiles; ++k) r[t][s][k] *= keep;
#pragma unroll
      for (int j = 0; j < kC / K::kKw; ++j) {
        if (j * K::kKw < m) {
          Frag fz[kTiles];
#pragma unroll
          for (int k = 0; k < kTiles; ++k) fz[k] = across(lz, kZs, j * K::kKw, (wave * kTiles + k) * 16, 4);
          if constexpr (!kMap) {
            Frag fv[kTiles];
#pragma unroll
            for (int k = 0; k < kTiles; ++k) fv[k] = fz[k];
            if (slow) {
#pragma unroll
              for (int k = 0; k < kTiles; ++k) fv[k] = finite_part(fz[k]);
            }
#pragma unroll
            for (int i = 0; i < kRowTiles; ++i)
              if (16 * (i + 1) > j * K::kKw) {
                const Frag fp = along<T>(lp, kPs, 16 * i, j * K::kKw);
#pragma unroll
                for (int k = 0; k < kTiles; ++k) o[i][k] = mfma(fv[k], fp, o[i][k]);
                if constexpr (K::kParts == 2) {
                  const Frag fl = along<T>(lp + kC * kPs, kPs, 16 * i, j * K::kKw);
#pragma unroll
                  for (int k = 0; k < kTiles; ++k) o[i][k] = mfma(fv[k], fl, o[i][k]);
                }
              }
          }
          constexpr int kZParts = sizeof(T) == 4 ? 1 : 3;
          Frag zw[kTiles][kZParts];
#pragma unroll
          for (int k = 0; k < kTiles; ++k) {
            if constexpr (sizeof(T) == 4) {
              zw[k][0] = f4{fz[k][0] * in[j][0], fz[k][1] * in[j][1], fz[k][2] * in[j][2], fz[k][3] * in[j][3]};
            } else {
              const uint4 u = __builtin_bit_cast(uint4, fz[k]);
              const uint32_t w[4] = {u.x, u.y, u.z, u.w};
              float v[8];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16) * in[j][2 * i];
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u) * in[j][2 * i + 1];
              }
              split(v, zw[k]);
            }
          }
#pragma unroll
          for (int t = 0; t < kSteps; ++t)
#pragma unroll
            for (int s = 0; s < kSub; ++s) {
              const Frag fy = across(ly, kXs, j * K::kKw, t * K::kKw + 4 * s, K::kEl);
#pragma unroll
              for (int k = 0; k < kTiles; ++k)
#pragma unroll
                for (int q = kZParts - 1; q >= 0; --q) r[t][s][k] = mfma(fy, zw[k][q], r[t][s][k]);
            }
        }
      }

      if constexpr (!kMap) {
        if (slow) {
          for (int j = 0; j < m; ++j)
#pragma unroll
            for (int k = 0; k < kTiles; ++k) {
              float v[4];
              bool any = false;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const Word w = lz[j * kZs + (wave * kTiles + k) * 16 + 4 * g + e];
                if constexpr (sizeof(T) == 4) v[e] = w;
                else v[e] = from_bf16(w);
                any |= !__builtin_isfinite(v[e]);
              }
              if (__builtin_amdgcn_ballot_w64(any) == 0) continue;
#pragma unroll
              for (int i = 0; i < kRowTiles; ++i) {
                const int row = 16 * i + li;
                float p;
                if constexpr (sizeof(T) == 4) p = lp[row * kPs + j];
                else p = from_bf16(lp[row * kPs + j]) + from_bf16(lp[(row + kC) * kPs + j]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (row >= j && !__builtin_isfinite(v[e])) o[i][k][e] += p * v[e];
              }
            }
        }
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i) {
          if (16 * i + li < m) {
            const int64_t row = row0 + dir * (c + 16 * i + li);
            const int64_t to = row * a.heads * a.outer + static_cast<int64_t>(head) * a.outer;
#pragma unroll
            for (int k = 0; k < kTiles; ++k) {
              const int col = col0 + (wave * kTiles + k) * 16 + 4 * g;
              if (a.out_vec) {
                if (col < a.outer) {
                  const float4 v = make_float4(o[i][k][0], o[i][k][1], o[i][k][2], o[i][k][3]);
                  if (a.out_float) store_four(static_cast<float*>(a.out) + to + col, v);
                  else store_four(static_cast<T*>(a.out) + to + col, v);
                }
              } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (col + e < a.outer) {
                    if (a.out_float) static_cast<float*>(a.out)[to + col + e] = o[i][k][e];
                    else store_value(static_cast<T*>(a.out) + to + col + e, o[i][k][e]);
                  }
              }
            }
          }
        }
      }
    }
  }
};

template <class T, int kInner, int kTiles, bool kMap>
__global__ __launch_bounds__(kThreads) void k_la_walk(const Walk a) {
  typedef Walker<T, kInner, kTiles, kMap> W;
  __shared__ __align__(16) unsigned char memory[W::kLds];
  typename W::Word* const lds = reinterpret_cast<typename W::Word*>(memory);
  const int units = a.heads * a.slices;
  const int p = blockIdx.x / units, unit = blockIdx.x % units, head = unit / a.slices, slice = unit % a.slices;
  const int col0 = slice * W::kCols;
  W w;
  const float l = a.log_decay[head] * kL2e;
  w.l2 = l < -1e30f ? -1e30f : l;           // a = 0: a^0 is 1
  w.in_for = -1;
  const int64_t state = static_cast<int64_t>(a.inner) * a.outer;
  if constexpr (!kMap) {
    // tiles of P above the diagonal that a fragment reaches are zeros throughout
    for (int i = threadIdx.x; i < W::kLds / 4; i += kThreads) reinterpret_cast<uint32_t*>(memory)[i] = 0;
    __syncthreads();
  }

  if constexpr (kMap) {
    // what the piece adds to the state of the sequence that crosses its far border
    const int border = a.back ? p * a.piece : min((p + 1) * a.piece, a.rows);
    const int s = border > 0 && border < a.rows ? sequence_before(a, border) : -1;
    int lo = 0, hi = 0, begins = -1;
    if (s >= 0 && first_row(a, s + 1) > border) {
      const int b = first_row(a, s), e = first_row(a, s + 1), far = min(p + 1 < a.pieces ? (p + 1) * a.piece : a.rows, a.rows);
      lo = a.back ? border : max(b, p * a.piece);
      hi = a.back ? min(e, far) : border;
      if (a.back ? e <= far : b >= p * a.piece) begins = s;
    }
    if (unit == 0 && threadIdx.x == 0) a.info[p] = make_int2(max(hi - lo, 0), begins);
    if (hi <= lo) return;
    w.zero();
    w.part(a, lo, hi, head, col0, lds);
    w.write_slot(a.slots + (static_cast<int64_t>(p) * units + unit) * W::kState);
  } else if (!a.piece) {
    const int b = first_row(a, p), e = first_row(a, p + 1);
    const int64_t at = (static_cast<int64_t>(p) * a.heads + head) * state;
    w.read_state(a, a.begin ? a.begin + at : nullptr, col0);
    if (e > b) w.part(a, b, e, head, col0, lds);
    if (a.end) w.write_state(a, a.end + at, col0);
  } else {
    const bool last = p + 1 == a.pieces;
    const int lo = p * a.piece, hi = last ? a.rows : lo + a.piece;
    const int s0 = sequence_from(a, lo), s1 = last ? a.sequences - 1 : sequence_before(a, hi);
    for (int i = s0; i <= s1; ++i) {
      const int s = a.back ? s1 - (i - s0) : i;
      const int b = first_row(a, s), e = max(first_row(a, s + 1), b);
      const int64_t at = (static_cast<int64_t>(s) * a.heads + head) * state;
      const int from = max(b, lo), to = min(e, hi);
      if (e > b && from >= to) continue;
      const bool enters = a.back ? e > hi : b < lo, leaves = a.back ? b < lo : e > hi;
      if (enters) w.read_slot(a.slots + (static_cast<int64_t>(a.back ? p + 1 : p - 1) * units + unit) * W::kState);
      else w.read_state(a, a.begin ? a.begin + at : nullptr, col0);
      if (to > from) w.part(a, from, to, head, col0, lds);
      if (a.end && !leaves) w.write_state(a, a.end + at, col0);
    }
  }
}

// From what every piece adds to the state with which the next is entered, in the
// slot of the piece that is left.
template <class T, int kInner, int kTiles>
__global__ __launch_bounds__(kThreads) void k_la_join(const Walk a) {
  typedef Walker<T, kInner, kTiles, true> W;
  const int units = a.heads * a.slices, per = W::kState / 4;
  const int64_t id = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  const int unit = static_cast<int>(id / per), at = static_cast<int>(id % per);
  if (unit >= units) return;
  const int head = unit / a.slices, slice = unit % a.slices;
  const int lane = at & 63, wave = (at >> 6) & 3, tile = at / kThreads;
  const int n = tile % kTiles, s = tile / kTiles % W::kSub, t = tile / kTiles / W::kSub;
  const int c = slice * W::kCols + W::outer_of(wave, n, lane), d = W::inner_of(t, s, lane);
  float l = a.log_decay[head] * kL2e;
  l = l < -1e30f ? -1e30f : l;
  f4 state = {0, 0, 0, 0};
  constexpr int kAhead = 8;
  for (int k0 = 0; k0 < a.pieces; k0 += kAhead) {
    f4 add[kAhead];
    int2 info[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = k0 + k, p = a.back ? a.pieces - 1 - i : i;
      info[k] = i < a.pieces ? a.info[p] : make_int2(0, -1);
      if (info[k].x > 0) add[k] = *reinterpret_cast<const f4*>(a.slots + (static_cast<int64_t>(p) * units + unit) * W::kState + at * 4);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (info[k].x <= 0) continue;
      const int p = a.back ? a.pieces - 1 - (k0 + k) : k0 + k;
      if (info[k].y >= 0) {
        const float* b = a.begin ? a.begin + (static_cast<int64_t>(info[k].y) * a.heads + head) * a.inner * a.outer : nullptr;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          state[i] = b && c < a.outer && d + i < a.inner ? b[(d + i) * a.row_stride + c * a.col_stride] : 0.0f;
      }
      state = state * __builtin_amdgcn_exp2f(l * static_cast<float>(info[k].x)) + add[k];
      *reinterpret_cast<f4*>(a.slots + (static_cast<int64_t>(p) * units + unit) * W::kState + at * 4) = state;
    }
  }
}

// Gradients of keys or values that several heads share: [rows][heads][width] fp32 to
// [rows][heads / share][width].
template <class T>
__global__ __launch_bounds__(kThreads) void k_la_share(const float* in, T* out, int64_t n, int width, int share,
                                                       const int32_t* offsets, int sequences, int rows, int row_values) {
  const int used = offsets ? min(max(offsets[sequences], 0), rows) : rows;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * kThreads) {
    if (i / row_values >= used) return;
    const int64_t group = i / width;
    const float* p = in + group * share * width + i % width;
    float sum = p[0];
    for (int k = 1; k < share; ++k) sum += p[static_cast<int64_t>(k) * width];
    store_value(out + i, sum);
  }
}

__global__ __launch_bounds__(kThreads) void k_la_copy(const float* in, float* out, int64_t n) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * kThreads)
    out[i] = in[i];
}

struct Step {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  const float *log_decay, *s0;
  float* sT;
  void* o;
  int heads, share, key, value;
  float scale;
};

// One token of one sequence and head: a lane has kVec columns of the state and every
// kRows-th row of it.  Reads and writes the state once; bound by memory.
template <class T, int kVec>
__global__ __launch_bounds__(kThreads) void k_la_step(const Step a) {
  __shared__ float q[256], k[256], sums[kThreads * kVec];
  const int head = blockIdx.x % a.heads;
  const int64_t n = blockIdx.x / a.heads;
  const T* const pq = static_cast<const T*>(a.q) + n * a.q_stride + static_cast<int64_t>(head) * a.key;
  const T* const pk = static_cast<const T*>(a.k) + n * a.k_stride + static_cast<int64_t>(head / a.share) * a.key;
  const T* const pv = static_cast<const T*>(a.v) + n * a.v_stride + static_cast<int64_t>(head / a.share) * a.value;
  if (static_cast<int>(threadIdx.x) < a.key) {
    q[threadIdx.x] = load_value(pq + threadIdx.x);
    k[threadIdx.x] = load_value(pk + threadIdx.x);
  }
  const float decay = expf(a.log_decay[head]);
  const int cols = (a.value + kVec - 1) / kVec, lines = kThreads / cols;
  const int c = static_cast<int>(threadIdx.x) % cols, first = static_cast<int>(threadIdx.x) / cols;
  const bool mine = first < lines;
  float v[kVec], sum[kVec] = {};
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = mine ? load_value(pv + c * kVec + i) : 0.0f;
  __syncthreads();
  const int64_t at = (n * a.heads + head) * a.key * a.value + static_cast<int64_t>(c) * kVec;
  if (mine) {
#pragma unroll 4
    for (int d = first; d < a.key; d += lines) {
      const int64_t e = at + static_cast<int64_t>(d) * a.value;
      float s[kVec] = {};
      if (a.s0) {
        if constexpr (kVec == 4) {
          const float4 u = *reinterpret_cast<const float4*>(a.s0 + e);
          s[0] = u.x, s[1] = u.y, s[2] = u.z, s[3] = u.w;
        } else {
          s[0] = a.s0[e];
        }
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        s[i] = s[i] * decay + k[d] * v[i];
        sum[i] += q[d] * s[i];
      }
      if constexpr (kVec == 4) *reinterpret_cast<float4*>(a.sT + e) = make_float4(s[0], s[1], s[2], s[3]);
      else a.sT[e] = s[0];
    }
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i) sums[threadIdx.x * kVec + i] = sum[i];
  __syncthreads();
  for (int i = threadIdx.x; i < a.value; i += kThreads) {
    float x = 0.0f;
    for (int w = 0; w < lines; ++w) x += sums[w * cols * kVec + i];
    store_value(static_cast<T*>(a.o) + (n * a.heads + head) * a.value + i, a.scale * x);
  }
}

// ---------------------------------------------------------------------------
// Host

constexpr int kMostPieces = 256;
constexpr int kEnough = 1024;      // blocks that fill the card

int check_shape(const soma_la_config* cfg) {
  if (!cfg) return set_error(SOMA_EINVAL, "cfg is NULL");
  const soma_la_config& c = *cfg;
  if (!is_type(c.type)) return set_error(SOMA_EINVAL, "type %d is none of enum soma_type", c.type);
  if (c.rows < 0 || c.rows > (1 << 30)) return set_error(SOMA_ESHAPE, "rows %d is out of range", c.rows);
  if (c.sequences < 1 || c.sequences > 65535) return set_error(SOMA_ESHAPE, "sequences %d is out of range", c.sequences);
  if (c.heads < 1 || c.heads > 1024) return set_error(SOMA_ESHAPE, "heads %d is out of range", c.heads);
  if (c.kv_heads < 1 || c.kv_heads > c.heads || c.heads % c.kv_heads)
    return set_error(SOMA_ESHAPE, "kv_heads %d must divide heads %d", c.kv_heads, c.heads);
  if (c.key_width < 1 || c.key_width > 256) return set_error(SOMA_ESHAPE, "key_width %d is out of range", c.key_width);
  if (c.value_width < 1 || c.value_width > 256) return set_error(SOMA_ESHAPE, "value_width %d is out of range", c.value_width);
  if (!std::isfinite(c.scale)) return set_error(SOMA_EINVAL, "scale must be finite");
  for (int64_t stride : {c.q_stride, c.k_stride, c.v_stride})
    if (stride > (int64_t{1} << 32)) return set_error(SOMA_ESHAPE, "a row stride is out of range");
  if (c.q_stride < static_cast<int64_t>(c.heads) * c.key_width || c.k_stride < static_cast<int64_t>(c.kv_heads) * c.key_width ||
      c.v_stride < static_cast<int64_t>(c.kv_heads) * c.value_width)
    return set_error(SOMA_ESHAPE, "a row stride is shorter than its row");
  return SOMA_OK;
}

// Which instance walks over these widths, and how its columns are shared out.
struct Shape {
  int inner, tiles, slices;
};
Shape shape_of(int inner, int outer) {
  Shape s;
  s.inner = inner <= 64 ? 64 : inner <= 128 ? 128 : 256;
  s.tiles = outer <= 64 || s.inner == 256 ? 1 : 2;
  s.slices = (outer + 64 * s.tiles - 1) / (64 * s.tiles);
  return s;
}

// Pieces: none where every sequence has its blocks and they are enough, or short.
// Their number goes by the heads alone, so that a workspace serves fewer rows too.
int most_pieces(const soma_la_config& c, const Shape& s) {
  const int64_t units = static_cast<int64_t>(c.heads) * s.slices;
  if (units * c.sequences >= kEnough || c.rows <= static_cast<int64_t>(c.sequences) * 256) return 0;
  return static_cast<int>(std::min<int64_t>(kMostPieces, (2 * kEnough + units - 1) / units));
}

size_t slots_size(const soma_la_config& c, int inner, int outer) {
  const Shape s = shape_of(inner, outer);
  const int most = most_pieces(c, s);
  if (!most) return 0;
  return up256(sizeof(float) * most * c.heads * s.slices * s.inner * 64 * s.tiles) + up256(sizeof(int2) * most);
}

// A copy of the states that a walk begins with, where it ends with the same array and
// goes in pieces: one block may then read a state after another has written it.
size_t copy_size(const soma_la_config& c) {
  if (!most_pieces(c, shape_of(c.key_width, c.value_width))) return 0;
  return up256(sizeof(float) * c.sequences * c.heads * c.key_width * c.value_width);
}

int kept(const soma_la_config& c, const float** begin, const float* end, unsigned char* at, hipStream_t st) {
  if (!*begin || *begin != end || !copy_size(c)) return SOMA_OK;
  const int64_t n = static_cast<int64_t>(c.sequences) * c.heads * c.key_width * c.value_width;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((n + kThreads - 1) / kThreads, 4096)));
  const float* from = *begin;
  *begin = reinterpret_cast<const float*>(at);
  return launch("k_la_copy", k_la_copy, grid, dim3(kThreads), 0, st, from, reinterpret_cast<float*>(at), n);
}

// fp32 gradients of every head, where heads share keys and values
size_t sums_size(const soma_la_config& c) {
  if (c.heads == c.kv_heads) return 0;
  return up256(sizeof(float) * c.rows * c.heads * std::max(c.key_width, c.value_width));
}

size_t la_workspace(const soma_la_config& c, bool grad) {
  size_t n = slots_size(c, c.key_width, c.value_width) + copy_size(c);
  if (grad) n = std::max(n, slots_size(c, c.value_width, c.key_width)) + sums_size(c);
  return n;
}

template <class T, int kInner, int kTiles>
int walk_as(const Walk& a, hipStream_t st) {
  const int units = a.heads * a.slices, parts = a.piece ? a.pieces : a.sequences;
  if (a.piece) {
    if (int rc = launch("k_la_walk (maps)", k_la_walk<T, kInner, kTiles, true>, dim3(static_cast<unsigned>(units) * parts),
                        dim3(kThreads), 0, st, a))
      return rc;
    const int64_t n = static_cast<int64_t>(units) * Walker<T, kInner, kTiles, true>::kState / 4;
    if (int rc = launch("k_la_join", k_la_join<T, kInner, kTiles>, dim3(static_cast<unsigned>((n + kThreads - 1) / kThreads)),
                        dim3(kThreads), 0, st, a))
      return rc;
  }
  return launch("k_la_walk", k_la_walk<T, kInner, kTiles, false>, dim3(static_cast<unsigned>(units) * parts), dim3(kThreads), 0,
                st, a);
}

template <class T>
int walk_of(const Walk& a, const Shape& s, hipStream_t st) {
  if (s.inner == 64) return s.tiles == 1 ? walk_as<T, 64, 1>(a, st) : walk_as<T, 64, 2>(a, st);
  if (s.inner == 128) return s.tiles == 1 ? walk_as<T, 128, 1>(a, st) : walk_as<T, 128, 2>(a, st);
  return walk_as<T, 256, 1>(a, st);
}

// An array of rows and what a walk needs to know of it.
struct Array {
  const void* p;
  int64_t stride;
  int share;
};

int walk(const soma_la_config& c, const Array& x, const Array& y, const Array& z, int inner, int outer, bool back,
         const float* log_decay, const int32_t* offsets, const float* begin, float* end, bool transposed, void* out,
         bool out_float, unsigned char* ws, hipStream_t st) {
  const Shape s = shape_of(inner, outer);
  const int64_t e = static_cast<int64_t>(type_size(c.type));
  const auto vec = [&](const Array& a, int width) { return is_aligned(a.p, 16) && a.stride * e % 16 == 0 && width * e % 16 == 0; };
  Walk a{};
  a.x = x.p, a.y = y.p, a.z = z.p;
  a.x_stride = x.stride, a.y_stride = y.stride, a.z_stride = z.stride;
  a.x_share = x.share, a.y_share = y.share, a.z_share = z.share;
  a.inner = inner, a.outer = outer;
  a.x_vec = vec(x, inner), a.y_vec = vec(y, inner), a.z_vec = vec(z, outer);
  a.out = out;
  a.out_float = out_float;
  a.out_vec = outer % 4 == 0 && is_aligned(out, out_float ? 16 : 4 * e);
  a.begin = begin, a.end = end, a.log_decay = log_decay;
  a.row_stride = transposed ? 1 : outer;
  a.col_stride = transposed ? inner : 1;
  a.offsets = offsets;
  a.rows = c.rows, a.length = c.rows / c.sequences, a.sequences = c.sequences, a.heads = c.heads, a.slices = s.slices;
  a.back = back;
  a.p_scale = c.scale;
  a.in_scale = back ? c.scale : 1.0f;
  a.front_scale = back ? 1.0f : c.scale;
  if (const int most = most_pieces(c, s)) {
    a.piece = ((c.rows + most - 1) / most + 63) / 64 * 64;
    a.pieces = (c.rows + a.piece - 1) / a.piece;
    a.slots = reinterpret_cast<float*>(ws);
    a.info = reinterpret_cast<int2*>(ws + up256(sizeof(float) * most * c.heads * s.slices * s.inner * 64 * s.tiles));
  }
  return c.type == SOMA_FLOAT ? walk_of<float>(a, s, st) : walk_of<bf16>(a, s, st);
}

// The arrays' bytes.
struct Spans {
  const soma_la_config& c;
  size_t e;
  explicit Spans(const soma_la_config& c) : c(c), e(type_size(c.type)) {}
  Span rows(const void* p, int64_t width, int64_t stride) const { return span_of(p, c.rows, width, stride, e); }
  Span q(const void* p) const { return rows(p, static_cast<int64_t>(c.heads) * c.key_width, c.q_stride); }
  Span k(const void* p) const { return rows(p, static_cast<int64_t>(c.kv_heads) * c.key_width, c.k_stride); }
  Span v(const void* p) const { return rows(p, static_cast<int64_t>(c.kv_heads) * c.value_width, c.v_stride); }
  Span whole(const void* p, int64_t width) const { return rows(p, width, width); }
  Span o(const void* p) const { return whole(p, static_cast<int64_t>(c.heads) * c.value_width); }
  Span dq(const void* p) const { return whole(p, static_cast<int64_t>(c.heads) * c.key_width); }
  Span dk(const void* p) const { return whole(p, static_cast<int64_t>(c.kv_heads) * c.key_width); }
  Span dv(const void* p) const { return whole(p, static_cast<int64_t>(c.kv_heads) * c.value_width); }
  Span state(const void* p) const {
    return {p, sizeof(float) * c.sequences * c.heads * c.key_width * c.value_width};
  }
  Span decay(const void* p) const { return {p, sizeof(float) * c.heads}; }
  Span of(const int32_t* offsets) const { return {offsets, sizeof(int32_t) * (c.sequences + 1)}; }
};

int check_rows(const soma_la_config& c, const int32_t* offsets) {
  if (!is_aligned(offsets, 4)) return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  if (!offsets && c.rows % c.sequences) return set_error(SOMA_ESHAPE, "%d rows are no multiple of %d sequences", c.rows, c.sequences);
  return SOMA_OK;
}

}  // namespace
}  // namespace soma

using namespace soma;

extern "C" {

int soma_la_workspace_size(const soma_la_config* cfg, int grad, size_t* bytes) {
  if (int rc = check_shape(cfg)) return rc;
  if (!bytes) return set_error(SOMA_EINVAL, "bytes is NULL");
  *bytes = la_workspace(*cfg, grad != 0);
  return set_ok();
}

int soma_la_forward(const soma_la_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                    const int32_t* offsets, const float* s0, void* o, float* sT, void* workspace, size_t ws_bytes,
                    void* stream) {
  if (int rc = check_shape(cfg)) return rc;
  const soma_la_config& c = *cfg;
  const size_t e = type_size(c.type);
  if (!log_decay || (c.rows > 0 && (!q || !k || !v || !o))) return set_error(SOMA_EINVAL, "NULL device pointer");
  if (!is_aligned(q, e) || !is_aligned(k, e) || !is_aligned(v, e) || !is_aligned(o, e) || !is_aligned(s0, 4) ||
      !is_aligned(sT, 4) || !is_aligned(log_decay, 4))
    return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  if (int rc = check_rows(c, offsets)) return rc;
  const Spans n(c);
  if (!are_apart({n.o(o), n.state(sT)}, {n.q(q), n.k(k), n.v(v), n.state(s0 == sT ? nullptr : s0), n.decay(log_decay), n.of(offsets)}))
    return set_error(SOMA_EINVAL, "an output overlaps another array");
  if (int rc = check_workspace(workspace, ws_bytes, la_workspace(c, false))) return rc;
  const int share = c.heads / c.kv_heads;
  unsigned char* const ws = static_cast<unsigned char*>(workspace);
  const hipStream_t st = stream_of(stream);
  if (int rc = kept(c, &s0, sT, ws + slots_size(c, c.key_width, c.value_width), st)) return rc;
  if (int rc = walk(c, {q, c.q_stride, 1}, {k, c.k_stride, share}, {v, c.v_stride, share}, c.key_width, c.value_width, false,
                    log_decay, offsets, s0, sT, false, o, false, ws, st))
    return rc;
  return set_ok();
}

int soma_la_backward(const soma_la_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                     const int32_t* offsets, const float* s0, const void* d_o, const float* dsT, void* dq, void* dk, void* dv,
                     float* ds0, void* workspace, size_t ws_bytes, void* stream) {
  if (int rc = check_shape(cfg)) return rc;
  const soma_la_config& c = *cfg;
  const size_t e = type_size(c.type);
  if (!log_decay || (c.rows > 0 && (!q || !k || !v || !d_o || !dq || !dk || !dv)))
    return set_error(SOMA_EINVAL, "NULL device pointer");
  if (!is_aligned(q, e) || !is_aligned(k, e) || !is_aligned(v, e) || !is_aligned(d_o, e) || !is_aligned(dq, e) ||
      !is_aligned(dk, e) || !is_aligned(dv, e) || !is_aligned(s0, 4) || !is_aligned(dsT, 4) || !is_aligned(ds0, 4) ||
      !is_aligned(log_decay, 4))
    return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  if (int rc = check_rows(c, offsets)) return rc;
  const Spans n(c);
  if (!are_apart({n.dq(dq), n.dk(dk), n.dv(dv), n.state(ds0)},
                 {n.q(q), n.k(k), n.v(v), n.o(d_o), n.state(s0), n.state(ds0 == dsT ? nullptr : dsT), n.decay(log_decay), n.of(offsets)}))
    return set_error(SOMA_EINVAL, "an output overlaps another array");
  if (int rc = check_workspace(workspace, ws_bytes, la_workspace(c, true))) return rc;
  const int share = c.heads / c.kv_heads;
  const Array aq{q, c.q_stride, 1}, ak{k, c.k_stride, share}, av{v, c.v_stride, share},
      ao{d_o, static_cast<int64_t>(c.heads) * c.value_width, 1};
  unsigned char* const ws = static_cast<unsigned char*>(workspace);
  const hipStream_t st = stream_of(stream);
  float* sums = nullptr;
  if (share > 1)
    sums = reinterpret_cast<float*>(ws + la_workspace(c, true) - sums_size(c));
  const auto shared = [&](void* out, int width) -> int {
    if (share == 1 || c.rows == 0) return SOMA_OK;
    const int64_t n = static_cast<int64_t>(c.rows) * c.kv_heads * width;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((n + kThreads - 1) / kThreads, 8192)));
    if (c.type == SOMA_FLOAT)
      return launch("k_la_share", k_la_share<float>, grid, dim3(kThreads), 0, st, static_cast<const float*>(sums),
                    static_cast<float*>(out), n, width, share, offsets, c.sequences, c.rows, c.kv_heads * width);
    return launch("k_la_share", k_la_share<bf16>, grid, dim3(kThreads), 0, st, static_cast<const float*>(sums),
                  static_cast<bf16*>(out), n, width, share, offsets, c.sequences, c.rows, c.kv_heads * width);
  };
  if (int rc = walk(c, ao, av, ak, c.value_width, c.key_width, false, log_decay, offsets, s0, nullptr, true, dq, false, ws, st))
    return rc;
  if (int rc = walk(c, av, ao, aq, c.value_width, c.key_width, true, log_decay, offsets, dsT, nullptr, true,
                    share > 1 ? static_cast<void*>(sums) : dk, share > 1, ws, st))
    return rc;
  if (int rc = shared(dk, c.key_width)) return rc;
  if (int rc = kept(c, &dsT, ds0, ws + slots_size(c, c.key_width, c.value_width), st)) return rc;
  if (int rc = walk(c, ak, aq, ao, c.key_width, c.value_width, true, log_decay, offsets, dsT, ds0, false,
                    share > 1 ? static_cast<void*>(sums) : dv, share > 1, ws, st))
    return rc;
  if (int rc = shared(dv, c.value_width)) return rc;
  return set_ok();
}

int soma_la_step(const soma_la_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                 const float* s0, float* sT, void* o, void* stream) {
  if (int rc = check_shape(cfg)) return rc;
  const soma_la_config& c = *cfg;
  const size_t e = type_size(c.type);
  if (c.rows != c.sequences) return set_error(SOMA_ESHAPE, "a step takes one row for every sequence");
  if (!q || !k || !v || !log_decay || !sT || !o) return set_error(SOMA_EINVAL, "NULL device pointer");
  if (!is_aligned(q, e) || !is_aligned(k, e) || !is_aligned(v, e) || !is_aligned(o, e) || !is_aligned(s0, 4) ||
      !is_aligned(sT, 4) || !is_aligned(log_decay, 4))
    return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  const Spans n(c);
  if (!are_apart({n.o(o), n.state(sT)}, {n.q(q), n.k(k), n.v(v), n.state(s0 == sT ? nullptr : s0), n.decay(log_decay)}))
    return set_error(SOMA_EINVAL, "an output overlaps another array");
  Step a{q, k, v, c.q_stride, c.k_stride, c.v_stride, log_decay, s0, sT, o, c.heads, c.heads / c.kv_heads, c.key_width,
         c.value_width, c.scale};
  const bool wide = c.value_width % 4 == 0 && is_aligned(s0, 16) && is_aligned(sT, 16);
  const dim3 grid(static_cast<unsigned>(c.sequences) * c.heads);
  const auto kernel = c.type == SOMA_FLOAT ? (wide ? k_la_step<float, 4> : k_la_step<float, 1>)
                                           : (wide ? k_la_step<bf16, 4> : k_la_step<bf16, 1>);
  if (int rc = launch("k_la_step", kernel, grid, dim3(kThreads), 0, stream_of(stream), a)) return rc;
  return set_ok();
}

}  // extern "C"
