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
#include <initializer_list>
#include <type_traits>

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
  int whole;                                // both widths are whole units of 16 bytes
  void* out;                                // [rows][heads outer] of T, or fp32
  int out_float;
  const float *begin, *log_decay;           // states [sequences][heads][..], or NULL: zeros
  float* end;                               // the same, or NULL: not wanted
  int64_t row_stride, col_stride;           // of begin and end, an inner and an outer index
  const int32_t* offsets;                   // [sequences + 1], or NULL: `length` rows each
  int rows, length, sequences, heads, slices;
  int back;                                 // from the last row to the first
  float p_scale, in_scale, front_scale;     // of P, of the state's update, of what R gives
  int piece, pieces;                        // rows a piece (0: a block a sequence), pieces
  float* slots;                             // [pieces][heads][slices][a block's state]
};

// Walks of one launch: of the same instance, rows and pieces.
// Those of a head and part lie side by side on one XCD, whose L2 then gives the second
// and third what they share.  (Three gradients apart and together: 15 sequences of 630
// rows, 2 heads of 20 x 9 in bf16, both passes 125 and 75 us; 64 of 1,024, 8 heads of
// 64 x 64, 222 and 209.)
constexpr int kMostWalks = 3, kXcds = 8;
struct Walks {
  Walk walk[kMostWalks];
  int count, parts;                         // sequences or pieces
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

// A value that is not finite, told by its exponent's carry into the bit above.
template <class T>
__device__ __forceinline__ uint32_t not_finite(const uint4& u) {
  constexpr uint32_t e = sizeof(T) == 2 ? 0x7F807F80u : 0x7F800000u, one = sizeof(T) == 2 ? 0x00800080u : 0x00800000u,
                     top = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
  return (((u.x & e) + one) | ((u.y & e) + one) | ((u.z & e) + one) | ((u.w & e) + one)) & top;
}

// A value that the compiler takes for another every time: what is seldom used and formed
// from it is formed again there, not kept over a loop in registers.
__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// A value that is the same in every lane, in a scalar register.
__device__ __forceinline__ float first_lane(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }

// (a = 0: a^0 is 1)
__device__ __forceinline__ float log2_decay(const Walk& a, int head) {
  const float l = a.log_decay[head] * kL2e;
  return l < -1e30f ? -1e30f : l;
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

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

// A buffer from p on; what is read behind `bytes` is 0, what is written there is lost.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, static_cast<int>(bytes), 0x00020000);
}
// (16 bytes from here on do not wrap, nor less the 2^30 that a chunk is short of)
constexpr uint32_t kNowhere = 0xC0000000u;

// Rows of one array on their way to LDS: kRows x kCols, kThreads lanes side by side.
// They come through a buffer that ends with the chunk's last row: row r lies at r
// strides (walking back, at kRows - 1 - r less the rows that the chunk is short of,
// which wraps for those), and what is not there lies behind the end.  Loads of 16 bytes
// take any element's alignment.  A row's last unit may reach into what follows, which
// becomes 0, and a buffer ends in whole words: the last of an odd number of bf16 comes
// by itself.
template <class T, int kRows, int kCols, bool kWhole>
struct Tile {
  typedef Kind<T> K;
  static constexpr int kUnits = kCols / K::kEl, kMine = kRows * kUnits / kThreads, kStride = kCols + K::kPad;
  static_assert(kMine * kThreads == kRows * kUnits && kThreads % kUnits == 0, "every lane has as many units, of the same columns");
  uint4 u[kMine];
  uint32_t off[kMine];
  uint64_t at;                // of the chunk's first row in memory, if it were full
  uint32_t line, bytes;       // between rows; of a full chunk
  int c0, width, back;

  // `row`: the first one walked over
  __device__ __forceinline__ void start(const void* p, int64_t stride, int head, int columns, int from, int backward, int row) {
    c0 = from, width = columns, back = backward;
    line = static_cast<uint32_t>(stride) * static_cast<uint32_t>(sizeof(T));
    bytes = (kRows - 1) * line + width * static_cast<uint32_t>(sizeof(T));
    at = reinterpret_cast<uint64_t>(static_cast<const T*>(p) + static_cast<int64_t>(head) * columns) +
         static_cast<int64_t>(back ? row - (kRows - 1) : row) * line;
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
      const int i = threadIdx.x + kThreads * k, r = i / kUnits, c = c0 + i % kUnits * K::kEl;
      off[k] = c < width ? static_cast<uint32_t>(back ? kRows - 1 - r : r) * line + c * static_cast<uint32_t>(sizeof(T)) : kNowhere;
    }
  }
  // The next m rows.
  __device__ __forceinline__ void load(int m) {
    const uint32_t few = static_cast<uint32_t>(kRows - m) * line, less = back ? few : 0u;
    const auto buffer = buffer_of(reinterpret_cast<const void*>(at + less), bytes - few);
    const int step = static_cast<int>(kRows * line);
    at += back ? -step : step;
#pragma unroll
    for (int k = 0; k < kMine; ++k) u[k] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(buffer, off[k] - less, 0, 0));
    const int left = width % K::kEl;        // elements of a row's last unit, where it is not full
    if (!kWhole && left) {
      const int from = width - left - c0, words = left * static_cast<int>(sizeof(T)) / 4;
      const bool mine = static_cast<int>(threadIdx.x) % kUnits * K::kEl == from;   // (of every unit of a lane: kThreads is a multiple)
#pragma unroll
      for (int k = 0; k < kMine; ++k) {
        uint32_t w[4] = {u[k].x, u[k].y, u[k].z, u[k].w}, last = 0;
        if (sizeof(T) == 2 && left % 2) last = __builtin_amdgcn_raw_buffer_load_b16(buffer, mine ? off[k] - less + 2 * (left - 1) : kNowhere, 0, 0) & 0xFFFF;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i >= words && mine) w[i] = i == words ? last : 0;
        u[k] = make_uint4(w[0], w[1], w[2], w[3]);
      }
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

// What a state is multiplied with, again and again, to be taken over n rows each time.  A
// rounding of a^n to fp32 would be the same every time and add up (16,384 rows of
// log a = -3e-6 in chunks of 32: 1.4e-5 of the state).  So the factors differ in their last
// bit, and the first c of them sum up to c a^n, to 2^-24: their product is a^(c n) to
// (3 |c n log a| + 1) 2^-23.  For a^n below a half a state is gone before roundings count.
struct Factors {
  float near, rest;           // a^n, and what it lacks in units of 2^-24
  // (e^t - 1 by its series, whose tenth term is 2^-26 of it at the most)
  __device__ __forceinline__ Factors(float l2, int n) {
    const float y = l2 * static_cast<float>(n), t = y * 0.69314718f;
    constexpr float over[] = {1.0f, 1.0f / 2, 1.0f / 6, 1.0f / 24, 1.0f / 120, 1.0f / 720, 1.0f / 5040, 1.0f / 40320, 1.0f / 362880};
    float p = over[8];
#pragma unroll
    for (int k = 7; k >= 0; --k) p = fmaf(p, t, over[k]);
    const float less = p * t, sum = 1.0f + less, left = ((1.0f - sum) + less) * 0x1p24f;
    near = y > -1.0f ? sum : __builtin_amdgcn_exp2f(y);
    rest = y > -1.0f ? left : 0.0f;
  }
  __device__ __forceinline__ float at(int c) const {
    return near + (rintf(rest * static_cast<float>(c + 1)) - rintf(rest * static_cast<float>(c))) * 0x1p-24f;
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
template <class T, int kInner, int kTiles, bool kMap, bool kWhole>
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
  Factors over_chunk;          // of a full one
  float in[kC / K::kKw][K::kEl];
  int in_for;

  __device__ __forceinline__ explicit Walker(float log2_decay) : l2(log2_decay), over_chunk(l2, kC), in_for(-1) {
    // (what has to stay over all chunks, where lanes have no registers left for it)
    if constexpr (!kMap && !kWhole && (sizeof(T) == 2 ? kTiles == 2 : kInner * kTiles == 64)) {
      over_chunk.near = first_lane(over_chunk.near);
      over_chunk.rest = first_lane(over_chunk.rest);
    }
  }

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
  static __device__ __forceinline__ int outer_of(int wave, int n, int lane) { return (n * 4 + wave) * 16 + (lane & 15); }

  // Where elements 0 .. 3 of r[t][s][n] lie in a state, and whether they are 16 bytes.
  static __device__ __forceinline__ bool in_state(const Walk& a, int col0, int t, int s, int n, int l, uint32_t (&at)[4]) {
    const int c = col0 + outer_of(l >> 6, n, l & 63), d = inner_of(t, s, l & 63);
    const uint32_t rows = static_cast<uint32_t>(a.row_stride), cols = static_cast<uint32_t>(a.col_stride);
#pragma unroll
    for (int i = 0; i < 4; ++i) at[i] = c < a.outer && d + i < a.inner ? 4 * ((d + i) * rows + c * cols) : kNowhere;
    return rows == 1 && a.inner % 4 == 0;
  }
  // (through buffers: without a branch for each element; NULL is an empty one)
  __device__ __forceinline__ void read_state(const Walk& a, const float* p, int col0) {
    const int l = fresh(threadIdx.x);
    const auto buffer = buffer_of(p, p ? 4u * a.inner * a.outer : 0u);
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
          uint32_t at[4];
          if (in_state(a, col0, t, s, n, l, at)) {
            r[t][s][n] = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(buffer, at[0], 0, 0));
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) r[t][s][n][i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buffer, at[i], 0, 0));
          }
        }
  }
  __device__ __forceinline__ void write_state(const Walk& a, float* p, int col0) const {
    const int l = fresh(threadIdx.x);
    const auto buffer = buffer_of(p, 4u * a.inner * a.outer);
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
          uint32_t at[4];
          if (in_state(a, col0, t, s, n, l, at)) {
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, r[t][s][n]), buffer, at[0], 0, 0);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(r[t][s][n][i]), buffer, at[i], 0, 0);
          }
        }
  }
  // A slot holds the registers as they lie.
  static __device__ __forceinline__ int in_slot(int t, int s, int n) { return (((t * kSub + s) * kTiles + n) * kThreads) * 4; }
  __device__ __forceinline__ void read_slot(const float* p) {
    const int at = fresh(threadIdx.x) * 4;
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) r[t][s][n] = *reinterpret_cast<const f4*>(p + in_slot(t, s, n) + at);
  }
  __device__ __forceinline__ void write_slot(float* p) const {
    const int at = fresh(threadIdx.x) * 4;
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) *reinterpret_cast<f4*>(p + in_slot(t, s, n) + at) = r[t][s][n];
  }

  // Rows lo .. hi - 1 of the arrays.
  __device__ __forceinline__ void part(const Walk& a, int lo, int hi, int head, int col0, Word* lds) {
    Word* const ly = lds;
    Word* const lz = ly + kC * kXs;
    Word* const lx = lz + kC * kZs;
    Word* const lp = lx + kC * kXs;
    uint32_t* const flags = reinterpret_cast<uint32_t*>(kMap ? lx : lp + kPWords);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, li = lane & 15;
    const int n = hi - lo, row0 = a.back ? hi - 1 : lo;
    // fp32 widths that nobody rounded: no products of columns that are filled up, which
    // the fp32 MFMA's rate makes worth the branches (45 x 77: walks 88 -> 68 us)
    constexpr bool kSkip = !kWhole && sizeof(T) == 4 && kInner < 256;
    const int own_wave = __builtin_amdgcn_readfirstlane(wave);
    const auto step_out = [&](int t) { return kSkip && t * K::kKw >= a.inner; };
    const auto tile_out = [&](int k) { return kSkip && col0 + (k * 4 + own_wave) * 16 >= a.outer; };

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

    Tile<T, kC, kInner, kWhole> tx, ty;
    Tile<T, kC, kCols, kWhole> tz;
    if constexpr (!kMap) tx.start(a.x, a.x_stride, head / a.x_share, a.inner, 0, a.back, row0);
    ty.start(a.y, a.y_stride, head / a.y_share, a.inner, 0, a.back, row0);
    tz.start(a.z, a.z_stride, head / a.z_share, a.outer, col0, a.back, row0);
    const auto fetch = [&](int c) {
      const int m = min(kC, n - c);
      if constexpr (!kMap) tx.load(m);
      ty.load(m);
      tz.load(m);
    };
    // out's rows, the same way
    const uint32_t size = a.out_float ? 4 : sizeof(T), line = static_cast<uint32_t>(a.heads) * a.outer * size;
    uint32_t out_off[kTiles];
#pragma unroll
    for (int k = 0; k < kTiles; ++k) {
      const int col = col0 + (k * 4 + wave) * 16 + 4 * g;
      out_off[k] = col < a.outer ? (a.back ? kC - 1 - li : li) * line + col * size : kNowhere;
    }
    const auto place = [&](int flag) {
      if constexpr (!kMap) tx.store(lx);
      ty.store(ly);
      const uint32_t bad = tz.store(lz);
      if constexpr (!kMap)
        if (bad) flags[flag] = 1;
    };
    uint64_t out_at = reinterpret_cast<uint64_t>(a.out) + static_cast<int64_t>(a.back ? row0 - (kC - 1) : row0) * line +
                      static_cast<int64_t>(head) * a.outer * size;
    fetch(0);
    place(0);
    __syncthreads();
    for (int c = 0; c < n; c += kC) {
      const int m = min(kC, n - c), flag = (c / kC) & 1;
      if (c + kC < n) fetch(c + kC);
      if (in_for != m) weights(a, m);
      bool slow = false;
      if constexpr (!kMap) {
        slow = flags[flag] != 0;
        // P, tiles 0 .. below and on the diagonal in the order of their rows
#pragma unroll
        for (int k = 0; k < (kRowTiles * (kRowTiles + 1) / 2 + 3) / 4; ++k) {
          const int t = own_wave + 4 * k;
          const int ti = t >= 6 ? 3 : t >= 3 ? 2 : t >= 1 ? 1 : 0, tj = t - ti * (ti + 1) / 2;
          if (tj > ti || ti >= kRowTiles || 16 * ti >= m) break;
          f4 p = {0, 0, 0, 0};
#pragma unroll
          for (int s = 0; s < kSteps; ++s)
            if (!step_out(s)) p = mfma(along<T>(ly, kXs, 16 * tj, s * K::kKw), along<T>(lx, kXs, 16 * ti, s * K::kKw), p);
          if (ti == tj) {
            const int below_at = fresh(li - 4 * g);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = below_at >= i ? p[i] * at[i] : 0.0f;
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
          if (step_out(s)) break;
          Frag fx[kRowTiles];
#pragma unroll
          for (int i = 0; i < kRowTiles; ++i) fx[i] = along<T>(lx, kXs, 16 * i, s * K::kKw);
#pragma unroll
          for (int k = 0; k < kTiles; ++k) {
            if (tile_out(k)) continue;
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
      const float keep = m == kC ? over_chunk.at(c / kC) : power(m);
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
          for (int k = 0; k < kTiles; ++k) fz[k] = across(lz, kZs, j * K::kKw, (k * 4 + wave) * 16, 4);
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
                for (int k = 0; k < kTiles; ++k)
                  if (!tile_out(k)) o[i][k] = mfma(fv[k], fp, o[i][k]);
                if constexpr (K::kParts == 2) {
                  const Frag fl = along<T>(lp + kC * kPs, kPs, 16 * i, j * K::kKw);
#pragma unroll
                  for (int k = 0; k < kTiles; ++k)
                    if (!tile_out(k)) o[i][k] = mfma(fv[k], fl, o[i][k]);
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
          for (int t = 0; t < kSteps; ++t) {
            if (step_out(t)) break;
#pragma unroll
            for (int s = 0; s < kSub; ++s) {
              const Frag fy = across(ly, kXs, j * K::kKw, t * K::kKw + 4 * s, K::kEl);
#pragma unroll
              for (int k = 0; k < kTiles; ++k)
                if (!tile_out(k)) {
#pragma unroll
                  for (int q = kZParts - 1; q >= 0; --q) r[t][s][k] = mfma(fy, zw[k][q], r[t][s][k]);
                }
            }
          }
        }
      }

      if constexpr (!kMap) {
        if (slow) {
          const int l = fresh(threadIdx.x);
          const int wave = l >> 6, g = (l & 63) >> 4, li = l & 15;
          for (int j = 0; j < m; ++j)
#pragma unroll
            for (int k = 0; k < kTiles; ++k) {
              float v[4];
              bool any = false;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const Word w = lz[j * kZs + (k * 4 + wave) * 16 + 4 * g + e];
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
      }
      __syncthreads();  // the tiles have been read
      // (the next ones in front of this chunk's stores: a wait for loads is one for what
      // was stored before them)
      if (c + kC < n) place(flag ^ 1);
      if constexpr (!kMap) {
        const uint32_t few = static_cast<uint32_t>(kC - m) * line, less = a.back ? few : 0u;
        const auto buffer = buffer_of(reinterpret_cast<const void*>(out_at + less), (kC - 1) * line + a.outer * size - few);
        const int step = static_cast<int>(kC * line);
        out_at += a.back ? -step : step;
        const bool ragged = !kWhole && a.outer % 4;
        const auto put = [&](auto wide) {
#pragma unroll
          for (int i = 0; i < kRowTiles; ++i)
#pragma unroll
            for (int k = 0; k < kTiles; ++k) {
              const f4& v = o[i][k];
              const uint32_t at = out_off[k] + (a.back ? -(16 * i * line) : 16 * i * line) - less;
              const uint32_t pair[2] = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
              const int left = a.outer - (col0 + (k * 4 + wave) * 16 + 4 * g);
              const uint32_t there = ragged && left < 4 ? kNowhere : at;   // (out_off is, where none is left)
              if constexpr (wide) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, v), buffer, there, 0, 0);
              else __builtin_amdgcn_raw_buffer_store_b64(u2{pair[0], pair[1]}, buffer, there, 0, 0);
              if (ragged) {
                const bool some = left > 0 && left < 4;
#pragma unroll
                for (int e = 0; e < 3; ++e) {
                  if constexpr (wide) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[e]), buffer, some && e < left ? at + 4 * e : kNowhere, 0, 0);
                  else __builtin_amdgcn_raw_buffer_store_b16(static_cast<short>(pair[e / 2] >> (16 * (e & 1))), buffer, some && e < left ? at + 2 * e : kNowhere, 0, 0);
                }
              }
            }
        };
        if constexpr (sizeof(T) == 4) {
          put(std::true_type());
        } else {
          if (a.out_float) put(std::true_type());
          else put(std::false_type());
        }
      }
      __syncthreads();
    }
  }
};

// 64 sequences of 1,024 rows, 8 heads of 64 x 64 in bf16: 70 to 76 us a walk, 3.5 to 3.8
// TB/s where a copy's rate would take 52 (forward 76, the three gradients together 210).
// Nothing is saturated: of a SIMD's cycles 38% issue vector instructions, most of them to
// split fp32 into parts, 20% keep the matrix cores busy, and LDS works in 42%; the rest
// are waits between a chunk's three barriers.  Without loads and stores it would take 55,
// without P 60.  Tried and left out: a third block a compute unit (no faster, and the
// registers do not reach), rows that leave through LDS as whole lines (70.7 for 71).
//
// Blocks that share a compute unit: what the state's registers leave room for (fp32, 158
// sequences of 483 rows, 2 heads of 32 x 53, both passes: four blocks 184 us, three 230).
constexpr int blocks_of(size_t element, int inner, int tiles) { return inner == 256 ? 1 : element == 4 && inner * tiles == 64 ? 4 : 2; }

template <class T, int kInner, int kTiles, bool kMap, bool kWhole>
__global__ __launch_bounds__(kThreads, blocks_of(sizeof(T), kInner, kTiles)) void k_la_walk(const Walks all) {
  typedef Walker<T, kInner, kTiles, kMap, kWhole> W;
  const int turn = blockIdx.x / kXcds, group = __builtin_amdgcn_readfirstlane(turn / all.count);
  const int block = group * kXcds + blockIdx.x % kXcds;
  const Walk a = all.walk[turn - group * all.count];
  __shared__ __align__(16) unsigned char memory[W::kLds];
  typename W::Word* const lds = reinterpret_cast<typename W::Word*>(memory);
  const int units = a.heads * a.slices;
  const int p = block / units, unit = block % units, head = unit / a.slices, slice = unit % a.slices;
  if (p >= all.parts) return;
  const int col0 = slice * W::kCols;
  W w(log2_decay(a, head));
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
    int lo = 0, hi = 0;
    if (s >= 0 && first_row(a, s + 1) > border) {
      const int b = first_row(a, s), e = first_row(a, s + 1), far = min(p + 1 < a.pieces ? (p + 1) * a.piece : a.rows, a.rows);
      lo = a.back ? border : max(b, p * a.piece);
      hi = a.back ? min(e, far) : border;
    }
    if (hi <= lo) return;
    w.zero();
    w.part(a, lo, hi, head, col0, lds);
    w.write_slot(a.slots + (static_cast<int64_t>(p) * units + unit) * W::kState);
  } else {
    // one sequence, or those of a piece
    const bool whole = !a.piece, last = whole || p + 1 == a.pieces;
    const int lo = whole ? 0 : p * a.piece, hi = last ? a.rows : lo + a.piece;
    const int s0 = whole ? p : sequence_from(a, lo), s1 = whole ? p : last ? a.sequences - 1 : sequence_before(a, hi);
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

// (one sequence of 16,384 rows, 16 heads of 128 x 128 in bf16: maps 41 us, joined 9, walk
// 105, where one block a head and slice would walk for more than a millisecond)
//
// From what every piece adds to the state with which the next is entered, in the slot
// of the piece that is left: for every sequence, one after another over its pieces.
template <class T, int kInner, int kTiles>
__global__ __launch_bounds__(kThreads) void k_la_join(const Walks all) {
  typedef Walker<T, kInner, kTiles, true, true> W;
  const Walk& a = all.walk[blockIdx.y];
  constexpr int kPer = W::kState / 4, kAhead = 8;
  const int units = a.heads * a.slices, blocks = (units * kPer + kThreads - 1) / kThreads;
  const int s = blockIdx.x / blocks, id = static_cast<int>(blockIdx.x % blocks) * kThreads + static_cast<int>(threadIdx.x);
  const int unit = id / kPer, at = id % kPer;
  const int b = first_row(a, s), e = first_row(a, s + 1);
  if (e <= b || unit >= units) return;
  const int front = b / a.piece, back = (e - 1) / a.piece, count = back - front;
  if (count == 0) return;
  const int head = unit / a.slices, slice = unit % a.slices;
  const float l = log2_decay(a, head);
  // (of the pieces that are left only the first may hold fewer rows of the sequence)
  const Factors over_piece(l, a.piece);
  const int first = (a.back ? e - back * a.piece : (front + 1) * a.piece - b);
  const float over_first = __builtin_amdgcn_exp2f(l * static_cast<float>(first));
  f4 state = {0, 0, 0, 0};
  if (a.begin) {
    const int lane = at & 63, wave = (at >> 6) & 3, tile = at / kThreads;
    const int n = tile % kTiles, sub = tile / kTiles % W::kSub, t = tile / kTiles / W::kSub;
    const int c = slice * W::kCols + W::outer_of(wave, n, lane), d = W::inner_of(t, sub, lane);
    const float* p = a.begin + (static_cast<int64_t>(s) * a.heads + head) * a.inner * a.outer;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c < a.outer && d + i < a.inner) state[i] = p[(d + i) * a.row_stride + c * a.col_stride];
  }
  const auto slot = [&](int i) {
    const int p = a.back ? back - i : front + i;
    return reinterpret_cast<f4*>(a.slots + (static_cast<int64_t>(p) * units + unit) * W::kState + at * 4);
  };
  for (int i0 = 0; i0 < count; i0 += kAhead) {
    f4 add[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i0 + k < count) add[k] = *slot(i0 + k);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i0 + k >= count) break;
      state = state * (i0 + k ? over_piece.at(i0 + k) : over_first) + add[k];
      *slot(i0 + k) = state;
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
// few rows one of them.  Reads and writes the state once; bound by memory (64 sequences,
// 8 heads of 64 x 64: 16.8 MB in 5.7 us, from and into the caches).
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
constexpr int kEnough = 512;       // blocks that fill the card
constexpr int64_t kMostStride = 1 << 22;   // a chunk's offsets in a buffer stay below 2^31

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
  if (static_cast<int64_t>(c.sequences) * c.heads * ((std::max(c.key_width, c.value_width) + 63) / 64) * kThreads >= kMostThreads)
    return set_error(SOMA_ESHAPE, "more sequences and heads than a launch has blocks for");
  for (int64_t stride : {c.q_stride, c.k_stride, c.v_stride})
    if (stride > kMostStride) return set_error(SOMA_ESHAPE, "a row stride is out of range");
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
  // (128 columns of X with two tiles a wave leave a compute unit one block: 16,384 rows of
  // 16 heads of 128 x 128 in bf16, forward, 223 us; in two slices 164)
  s.tiles = outer <= 64 || s.inner >= 128 ? 1 : 2;
  s.slices = (outer + 64 * s.tiles - 1) / (64 * s.tiles);
  return s;
}

// Pieces: none where every sequence has its blocks and they are enough, or short.
// Their number goes by the heads alone, so that a workspace serves fewer rows too.
int most_pieces(const soma_la_config& c, const Shape& s, int walks) {
  const int64_t units = static_cast<int64_t>(c.heads) * s.slices * walks;
  const int few = c.type == SOMA_FLOAT ? 4 * Kind<float>::kC : 4 * Kind<bf16>::kC;
  if (units * c.sequences >= kEnough || c.rows <= static_cast<int64_t>(c.sequences) * few) return 0;
  return static_cast<int>(std::min<int64_t>(kMostPieces, (kEnough + units - 1) / units));
}

size_t slots_size(const soma_la_config& c, int inner, int outer, int walks) {
  const Shape s = shape_of(inner, outer);
  const int most = most_pieces(c, s, walks);
  if (!most) return 0;
  return up256(sizeof(float) * most * c.heads * s.slices * s.inner * 64 * s.tiles);
}

// A copy of the states that a walk begins with, where it ends with the same array and
// goes in pieces: one block may then read a state after another has written it.  (A walk in
// pieces as `together` would be is in pieces by itself: the size holds for both.)
size_t copy_size(const soma_la_config& c) {
  if (!most_pieces(c, shape_of(c.key_width, c.value_width), 1)) return 0;
  return up256(sizeof(float) * c.sequences * c.heads * c.key_width * c.value_width);
}

int kept(const soma_la_config& c, int together, const float** begin, const float* end, unsigned char* at, hipStream_t st) {
  if (!*begin || *begin != end || !most_pieces(c, shape_of(c.key_width, c.value_width), together)) return SOMA_OK;
  const int64_t n = static_cast<int64_t>(c.sequences) * c.heads * c.key_width * c.value_width;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((n + kThreads - 1) / kThreads, 4096)));
  const float* from = *begin;
  *begin = reinterpret_cast<const float*>(at);
  return launch("k_la_copy", k_la_copy, grid, dim3(kThreads), 0, st, from, reinterpret_cast<float*>(at), n);
}

// fp32 gradients of every head, where heads share keys and values: of keys or values
size_t sums_size(const soma_la_config& c, int width) {
  return c.heads == c.kv_heads ? 0 : up256(sizeof(float) * c.rows * c.heads * width);
}

// Whether the walks for dq, dk and dv are of one shape.
bool are_alike(const soma_la_config& c) {
  const Shape a = shape_of(c.key_width, c.value_width), b = shape_of(c.value_width, c.key_width);
  return a.inner == b.inner && a.tiles == b.tiles && a.slices == b.slices;
}

// Slots of the walks that run together, and behind them the copy and the sums.
size_t all_slots(const soma_la_config& c, bool grad) {
  const size_t one = slots_size(c, c.key_width, c.value_width, 1);
  if (!grad) return one;
  return are_alike(c) ? std::max(one, 3 * slots_size(c, c.value_width, c.key_width, 3))
                      : std::max(one, 2 * slots_size(c, c.value_width, c.key_width, 2));
}

size_t la_workspace(const soma_la_config& c, bool grad) {
  const size_t n = all_slots(c, grad) + copy_size(c);
  return grad ? n + sums_size(c, c.key_width) + sums_size(c, c.value_width) : n;
}

template <class T, int kInner, int kTiles>
int walk_as(const Walks& all, hipStream_t st) {
  const Walk& a = all.walk[0];
  const int units = a.heads * a.slices;
  // (several walks share out whole rounds of the XCDs; one may have as many blocks as a launch)
  const unsigned each = static_cast<unsigned>(units) * all.parts;
  const dim3 grid(all.count == 1 ? each : (each + kXcds - 1) / kXcds * kXcds * all.count), block(kThreads);
  if (a.piece) {
    if (int rc = launch("k_la_walk (maps)", a.whole ? k_la_walk<T, kInner, kTiles, true, true> : k_la_walk<T, kInner, kTiles, true, false>,
                        grid, block, 0, st, all))
      return rc;
    const unsigned blocks = (units * (kInner * 64 * kTiles / 4) + kThreads - 1) / kThreads;
    if (int rc = launch("k_la_join", k_la_join<T, kInner, kTiles>, dim3(blocks * a.sequences, all.count), block, 0, st, all))
      return rc;
  }
  return launch("k_la_walk", a.whole ? k_la_walk<T, kInner, kTiles, false, true> : k_la_walk<T, kInner, kTiles, false, false>, grid,
                block, 0, st, all);
}

template <class T>
int walk_of(const Walks& all, const Shape& s, hipStream_t st) {
  if (s.inner == 64) return s.tiles == 1 ? walk_as<T, 64, 1>(all, st) : walk_as<T, 64, 2>(all, st);
  if (s.inner == 128) return walk_as<T, 128, 1>(all, st);
  return walk_as<T, 256, 1>(all, st);
}

// An array of rows and what a walk needs to know of it.
struct Array {
  const void* p;
  int64_t stride;
  int share;
};

Walk walk_over(const soma_la_config& c, const Array& x, const Array& y, const Array& z, int inner, int outer, bool back,
               const float* begin, float* end, bool transposed, void* out, bool out_float) {
  Walk a{};
  a.x = x.p, a.y = y.p, a.z = z.p;
  a.x_stride = x.stride, a.y_stride = y.stride, a.z_stride = z.stride;
  a.x_share = x.share, a.y_share = y.share, a.z_share = z.share;
  a.inner = inner, a.outer = outer;
  a.out = out;
  a.out_float = out_float;
  a.begin = begin, a.end = end;
  a.row_stride = transposed ? 1 : outer;
  a.col_stride = transposed ? inner : 1;
  a.back = back;
  a.p_scale = c.scale;
  a.in_scale = back ? c.scale : 1.0f;
  a.front_scale = back ? 1.0f : c.scale;
  return a;
}

// Up to kMostWalks walks of one shape in one launch, in pieces as `together` would be.
int walk(const soma_la_config& c, std::initializer_list<Walk> walks, int together, const float* log_decay, const int32_t* offsets,
         unsigned char* ws, hipStream_t st) {
  Walks all{};
  const Shape s = shape_of(walks.begin()->inner, walks.begin()->outer);
  const int most = most_pieces(c, s, together);
  if (walks.size() > 1 && !most && (static_cast<int64_t>(c.sequences) * c.heads * s.slices + kXcds) * walks.size() * kThreads >= kMostThreads) {
    for (const Walk& w : walks)
      if (int rc = walk(c, {w}, together, log_decay, offsets, ws, st)) return rc;
    return SOMA_OK;
  }
  for (const Walk& w : walks) {
    Walk& a = all.walk[all.count];
    a = w;
    a.whole = a.inner * type_size(c.type) % 16 == 0 && a.outer * type_size(c.type) % 16 == 0;
    a.log_decay = log_decay, a.offsets = offsets;
    a.rows = c.rows, a.length = c.rows / c.sequences, a.sequences = c.sequences, a.heads = c.heads, a.slices = s.slices;
    if (most) {
      a.piece = ((c.rows + most - 1) / most + 63) / 64 * 64;
      a.pieces = (c.rows + a.piece - 1) / a.piece;
      a.slots = reinterpret_cast<float*>(ws + all.count * slots_size(c, a.inner, a.outer, together));
    }
    ++all.count;
  }
  all.parts = most ? all.walk[0].pieces : c.sequences;
  return c.type == SOMA_FLOAT ? walk_of<float>(all, s, st) : walk_of<bf16>(all, s, st);
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
  if (int rc = kept(c, 1, &s0, sT, ws + all_slots(c, false), st)) return rc;
  const Walk to_o = walk_over(c, {q, c.q_stride, 1}, {k, c.k_stride, share}, {v, c.v_stride, share}, c.key_width, c.value_width,
                              false, s0, sT, false, o, false);
  if (int rc = walk(c, {to_o}, 1, log_decay, offsets, ws, st)) return rc;
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
  float *key_sums = nullptr, *value_sums = nullptr;
  if (share > 1) {
    unsigned char* const at = ws + all_slots(c, true) + copy_size(c);
    key_sums = reinterpret_cast<float*>(at);
    value_sums = reinterpret_cast<float*>(at + sums_size(c, c.key_width));
  }
  const auto shared = [&](const float* sums, void* out, int width) -> int {
    if (share == 1 || c.rows == 0) return SOMA_OK;
    const int64_t n = static_cast<int64_t>(c.rows) * c.kv_heads * width;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((n + kThreads - 1) / kThreads, 8192)));
    if (c.type == SOMA_FLOAT)
      return launch("k_la_share", k_la_share<float>, grid, dim3(kThreads), 0, st, sums, static_cast<float*>(out), n, width, share,
                    offsets, c.sequences, c.rows, c.kv_heads * width);
    return launch("k_la_share", k_la_share<bf16>, grid, dim3(kThreads), 0, st, sums, static_cast<bf16*>(out), n, width, share,
                  offsets, c.sequences, c.rows, c.kv_heads * width);
  };
  const Walk to_dq = walk_over(c, ao, av, ak, c.value_width, c.key_width, false, s0, nullptr, true, dq, false);
  const Walk to_dk = walk_over(c, av, ao, aq, c.value_width, c.key_width, true, dsT, nullptr, true,
                               share > 1 ? static_cast<void*>(key_sums) : dk, share > 1);
  const auto to_dv = [&] {
    return walk_over(c, ak, aq, ao, c.key_width, c.value_width, true, dsT, ds0, false,
                     share > 1 ? static_cast<void*>(value_sums) : dv, share > 1);
  };
  // (dsT in ds0's place is read for dk before dv's walk writes it; the pieces stay the
  // same, and with them the bits)
  const bool alike = are_alike(c);
  if (alike && (!dsT || dsT != ds0)) {
    if (int rc = walk(c, {to_dv(), to_dk, to_dq}, 3, log_decay, offsets, ws, st)) return rc;
  } else {
    if (int rc = walk(c, {to_dk, to_dq}, alike ? 3 : 2, log_decay, offsets, ws, st)) return rc;
    if (int rc = kept(c, alike ? 3 : 1, &dsT, ds0, ws + all_slots(c, true), st)) return rc;
    if (int rc = walk(c, {to_dv()}, alike ? 3 : 1, log_decay, offsets, ws, st)) return rc;
  }
  if (int rc = shared(key_sums, dk, c.key_width)) return rc;
  if (int rc = shared(value_sums, dv, c.value_width)) return rc;
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
