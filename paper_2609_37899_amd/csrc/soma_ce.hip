// soma_ce.hip -- softmax cross entropy of a linear head over a large vocabulary
// and its gradients, without the logits in memory.
//
//   l_rv = f_r . E_v,   lse_r = log sum_v e^l_rv,   loss_r = lse_r - l_{r,t_r};
//   G_rv = w_r (e^(l_rv - lse_r) - [v = t_r]),   df = G E,   dE = G^T f.
//
// All four products run on the matrix cores (k_ce_mm) over operands in MFMA
// fragment order (below).  The loss keeps, of every row, the maximum and the
// sum of exponentials of each 64 or 128 logits, and joins them at the end; the
// gradient forms the logits again, a piece of the vocabulary at a time,
// stores the piece of G only (in 16 bits, in the order that either product
// reads), and multiplies it by the piece of E (added to df) and by f (the piece
// of dE).  So the work is 8 R V K operations instead of 6, for a piece's
// values in memory instead of R V.
//
// Types.  bf16: E and f as they are, G rounded to bf16 (half a step, 2^-8, of
// every value; as much as the result's own rounding), sums in fp32.  fp32: every
// operand as two fp16 parts, x s = hi + lo to nearest with a power of two s that
// brings its array's largest magnitude to 2^13 .. 2^14, and a b as lo hi + hi lo
// + hi hi: 2^-22 of a value, or 2^-38 of its array's largest.  The weight w_r
// enters as c (w_r / c) with c the largest finite |w|, whose c is multiplied in fp32:
// under a mean, the common case, the factor inside is exactly 1.  (A weight that is
// not finite is its row's alone.)
//
// Fragment order: a matrix [rows][K] is blocks of 1 KiB, [row / 16][part][k / 32],
// of 64 words of 8 halves, word 16 lg + lr holding row lr, k 8 lg .. + 7: what lane
// (lr, lg) feeds an MFMA.  A block moves to LDS by one DMA.  The packing kernels
// write it (rows and their transpose), zeros beyond the matrix; so sizes, strides
// and rows without a target are theirs alone to deal with.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "soma.h"
#include "soma_host.hpp"
#include "soma_kernels.hpp"
#include "soma_types.hpp"

namespace soma {
namespace {

// Vocabulary rows of a piece.  Each adds its part of df to the sums of the ones
// before (8 bytes of each output moved), and at 16,384 the products of a training
// batch of 8,192 rows fill the card without shares; at more rows 8,192, which
// halves what a piece of G takes.
constexpr int kPiece = 8192, kLongPiece = 16384, kLongRows = 8192;
constexpr int kMaxima = 1024;         // partial maxima of an array
constexpr float kLog2 = 0.6931471805599453f;
constexpr float kLowest = -2.3e38f;   // below every logit that counts; log2 e times it is finite
constexpr int kBlk = 512;             // halves of a fragment block
constexpr int kXcd = 8;

// One row's part of the problem.  A row without a target has rho = 0, lse = 0.
struct RowMeta {
  float lse, rho;
  int target, pad;
};

// Scales of the fp32 path (1 for bf16) and the largest finite weight.
struct Scales {
  float f, e, c, pad;
};
constexpr float kScaleG = 8192.0f;    // |G / c| <= 1

// 2^n with n chosen so that top 2^n lies in [2^13, 2^14).
__device__ __forceinline__ float power_scale(float top) {
  if (!(top > 0.0f)) return 1.0f;
  int n = 13 - (static_cast<int>((__float_as_uint(top) >> 23) & 255u) - 127);
  n = n > 120 ? 120 : n;              // tiny arrays: the scale stays finite
  return __uint_as_float(static_cast<uint32_t>(n + 127) << 23);
}

__device__ __forceinline__ float finite_abs(float x) {
  const float a = __builtin_fabsf(x);
  return a <= 3.402823466e38f ? a : 0.0f;
}

// Values at any address of their type: the card loads 16 bytes from any of them
// (1 row, 25,969 x 510 in bf16: 14.7 us, value by value into a packed copy 54.6).
template <class V, class T>
__device__ __forceinline__ V load_any(const T* p) {
  V v;
  __builtin_memcpy(&v, p, sizeof(V));
  return v;
}
__device__ __forceinline__ float4 load_four_any(const float* p) { return load_any<float4>(p); }
__device__ __forceinline__ float4 load_four_any(const bf16* p) {
  const uint2 u = load_any<uint2>(p);
  return make_float4(from_bf16(u.x), __uint_as_float(u.x & 0xFFFF0000u), from_bf16(u.y), __uint_as_float(u.y & 0xFFFF0000u));
}

// Maximum over a block of 256 threads.
__device__ __forceinline__ float block_max(float v, float* lds) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
  __syncthreads();
  return v;
}

// The largest of an array's partial maxima.
__device__ __forceinline__ float maximum_of(const float* m, int n, float* lds) {
  static_assert(kMaxima == 4 * 256, "four a thread");
  const float4 v = int(threadIdx.x) * 4 < n ? reinterpret_cast<const float4*>(m)[threadIdx.x] : make_float4(0.f, 0.f, 0.f, 0.f);
  return block_max(fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)), lds);
}

// ---------------------------------------------------------------------------
// Largest finite magnitudes: f (rows with a target), E, and the weights.
// Block x of array y writes maxima[y][x].  Bound by memory: 33 MB of f in 8 us
// (4.2 TB/s).
// ---------------------------------------------------------------------------
struct MaxArgs {
  const void *f, *E;
  const float* w;
  const int32_t* targets;
  int64_t f_stride, e_stride;
  int R, V, K;
  float* maxima;        // [3][kMaxima]
};

template <class T>
__global__ __launch_bounds__(256) void k_ce_max(MaxArgs a, int first) {
  __shared__ float lds[4];
  const int which = first + blockIdx.y;
  float top = 0.0f;
  if (which < 2) {
    const T* x = static_cast<const T*>(which ? a.E : a.f);
    const int64_t stride = which ? a.e_stride : a.f_stride;
    const int rows = which ? a.V : a.R;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int r = blockIdx.x * 4 + wave; r < rows; r += gridDim.x * 4) {
      if (!which && a.targets[r] < 0) continue;
      const T* p = x + r * stride;
      int k = lane * 4;
#pragma unroll 4
      for (; k + 4 <= a.K; k += 256) {
        const float4 v = load_four_any(p + k);
        top = fmaxf(fmaxf(fmaxf(top, finite_abs(v.x)), fmaxf(finite_abs(v.y), finite_abs(v.z))), finite_abs(v.w));
      }
      for (int i = 0; i < 4 && k + i < a.K; ++i) top = fmaxf(top, finite_abs(load_value(p + k + i)));
    }
  } else if (a.w) {
    for (int r = blockIdx.x * 256 + threadIdx.x; r < a.R; r += gridDim.x * 256)
      if (a.targets[r] >= 0) top = fmaxf(top, finite_abs(a.w[r]));
  }
  top = block_max(top, lds);
  if (threadIdx.x == 0) a.maxima[which * kMaxima + blockIdx.x] = top;
}

// ---------------------------------------------------------------------------
// Packing: rows [row0, row0 + n) of a matrix into fragment order, and its
// transpose.  A block takes 64 rows x 64 columns through LDS; out-of-range ones
// and rows without a target are zeros.
// ---------------------------------------------------------------------------
struct PackArgs {
  const void* x;
  int64_t stride;
  int n, K;                  // rows, columns
  int np, Kp;                // padded to 128
  const int32_t* targets;    // f only: rows with a negative target are zeros
  uint16_t *frag, *fragT;    // [np / 16][parts][Kp / 32], [Kp / 16][parts][np / 32] blocks; or NULL
  const float* maxima;       // [3][kMaxima] or NULL: scale 1, c 1
  int which;                 // the scale to use: 0 f, 1 E
  int nmax;                  // partial maxima in use, a multiple of 4
  Scales* scales;            // f: written by block (0, 0)
  RowMeta* meta;             // f: rows' constants, or NULL
  const float *lse, *w;
  int V;
};

// f and the first piece of E in one launch, or a later piece alone: blocks from
// `first` on (of the grid's x) take the second.
struct PackPair {
  PackArgs a[2];
  int first;
};

__device__ __forceinline__ void split_rn(float x, uint16_t& hi, uint16_t& lo) {
  const _Float16 h = static_cast<_Float16>(x);
  hi = __builtin_bit_cast(uint16_t, h);
  lo = __builtin_bit_cast(uint16_t, static_cast<_Float16>(x - static_cast<float>(h)));
}

__device__ __forceinline__ uint4 pack8(const uint16_t (&h)[8]) {
  return make_uint4(h[0] | uint32_t(h[1]) << 16, h[2] | uint32_t(h[3]) << 16, h[4] | uint32_t(h[5]) << 16,
                    h[6] | uint32_t(h[7]) << 16);
}

// Eight values as a word of 8 halves of each part.
template <int PARTS>
__device__ __forceinline__ void fragment_words(const float (&v)[8], float scale, uint4 (&w)[PARTS]) {
  if constexpr (PARTS == 1) {
    w[0] = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
  } else {
    uint16_t hi[8], lo[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) split_rn(v[i] * scale, hi[i], lo[i]);
    w[0] = pack8(hi);
    w[PARTS - 1] = pack8(lo);
  }
}

// A wave takes a row tile (16 rows) of the block's 64 columns: a lane's eight
// values are a word of the fragment as they come from memory.  For the transpose
// the words go through LDS, where a lane picks eight rows of its column.  Bound by
// memory: 16,320 fp32 rows of 512 columns as two parts in 13 us (5.1 TB/s), with
// the transpose in 18 (5.6 TB/s, part of it held by the L2).
template <class T, int PARTS>
__global__ __launch_bounds__(256) void k_ce_pack(PackPair pair) {
  constexpr int kRow = 64 + 8;               // halves: 16-byte rows, columns of 8 rows on different banks
  __shared__ __attribute__((aligned(16))) uint16_t tile[PARTS][64][kRow];
  __shared__ float red[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const bool second = int(blockIdx.x) >= pair.first;
  const PackArgs& a = pair.a[second];
  const int r0 = (int(blockIdx.x) - (second ? pair.first : 0)) * 64, k0 = blockIdx.y * 64;
  const T* x = static_cast<const T*>(a.x);
  const int row = r0 + wave * 16 + lr;
  float v[2][8] = {};
  if (row < a.n && (!a.targets || a.targets[row] >= 0)) {
    const T* p = x + row * a.stride + k0 + 8 * lg;
#pragma unroll
    for (int kc = 0; kc < 2; ++kc) {
      const int left = a.K - (k0 + 32 * kc + 8 * lg);
      if (left >= 8) {
        const float4 lo = load_four_any(p + 32 * kc), hi = load_four_any(p + 32 * kc + 4);
        v[kc][0] = lo.x, v[kc][1] = lo.y, v[kc][2] = lo.z, v[kc][3] = lo.w;
        v[kc][4] = hi.x, v[kc][5] = hi.y, v[kc][6] = hi.z, v[kc][7] = hi.w;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < left) v[kc][j] = load_value(p + 32 * kc + j);
      }
    }
  }
  float scale = 1.0f, c = 1.0f;
  if (a.maxima) {
    if constexpr (PARTS == 2) {
      scale = power_scale(maximum_of(a.maxima + a.which * kMaxima, a.nmax, red));
    }
    if (a.scales && blockIdx.y == 0) {       // f, its first columns: the rows' constants too
      c = maximum_of(a.maxima + 2 * kMaxima, a.nmax, red);
      float e = 1.0f;
      if constexpr (PARTS == 2) {
        e = power_scale(maximum_of(a.maxima + kMaxima, a.nmax, red));
      }
      if (r0 == 0 && threadIdx.x == 0) *a.scales = Scales{scale, e, c, 0.0f};
    }
  }
  if (a.meta && blockIdx.y == 0 && threadIdx.x < 64) {
    const int r = r0 + threadIdx.x;          // < np
    RowMeta m{0.0f, 0.0f, -1, 0};
    if (r < a.n) {
      const int t = a.targets[r];
      if (t >= 0) {
        m.lse = a.lse[r];
        m.rho = c > 0.0f ? a.w[r] / c : a.w[r];   // c = 0: 0, infinite or NaN
        m.target = t;
        if (t >= a.V) m.rho = __builtin_nanf("");
      }
    }
    a.meta[r] = m;
  }
#pragma unroll
  for (int kc = 0; kc < 2; ++kc) {
    uint4 w[PARTS];
    fragment_words<PARTS>(v[kc], scale, w);
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      if (a.frag)
        *reinterpret_cast<uint4*>(a.frag + ((int64_t(r0 / 16 + wave) * PARTS + part) * (a.Kp / 32) + k0 / 32 + kc) * kBlk +
                                  lane * 8) = w[part];
      if (a.fragT) *reinterpret_cast<uint4*>(&tile[part][wave * 16 + lr][kc * 32 + 8 * lg]) = w[part];
    }
  }
  if (!a.fragT) return;                      // block-uniform
  __syncthreads();
#pragma unroll
  for (int rc = 0; rc < 2; ++rc)
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      uint16_t h[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = tile[part][rc * 32 + 8 * lg + j][wave * 16 + lr];
      *reinterpret_cast<uint4*>(a.fragT + ((int64_t(k0 / 16 + wave) * PARTS + part) * (a.np / 32) + r0 / 32 + rc) * kBlk +
                                lane * 8) = pack8(h);
    }
}

// ---------------------------------------------------------------------------
// Products: C[m][n] = sum_k A[m][k] W[n][k], both in fragment order.
// ---------------------------------------------------------------------------

// Rows of eight from fours: lanes lr of which (lr & 4) == 0 receive their own a and
// lane lr ^ 4's, the others lane lr ^ 4's b and their own.
__device__ __forceinline__ uint4 join_eight(const uint2& a, const uint2& b, int lane) {
  // from lane + 4 (a rotation by 12 of 16) in the even groups of four, from lane
  // - 4 (by 4) in the odd ones
  uint32_t x = __builtin_amdgcn_update_dpp(0u, a.x, 0x12C, 0xF, 0x5, false);
  uint32_t y = __builtin_amdgcn_update_dpp(0u, a.y, 0x12C, 0xF, 0x5, false);
  x = __builtin_amdgcn_update_dpp(x, b.x, 0x124, 0xF, 0xA, false);
  y = __builtin_amdgcn_update_dpp(y, b.y, 0x124, 0xF, 0xA, false);
  return lane & 4 ? make_uint4(x, y, b.x, b.y) : make_uint4(a.x, a.y, x, y);
}

// Division by a number that is known on the host: n / d = (mulhi(m, n) + n) >> l
// with l = ceil(log2 d), m = floor(2^32 (2^l - d) / d) + 1, for 0 <= n < 2^31.
struct Divider {
  uint32_t m, l;
  int d;
  __device__ __forceinline__ int of(int n) const {
    return static_cast<int>((__umulhi(m, static_cast<uint32_t>(n)) + static_cast<uint32_t>(n)) >> l);
  }
};

enum CeEpi { kStats = 0, kGrad = 1, kOut = 2, kPart = 3 };

struct CeMmArgs {
  const uint16_t *A, *W;
  int ta, tw;                // row tiles of 16 in A and W
  int KC;                    // chunks of 32 columns
  int ntm, ntn, splits;
  int stages;                // pairs of a row tile's: 64 columns each
  int items;
  Divider by_tiles, by_band, by_rest, by_splits;   // ntm ntn, 8 ntm, ntn % 8, splits
  const Scales* scales;      // NULL: all 1
  // kStats
  float2* part;              // [sub][part_stride]
  int part_stride, sub0;
  int tile_subs;             // parts of a row in one tile (the host's)
  float* hit;                // [rows]: the target's logit
  const int32_t* targets;
  int R, V, v0;              // rows; vocabulary rows of the piece; its first
  // kGrad
  const RowMeta* meta;
  uint16_t *G, *GT;          // [ta][parts][tw / 2], [tw][parts][ta / 2] blocks
  // kOut: C to out; kPart: fp32 accumulators, added to if `add`
  void* out;
  int M, N;                  // of out
  int is_de;                 // the scale to undo: 0 df (E), 1 dE (f)
  float4* acc;
  int add;
};

typedef __bf16 b8 __attribute__((ext_vector_type(8)));

template <int PARTS>
__device__ __forceinline__ f32x4 mma(const uint4& a, const uint4& b, f32x4 c) {
  if constexpr (PARTS == 1)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// What multiplies an accumulator of a product with G.
__device__ __forceinline__ float out_scale(const CeMmArgs& p, int parts) {
  const float c = p.scales->c;
  return parts == 1 ? c : c * (1.0f / kScaleG) * (1.0f / (p.is_de ? p.scales->f : p.scales->e));
}

template <class T>
__device__ __forceinline__ void store_out(const CeMmArgs& p, int m, int n, const f32x4& v, float s) {
  T* o = static_cast<T*>(p.out) + int64_t(m) * p.N + n;
  const float x[4] = {v[0] * s, v[1] * s, v[2] * s, v[3] * s};
  if (n + 4 <= p.N && p.N % 4 == 0) {
    store_four(o, make_float4(x[0], x[1], x[2], x[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < p.N) store_value(o + i, x[i]);
  }
}

// A 4 x 4 transpose of 16-bit values within quads of lanes: lane q (of 4) holds
// x[i] for i = 0 .. 3 (pairs p01, p23) and receives element q of lanes 0 .. 3.
__device__ __forceinline__ uint2 transpose4(uint32_t p01, uint32_t p23, int lane) {
  const uint32_t q01 = __builtin_amdgcn_mov_dpp(p01, 0xB1, 0xF, 0xF, true);   // the neighbour's
  const uint32_t q23 = __builtin_amdgcn_mov_dpp(p23, 0xB1, 0xF, 0xF, true);
  // even lanes: (own even, neighbour's even); odd: (neighbour's odd, own odd).
  // v_perm: bytes 0 - 3 come from the second operand, 4 - 7 from the first.
  const uint32_t sel = lane & 1 ? 0x03020706u : 0x05040100u;
  const uint32_t r0 = __builtin_amdgcn_perm(q01, p01, sel);
  const uint32_t r1 = __builtin_amdgcn_perm(q23, p23, sel);
  const uint32_t s = lane & 2 ? r0 : r1;
  const uint32_t t = __builtin_amdgcn_mov_dpp(s, 0x4E, 0xF, 0xF, true);       // lane ^ 2's
  return lane & 2 ? make_uint2(t, r1) : make_uint2(r0, t);
}

// Item t: its tile, and the stages [s0, s1) of its share.
struct CeItem {
  int nt, mt, split, s0, s1;
};
__device__ __forceinline__ CeItem item_at(const CeMmArgs& p, int t) {
  CeItem w;
  w.split = p.by_tiles.of(t);
  int i = t - w.split * p.by_tiles.d;
  const int band = p.by_band.of(i);                     // 8 n tiles
  i -= band * p.by_band.d;
  const bool full = 8 * band + 8 <= p.ntn;
  w.mt = full ? i >> 3 : p.by_rest.of(i);
  w.nt = 8 * band + i - w.mt * (full ? 8 : p.by_rest.d);
  w.s0 = p.by_splits.of(p.stages * w.split);
  w.s1 = p.by_splits.of(p.stages * (w.split + 1));
  return w;
}

// e^(x - top).  bf16: one rounding of x log2 e - top log2 e, 2^-24 |top| beside
// bf16's own; fp32 operands: the difference first, exact for x near top.
template <int PARTS>
__device__ __forceinline__ float shifted_exp(float x, float top) {
  return exp2_f(PARTS == 1 ? __builtin_fmaf(x, kLog2e, -kLog2e * top) : kLog2e * (x - top));
}

// What becomes of a wave's accumulators:
// acc[i][j][q] = C[16 (mt0 + j) + lr][16 (nt0 + i) + 4 lg + q].
// It reads the kernel's arguments again from where they were passed, and hides
// the lane from the compiler: what it would compute from them ahead of the main
// loop takes the loop's registers, whose spills wait for the DMAs in flight.
template <class T, int PARTS, int kEpi, int TN, int TM, int tn, int tm>
__device__ __forceinline__ void ce_epilogue(f32x4 (&acc)[tn][tm], int mt0, int nt0, int split, int wave, int lane) {
#ifdef __HIP_DEVICE_COMPILE__
  typedef const __attribute__((address_space(4))) CeMmArgs* ArgsPtr;
  uint64_t at = reinterpret_cast<uint64_t>(__builtin_amdgcn_kernarg_segment_ptr());
  asm volatile("" : "+s"(at), "+v"(lane));
  const CeMmArgs p = *reinterpret_cast<ArgsPtr>(at);
#else
  const CeMmArgs p{};
#endif
  const int lr = lane & 15, lg = lane >> 4;
  if constexpr (kEpi == kStats) {
    const float undo = PARTS == 1 ? 1.0f : (1.0f / p.scales->f) * (1.0f / p.scales->e);
    const int sub = p.sub0 + nt0 / tn;                    // tn: a wave's share of the columns
    const int left = p.V - nt0 * 16 - 4 * lg;             // this lane's columns 16 i + q below it are in the vocabulary
    // No branch inside: results wait in registers until the end, and the tile
    // that the vocabulary ends in has code of its own.
    float tops[tm], sums[tm];
    int targets[tm];
#pragma unroll
    for (int j = 0; j < tm; ++j) targets[j] = p.targets[min((mt0 + j) * 16 + lr, p.R - 1)] - p.v0 - nt0 * 16 - 4 * lg;
    auto rows = [&](auto whole) {
#pragma unroll
      for (int j = 0; j < tm; ++j) {
        __builtin_amdgcn_sched_barrier(0);  // one column of tiles at a time: the accumulators fill half of the registers
        int l = left;
        if constexpr (!decltype(whole)::value) asm volatile("" : "+v"(l));   // the comparisons are not kept from j to j
        float top = kLowest, x[tn][4];
#pragma unroll
        for (int i = 0; i < tn; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            x[i][q] = acc[i][j][q] * undo;
            if constexpr (!decltype(whole)::value) x[i][q] = 16 * i + q < l ? x[i][q] : -__builtin_inff();
            top = fmaxf(top, x[i][q]);
          }
        top = group4_max(top);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < tn; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) sum += shifted_exp<PARTS>(x[i][q], top);
        tops[j] = top, sums[j] = group4_sum(sum);
      }
    };
    if (p.V - nt0 * 16 >= 16 * tn)                        // wave-uniform
      rows(std::true_type{});
    else
      rows(std::false_type{});
#pragma unroll
    for (int j = 0; j < tm; ++j) {
      const int m = (mt0 + j) * 16 + lr, t = targets[j];
      const bool in = m < p.R && t >= 0 && t < 16 * tn && t < left && (t & 15) < 4;
      if (__any(in)) {                                    // few tiles of a large vocabulary hold a row's target
        float hit = 0.0f;
#pragma unroll
        for (int i = 0; i < tn; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) hit = t == 16 * i + q ? acc[i][j][q] : hit;
        if (in) p.hit[m] = hit * undo;
      }
      if (m < p.R && lg == 0) p.part[int64_t(sub) * p.part_stride + m] = make_float2(tops[j], sums[j]);
    }
  } else if constexpr (kEpi == kGrad) {
    const float undo = PARTS == 1 ? 1.0f : (1.0f / p.scales->f) * (1.0f / p.scales->e);
    const int GC = p.tw / 2, TC = p.ta / 2;               // chunks of 32 in G's and GT's rows
    const int left = p.V - nt0 * 16 - 4 * lg;             // this lane's columns 16 i + q below it are in the vocabulary
    const bool whole = p.V - nt0 * 16 >= 16 * tn;         // wave-uniform
    static_assert(tm % 2 == 0 && tn % 2 == 0, "tiles are stored in pairs, a block of 32 columns each way");
    RowMeta meta[tm];
#pragma unroll
    for (int j = 0; j < tm; ++j) meta[j] = p.meta[min((mt0 + j) * 16, (p.ta - 1) * 16) + lr];
    // They arrive here: a load that is still out on some path makes the
    // compiler wait for everything, DMAs too, where its register is used next.
#pragma unroll
    for (int j = 0; j < tm; ++j) asm volatile("" : "+v"(meta[j].lse), "+v"(meta[j].rho), "+v"(meta[j].target));
    // Column tiles i, i + 1 of row tiles j, j + 1 (an even number of either):
    // g of all four, then two blocks of G and two of G^T.
    auto quad = [&](auto has_target, int j, int i) {
      uint32_t x[2][2][PARTS][2];                         // [row tile][column tile][part][pairs of columns]
#pragma unroll
      for (int jj = 0; jj < 2; ++jj)
#pragma unroll
        for (int ii = 0; ii < 2; ++ii) {
          const float lse = meta[j + jj].lse, rho = meta[j + jj].rho;
          const int target = meta[j + jj].target - p.v0 - nt0 * 16 - 4 * lg;
          float g[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float e = shifted_exp<PARTS>(acc[i + ii][j + jj][q] * undo, lse);
            if constexpr (decltype(has_target)::value) e = target == 16 * (i + ii) + q ? e - 1.0f : e;
            g[q] = rho * e;
          }
          if (!whole) {
#pragma unroll
            for (int q = 0; q < 4; ++q) g[q] = 16 * (i + ii) + q < left ? g[q] : 0.0f;
          }
          if constexpr (PARTS == 1) {
            x[jj][ii][0][0] = bf16_pair(g[0], g[1]), x[jj][ii][0][1] = bf16_pair(g[2], g[3]);
          } else {
            uint16_t hi[4], lo[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) split_rn(g[q] * kScaleG, hi[q], lo[q]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              x[jj][ii][0][h] = hi[2 * h] | uint32_t(hi[2 * h + 1]) << 16;
              x[jj][ii][PARTS - 1][h] = lo[2 * h] | uint32_t(lo[2 * h + 1]) << 16;
            }
          }
        }
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
#pragma unroll
        for (int jj = 0; jj < 2; ++jj) {
          // G: a lane has columns 4 lg .. + 3 of two tiles; with the neighbouring
          // group's (rows of 16 lanes trade places) it has 8 of one: the block's
          // word of lane (lr, 2 (lg & 1) + lg / 2).
          const auto s0 = __builtin_amdgcn_permlane16_swap(x[jj][0][part][0], x[jj][1][part][0], false, false);
          const auto s1 = __builtin_amdgcn_permlane16_swap(x[jj][0][part][1], x[jj][1][part][1], false, false);
          uint16_t* G = p.G + ((int64_t(mt0 + j + jj) * PARTS + part) * GC + (nt0 + i) / 2) * kBlk +
                        (16 * (2 * (lg & 1) + (lg >> 1)) + lr) * 8;
          *reinterpret_cast<uint4*>(G) = make_uint4(s0[0], s1[0], s0[1], s1[1]);
        }
#pragma unroll
        for (int ii = 0; ii < 2; ++ii) {
          // G^T: transposed, a lane has rows 4 (lr / 4) .. + 3 of column 4 lg +
          // lr % 4 of two row tiles; with those of lane lr ^ 4 it has 8 of one.
          const uint2 t0 = transpose4(x[0][ii][part][0], x[0][ii][part][1], lane);
          const uint2 t1 = transpose4(x[1][ii][part][0], x[1][ii][part][1], lane);
          const uint4 t = join_eight(t0, t1, lane);
          uint16_t* GT = p.GT + ((int64_t(nt0 + i + ii) * PARTS + part) * TC + (mt0 + j) / 2) * kBlk +
                         (16 * (2 * ((lr >> 2) & 1) + (lr >> 3)) + 4 * lg + (lr & 3)) * 8;
          *reinterpret_cast<uint4*>(GT) = t;
        }
      }
    };
#pragma unroll
    for (int j = 0; j < tm; j += 2) {
      if (mt0 + j >= p.ta) continue;                      // wave-uniform; the tiles come in fours
      const int t0 = meta[j].target - p.v0 - nt0 * 16, t1 = meta[j + 1].target - p.v0 - nt0 * 16;
      const bool hit = (t0 >= 0 && t0 < 16 * tn) || (t1 >= 0 && t1 < 16 * tn);
      if (__any(hit)) {                                   // few tiles of a large vocabulary
#pragma unroll
        for (int i = 0; i < tn; i += 2)
          if (nt0 + i < p.tw) quad(std::true_type{}, j, i);
      } else {
#pragma unroll
        for (int i = 0; i < tn; i += 2)
          if (nt0 + i < p.tw) quad(std::false_type{}, j, i);
      }
    }
  } else if constexpr (kEpi == kOut) {
    float s = out_scale(p, PARTS);
    asm volatile("" : "+v"(s));                           // arrived, as above
#pragma unroll
    for (int i = 0; i < tn; ++i)
#pragma unroll
      for (int j = 0; j < tm; ++j) {
        __builtin_amdgcn_sched_barrier(0);
        const int m = (mt0 + j) * 16 + lr, n = (nt0 + i) * 16 + 4 * lg;
        if (m < p.M && n < p.N) store_out<T>(p, m, n, acc[i][j], s);
      }
  } else {
    // [split][m tile][n tile][TN][TM][lane], however many waves share it
    float4* a = p.acc + ((int64_t(split) * p.ntm + mt0 / TM) * p.ntn + nt0 / TN) * (TN * TM * 64) +
                ((nt0 % TN) * TM + mt0 % TM) * 64 + lane;
#pragma unroll
    for (int i = 0; i < tn; ++i) {
      __builtin_amdgcn_sched_barrier(0);    // a row's loads at a time
      float4 o[tm];
#pragma unroll
      for (int j = 0; j < tm; ++j) o[j] = p.add ? a[(i * TM + j) * 64] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int j = 0; j < tm; ++j)
        a[(i * TM + j) * 64] = make_float4(o[j].x + acc[i][j][0], o[j].y + acc[i][j][1], o[j].z + acc[i][j][2],
                                           o[j].w + acc[i][j][3]);
    }
  }
}

// Blocks of 4 waves work through items: a tile, or one of `splits` shares of a
// tile's columns.  Each XCD (blocks go round-robin) works through a contiguous
// range of items, 8 n tiles wide at a time, so that the tiles in flight share
// operands in its L2.  Tiles (rows of A x rows of W; 4 waves share it WN ways over
// the rows of W):
//   bf16, products with G   256 x 256, 128 x 128 a wave, one wave on each SIMD.
//     8 waves of 128 x 64 would move 256 KiB through the LDS for 64 columns (192
//     read, 64 written by DMA), 2,048 clocks, as long as their MFMAs take;
//     128 x 128 a wave moves 192 KiB.
//   bf16, logits            256 x 128, 64 x 128 a wave, two blocks a compute unit:
//     what becomes of a tile (exponentials, stores) runs beside the other block's
//     MFMAs.
//   split                   256 x 128, one block a compute unit (three products
//     for twice the bytes).
//   few tiles               128 x 128.
// A stage is one chunk of 32 columns (of both parts).  One or two waves a SIMD
// have little to hide behind, so everything is ahead of time: a stage's DMA is
// issued as many stages before as there are LDS buffers, its fragments are read
// into registers under the MFMAs of the stage before (the second of two register
// sets; stages come in pairs), and both are dealt out between the MFMAs.  A stage
// has no branch: while an item's last stages run, the next item's first are fetched
// (behind the last item its own first again, which nobody reads).  An item has
// four stages at least: every matrix is padded to 128 columns.
//
// Measured, bf16, 8,192 rows, a piece of 16,384 of the vocabulary, width 1,024 (275
// GFLOP each): logits with their statistics 230 us (1.2 PF/s, where a library product
// of 16,384^3 reaches 1.36), logits with G 328 (537 MB of stores beside them), df
// 242, dE 230 (1.2 PF/s).  fp32, 16,320 rows, vocabulary 256, width 512 (4.3 GFLOP,
// 12.8 executed): logits 17.5 us, with G 22, df 24.5, dE 19: half of each is the
// reading and writing of its operands.
template <class T, int PARTS, int kEpi, int TN, int TM, int WN, int kBufs, int kPerEu>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kPerEu, kPerEu))) void k_ce_mm(CeMmArgs p) {
  constexpr int WM = 4 / WN, tn = TN / WN, tm = TM / WM;
  constexpr int FW = PARTS * TN / 4, FA = PARTS * TM / 4, DPW = FW + FA;   // blocks of W and of A that a wave fetches
  constexpr int BUF = PARTS * (TN + TM) * kBlk;         // one stage, in halves
  constexpr int kFrags = PARTS * (tn + tm);
  constexpr int kPasses = PARTS == 1 ? 1 : 3;           // products of parts
  // Stores of a whole tile's epilogue that the first two stages of the next item
  // need not wait for: they are younger than what those need.
  constexpr int kAll = kEpi == kGrad ? PARTS * tn * tm : 0;
  constexpr int kStores = (kBufs - 2) * DPW + kAll < 64 ? kAll : 0;        // the counter has six bits
  extern __shared__ __attribute__((aligned(16))) unsigned char ce_lds[];
  uint16_t* const lds = reinterpret_cast<uint16_t*>(ce_lds);
  const int per_xcd = (p.items + kXcd - 1) / kXcd;
  const int first = (blockIdx.x % kXcd) * per_xcd;
  const int last = min(first + per_xcd, p.items);
  const int stride = gridDim.x / kXcd;
  int item = first + blockIdx.x / kXcd;
  if (item >= last) return;                             // block-uniform
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int wn = wave % WN, wm = wave / WN;
  i32x4 rw, ra;
  uint32_t soff[DPW];                                   // scalars: no vector registers are to spare
  const uint32_t voff = lane * 16;
  const uint32_t dw = lds_address(lds + wave * FW * kBlk), da = lds_address(lds + (PARTS * TN + wave * FA) * kBlk);
  auto aim = [&](const CeItem& w) {
    // Row tiles past the matrix repeat its last: nothing of theirs is used.
    const int hw = min(TN, p.tw - w.nt * TN), ha = min(TM, p.ta - w.mt * TM);
    const int row = PARTS * p.KC;                       // blocks of a row tile
    rw = buffer_words(p.W + int64_t(w.nt) * TN * row * kBlk, static_cast<uint32_t>(hw) * row * (kBlk * 2));
    ra = buffer_words(p.A + int64_t(w.mt) * TM * row * kBlk, static_cast<uint32_t>(ha) * row * (kBlk * 2));
#pragma unroll
    for (int i = 0; i < DPW; ++i) {
      const int b = i < FW ? wave * FW + i : wave * FA + i - FW;           // [tile][part]
      const int tile = min(b / PARTS, (i < FW ? hw : ha) - 1);
      soff[i] = static_cast<uint32_t>(tile * row + (b % PARTS) * p.KC + 2 * w.s0) * (kBlk * 2);
    }
  };
  auto fetch = [&](int i, int buf) {
    if (i < FW)
      dma16(rw, voff, soff[i], dw + static_cast<uint32_t>((buf * BUF + i * kBlk) * 2));
    else
      dma16(ra, voff, soff[i], da + static_cast<uint32_t>((buf * BUF + (i - FW) * kBlk) * 2));
    soff[i] += kBlk * 2;
  };
  const uint16_t* const wl = lds + wn * tn * PARTS * kBlk + lane * 8;
  const uint16_t* const al = lds + (TN + wm * tm) * PARTS * kBlk + lane * 8;
  uint4 fw[2][tn * PARTS], fa[2][tm * PARTS];           // [set][tile, part]
  auto read = [&](int set, int buf, int k) {            // fragment k: A's first, all of which the first MFMAs need
    if (k < tm * PARTS)
      fa[set][k] = *reinterpret_cast<const uint4*>(al + buf * BUF + k * kBlk);
    else
      fw[set][k - tm * PARTS] = *reinterpret_cast<const uint4*>(wl + buf * BUF + (k - tm * PARTS) * kBlk);
  };
  CeItem w = item_at(p, item);
  aim(w);
#pragma unroll
  for (int s = 0; s < kBufs; ++s)
#pragma unroll
    for (int i = 0; i < DPW; ++i) fetch(i, s);
  wait_vmem();
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kFrags; ++k) read(0, 0, k);
  int buf = 0;
  bool stored = false;
  for (;;) {
    f32x4 acc[tn][tm];
#pragma unroll
    for (int i = 0; i < tn; ++i)
#pragma unroll
      for (int j = 0; j < tm; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto stage = [&](auto set, bool after_stores) {
      constexpr int half = decltype(set)::value;
      // The next stage has landed (those behind it may be out, and at the start
      // of an item the stores of the one before), and every wave holds this
      // one's fragments, so its buffer is free.
      if (kStores > 0 && after_stores)
        wait_vmem_but<(kBufs - 2) * DPW + kStores>();
      else
        wait_vmem_but<(kBufs - 2) * DPW>();
      __syncthreads();
      const int here = buf, next = buf == kBufs - 1 ? 0 : buf + 1;
      // Groups of four MFMAs, all but the last ones (LDS reads take time) with
      // their share of the DMAs and of the next stage's fragments.
      constexpr int kGroups = kPasses * tn * tm / 4, kLoaded = kGroups - kGroups / 4;
      static_assert(tm % 4 == 0, "a group is within one row of tiles");
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = DPW * g / kLoaded; d < DPW * (g + 1) / kLoaded && d < DPW; ++d) fetch(d, here);
#pragma unroll
        for (int k = kFrags * g / kLoaded; k < kFrags * (g + 1) / kLoaded && k < kFrags; ++k) read(half ^ 1, next, k);
        // lo hi, hi lo, hi hi over a row of tiles
        const int i = g * 4 / (kPasses * tm), pass = g * 4 / tm % kPasses;
        const int pw = PARTS == 2 && pass == 0 ? 1 : 0, pa = PARTS == 2 && pass == 1 ? 1 : 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int j = g * 4 % tm + q;
          acc[i][j] = mma<PARTS>(fw[half][i * PARTS + pw], fa[half][j * PARTS + pa], acc[i][j]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      buf = next;
    };
    constexpr std::integral_constant<int, 0> even;
    constexpr std::integral_constant<int, 1> odd;
    for (int c = w.s0; c < w.s1 - 2; ++c) {
      stage(even, stored);
      stage(odd, stored);
      stored = false;
    }
    const int mt0 = w.mt * TM + wm * tm, nt0 = w.nt * TN + wn * tn, split = w.split;
    item += stride;
    const bool more = item < last;                      // block-uniform
    if (more) w = item_at(p, item);
    static_assert(kBufs == 3 || kBufs == 4, "the last kBufs stages fetch from the next item");
    if constexpr (kBufs == 4) aim(w);
    stage(even, false);
    if constexpr (kBufs == 3) aim(w);
    stage(odd, false);
    stage(even, false);
    stage(odd, false);
    ce_epilogue<T, PARTS, kEpi, TN, TM, tn, tm>(acc, mt0, nt0, split, wave, lane);
    stored = mt0 + tm <= p.ta && nt0 + tn <= p.tw;      // every store was issued
    if (!more) break;
  }
  wait_vmem();                                          // the last fetches, before the LDS is another block's
}

// The shares of kPart's accumulators summed in order, to the result.  Bound by
// memory; 5 us for few, 15 for 34 MB of sums.
template <class T, int PARTS, int TN, int TM>
__global__ __launch_bounds__(256) void k_ce_sum(CeMmArgs p) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int tile = blockIdx.x, mt = tile / p.ntn, nt = tile % p.ntn;
  const int part = blockIdx.y * 4 + wave, i = part / TM, j = part % TM;
  const int m = (mt * TM + j) * 16 + lr, n = (nt * TN + i) * 16 + 4 * lg;
  if (m >= p.M || n >= p.N) return;
  const float4* a = p.acc + int64_t(tile) * (TN * TM * 64) + part * 64 + lane;
  const int64_t step = int64_t(p.ntm) * p.ntn * (TN * TM * 64);
  f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < p.splits; ++s) {
    const float4 x = a[s * step];
    v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
  }
  store_out<T>(p, m, n, v, out_scale(p, PARTS));
}

// ---------------------------------------------------------------------------
// The loss of a few rows: E is read once (twice, rows_of) and is all there is to
// read.  A wave takes 16 vocabulary rows at a time straight from E into MFMA
// operands (lane (lr, lg): row lr, 8 or 4 consecutive columns), the rows of f, RT
// tiles of 16, wait in LDS; a lane keeps the running maximum and sum of its
// logits.  fp32 uses the fp32 matrix instruction.  A head of 50,257 x 1,024 in bf16, 103 MB: 21.3 us
// (4.8 TB/s), and 4 for the join.
// ---------------------------------------------------------------------------
struct RowsArgs {
  const void *f, *E;
  int64_t f_stride, e_stride;
  const int32_t* targets;
  int R, V, K;
  float2* part;             // [gridDim.x][part_stride]
  int part_stride, part_rows;   // the rows of this pass that have a place in it
  float* hit;
};

constexpr int kRowsWaves = 16;

template <class T, int RT>
__global__ __launch_bounds__(64 * kRowsWaves) void k_ce_rows(RowsArgs a) {
  constexpr bool kB = sizeof(T) == 2;
  constexpr int kW = 16 / sizeof(T);                    // columns of a lane's 16 bytes
  constexpr int kChunk = 4 * kW;                        // columns of one step
  extern __shared__ __attribute__((aligned(16))) unsigned char ce_lds[];
  T* const fl = reinterpret_cast<T*>(ce_lds);           // [chunk][row tile][lane][kW]
  __shared__ float2 red[kRowsWaves][16 * RT];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int chunks = (a.K + kChunk - 1) / kChunk;
  const T* f = static_cast<const T*>(a.f);
  const int full = a.K / kChunk;                        // chunks without a tail
  const T* E = static_cast<const T*>(a.E);
  // The block's tiles: a contiguous share, so that every compute unit gets the
  // same number but for one.
  const int tiles = (a.V + 15) / 16;
  const int last = static_cast<int>(int64_t(tiles) * (blockIdx.x + 1) / gridDim.x);
  int t = static_cast<int>(int64_t(tiles) * blockIdx.x / gridDim.x) + wave;
  // rows past the end repeat the last and are masked below
  auto row_of = [&](int tile) { return E + min(tile * 16 + lr, a.V - 1) * a.e_stride + lg * kW; };
  // Two batches of eight loads (four, where accumulators need the registers): one is
  // multiplied while the other is on its way, the next tile's first behind the last
  // of this one, the first of all before f is brought to LDS.
  constexpr int U = RT == 1 ? 8 : 4;
  auto load = [&](uint4 (&x)[U], const T* e, int c) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c + u < full) x[u] = load_any<uint4>(e + (c + u) * kChunk);
  };
  uint4 x0[U], x1[U];
  const T* e = row_of(t);
  if (t < last) load(x0, e, 0);
  bool on[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) on[i] = 16 * i + lr < a.R && a.targets[16 * i + lr] >= 0;
  for (int c = wave; c < chunks; c += kRowsWaves) {
    const int k = c * kChunk + lg * kW;
    uint4 y[RT];
    if (c < full) {
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        y[i] = make_uint4(0, 0, 0, 0);
        if (on[i]) y[i] = load_any<uint4>(f + (16 * i + lr) * a.f_stride + k);
      }
    } else {
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        T one[kW] = {};
#pragma unroll
        for (int j = 0; j < kW; ++j)
          if (on[i] && k + j < a.K) one[j] = f[(16 * i + lr) * a.f_stride + k + j];
        __builtin_memcpy(&y[i], one, 16);
      }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) *reinterpret_cast<uint4*>(fl + ((c * RT + i) * 64 + lane) * kW) = y[i];
  }
  __syncthreads();
  int target[RT];
  float top[RT], sum[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
    target[i] = 16 * i + lr < a.R ? a.targets[16 * i + lr] : -1, top[i] = kLowest, sum[i] = 0.0f;
  for (; t < last; t += kRowsWaves) {
    f32x4 acc[RT], acc2{0.f, 0.f, 0.f, 0.f};            // acc2: one tile alone takes turns
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto step = [&](const uint4& x, int c, bool odd) {
      uint4 y[RT];
#pragma unroll
      for (int i = 0; i < RT; ++i) y[i] = *reinterpret_cast<const uint4*>(fl + ((c * RT + i) * 64 + lane) * kW);
      if constexpr (kB) {
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          f32x4& to = RT == 1 && odd ? acc2 : acc[i];
          to = mma<1>(x, y[i], to);
        }
      } else {
        const f32x4 xf = __builtin_bit_cast(f32x4, x);
#pragma unroll
        for (int j = 0; j < 4; ++j)                     // tile by tile: one's next product would wait for its last
#pragma unroll
          for (int i = 0; i < RT; ++i) {
            f32x4& to = RT == 1 && odd ? acc2 : acc[i];
            to = __builtin_amdgcn_mfma_f32_16x16x4f32(xf[j], __builtin_bit_cast(f32x4, y[i])[j], to, 0, 0, 0);
          }
      }
    };
    const T* ahead = row_of(t + kRowsWaves);
    for (int c = 0; c < full; c += 2 * U) {
      load(x1, e, c + U);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c + u < full) step(x0[u], c + u, u & 1);
      if (c + 2 * U < full)
        load(x0, e, c + 2 * U);
      else if (t + kRowsWaves < last)
        load(x0, ahead, 0);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c + U + u < full) step(x1[u], c + U + u, u & 1);
    }
    int c = full;
    if (c < chunks) {                                   // the tail, column by column
      T tail[kW];
#pragma unroll
      for (int j = 0; j < kW; ++j) {
        T z{};
        tail[j] = c * kChunk + lg * kW + j < a.K ? e[c * kChunk + j] : z;
      }
      uint4 x;
      __builtin_memcpy(&x, tail, 16);
      step(x, c, false);
    }
    e = ahead;
    // acc[i][q] = logit of row 16 i + lr, vocabulary row 16 t + 4 lg + q
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float l[4], most = top[i];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int v = t * 16 + 4 * lg + q;
        l[q] = v < a.V ? (RT == 1 ? acc[i][q] + acc2[q] : acc[i][q]) : -__builtin_inff();
        most = fmaxf(most, l[q]);
        if (v == target[i] && v < a.V) a.hit[16 * i + lr] = l[q];
      }
      sum[i] *= exp2_f(kLog2e * (top[i] - most));
#pragma unroll
      for (int q = 0; q < 4; ++q) sum[i] += exp2_f(kLog2e * (l[q] - most));
      top[i] = most;
    }
  }
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const float all = group4_max(top[i]);
    const float of_all = group4_sum(sum[i] * exp2_f(kLog2e * (top[i] - all)));
    if (lg == 0) red[wave][16 * i + lr] = make_float2(all, of_all);
  }
  __syncthreads();
  const int r = threadIdx.x;
  if (r < 16 * RT && r < a.part_rows) {
    float m = kLowest, s = 0.0f;
    for (int w = 0; w < kRowsWaves; ++w) m = fmaxf(m, red[w][r].x);
    for (int w = 0; w < kRowsWaves; ++w) s += red[w][r].y * exp2_f(kLog2e * (red[w][r].x - m));
    a.part[int64_t(blockIdx.x) * a.part_stride + r] = make_float2(m, s);
  }
}

// ---------------------------------------------------------------------------
// The parts of every row joined, 16 rows a block: lse and loss.  Latency of a few
// loads: 4 us; 7 for 8,192 rows of 393 parts.
// ---------------------------------------------------------------------------
template <int kParts>
__global__ __launch_bounds__(16 * kParts) void k_ce_join(const float2* part, int subs, int stride, const int32_t* targets,
                                                 const float* hit, int R, int V, float* loss, float* lse) {
  __shared__ float2 red[kParts][17];
  const int lr = threadIdx.x & 15, w = threadIdx.x >> 4, r = blockIdx.x * 16 + lr;
  float top = kLowest, sum = 0.0f;
  if (r < R)
#pragma unroll 4
    for (int s = w; s < subs; s += kParts) {
      const float2 x = part[int64_t(s) * stride + r];
      const float m = fmaxf(top, x.x);
      sum = sum * exp2_f(kLog2e * (top - m)) + x.y * exp2_f(kLog2e * (x.x - m));
      top = m;
    }
  red[w][lr] = make_float2(top, sum);
  __syncthreads();
  // The first half of the parts takes the other's in, and so on.
  for (int h = kParts / 2; h >= 8; h /= 2) {
    if (w < h) {
      const float2 x = red[w][lr], y = red[w + h][lr];
      const float m = fmaxf(x.x, y.x);
      red[w][lr] = make_float2(m, x.y * exp2_f(kLog2e * (x.x - m)) + y.y * exp2_f(kLog2e * (y.x - m)));
    }
    __syncthreads();
  }
  if (w != 0 || r >= R) return;
  float m = kLowest, s = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, red[i][lr].x);
#pragma unroll
  for (int i = 0; i < 8; ++i) s += red[i][lr].y * exp2_f(kLog2e * (red[i][lr].x - m));
  const int t = targets[r];
  float l = 0.0f, out = 0.0f;
  if (t >= 0) {
    l = m + kLog2 * __builtin_amdgcn_logf(s);
    out = t < V ? (m - hit[r]) + kLog2 * __builtin_amdgcn_logf(s) : __builtin_nanf("");
  }
  if (lse) lse[r] = l;
  if (loss) loss[r] = out;
}

__global__ __launch_bounds__(256) void k_ce_zero(uint16_t* x, int64_t halves) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < halves; i += int64_t(gridDim.x) * 256) x[i] = 0;
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
constexpr int64_t kFill = 256;            // tiles that fill the card
constexpr int kRowsBlocks = 256;          // blocks of k_ce_rows
constexpr size_t kRowsLds = 147456;       // f's rows in LDS, beside 8 KiB of the waves' results
constexpr int64_t kTwiceBytes = 1 << 24;  // of a head that k_ce_rows reads twice
constexpr int kRowsMost = 128;            // rows that k_ce_rows takes at most: two passes of 64

int64_t up(int64_t x, int64_t q) { return (x + q - 1) / q * q; }

struct Sizes {
  int64_t Rp, Kp, Vp;                     // padded to 128; Vp of the largest piece
  int parts;
  size_t part, hit, maxima, scales, meta, f, fT, e, eT, G, GT, accf, acce, total;
};

// Accumulators of a product of m x n outputs whose columns are shared out: at
// most max(tiles, 2 kFill) tiles (choose_splits), of whichever size.
size_t acc_bytes(int64_t m, int64_t n, int64_t columns) {
  int64_t most = 0;
  for (int tm : {8, 16})
    for (int tn : {8, 16}) {
      const int64_t tiles = up(m, 16 * tm) / (16 * tm) * (up(n, 16 * tn) / (16 * tn));
      most = std::max(most, std::max(tiles, std::min(tiles * (columns / 128), 2 * kFill)) * tm * tn * 256);
    }
  return size_t(most) * 4;
}

int piece_of(const soma_ce_config& c) { return c.rows <= kLongRows ? kLongPiece : kPiece; }

// Every part grows with the rows, also where the piece gets shorter, so that a
// workspace for many rows holds a call of fewer.
Sizes sizes_of(const soma_ce_config& c, bool grad) {
  Sizes s{};
  s.Rp = up(c.rows, 128);
  s.Kp = up(c.width, 128);
  s.Vp = up(std::min<int64_t>(c.vocab, piece_of(c)), 128);
  s.parts = c.type == SOMA_FLOAT ? 2 : 1;
  const int64_t longest = up(std::min<int64_t>(c.vocab, kLongPiece), 128);
  const int64_t area = std::max(s.Rp * s.Vp, std::min<int64_t>(s.Rp, kLongRows) * longest);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += up256(bytes);
    return o;
  };
  const size_t half = size_t(s.parts) * 2;
  if (!grad) {
    s.part = take(std::max(size_t(up(c.vocab, 64) / 64 + 4 * (c.vocab / kPiece + 1)) * s.Rp, size_t(kRowsBlocks) * std::min<int64_t>(up(c.rows, 16), kRowsMost)) * 8);
    s.hit = take(size_t(s.Rp) * 4);
  } else {
    s.meta = take(size_t(s.Rp) * sizeof(RowMeta));
  }
  s.maxima = take(3 * kMaxima * 4);
  s.scales = take(sizeof(Scales));
  s.f = take(size_t(s.Rp) * s.Kp * half);
  s.e = take(size_t(longest) * s.Kp * half);
  if (grad) {
    s.fT = take(size_t(s.Rp) * s.Kp * half);
    s.eT = take(size_t(longest) * s.Kp * half);
    s.G = take(size_t(area) * half);
    s.GT = take(size_t(area) * half);
    s.accf = take(acc_bytes(s.Rp, s.Kp, longest));
    s.acce = take(acc_bytes(longest, s.Kp, s.Rp));
  }
  s.total = at;
  return s;
}

int check_ce(const soma_ce_config* c) {
  if (!c) return set_error(SOMA_EINVAL, "cfg is NULL");
  if (!is_type(c->type)) return set_error(SOMA_EINVAL, "unknown type %d", c->type);
  // a row tile of G^T is addressed in 32 bits
  if (c->rows < 0 || c->rows > (1 << 20)) return set_error(SOMA_ESHAPE, "rows must be in [0, 2^20]");
  if (c->vocab < 1 || c->vocab > (1 << 24)) return set_error(SOMA_ESHAPE, "vocab must be in [1, 2^24]");
  if (c->width < 1 || c->width > (1 << 16)) return set_error(SOMA_ESHAPE, "width must be in [1, 2^16]");
  if (c->f_stride < c->width || c->e_stride < c->width || c->f_stride > (int64_t(1) << 32) ||
      c->e_stride > (int64_t(1) << 32))
    return set_error(SOMA_ESHAPE, "f_stride and e_stride must be at least width");
  return SOMA_OK;
}

// Shares of every tile's columns: as many as bring the items to `fill`, at
// least two pairs of stages each.
int choose_splits(int64_t tiles, int64_t stages, int64_t fill) {
  return int(std::max<int64_t>(1, std::min(fill / std::max<int64_t>(tiles, 1), stages / 2)));
}

Divider divider(int d) {
  uint32_t l = 0;
  while ((int64_t(1) << l) < d) ++l;
  return {uint32_t((uint64_t(1) << 32) * ((uint64_t(1) << l) - uint64_t(d)) / uint64_t(d)) + 1u, l, d};
}

// most: blocks that the card holds at once.
int launch_items(void (*kernel)(CeMmArgs), CeMmArgs& p, int64_t most, unsigned lds, hipStream_t st) {
  const int64_t items = int64_t(p.ntm) * p.ntn * p.splits;
  if (items >= (int64_t(1) << 30)) return set_error(SOMA_ESHAPE, "too many tiles in one launch");
  p.items = int(items);
  p.by_tiles = divider(p.ntm * p.ntn), p.by_band = divider(8 * p.ntm), p.by_rest = divider(std::max(p.ntn % 8, 1));
  p.by_splits = divider(p.splits);
  const int64_t blocks = std::min(up(items, kXcd), most);
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
  if (e != hipSuccess) return device_error("hipFuncSetAttribute", e);
  return launch("k_ce_mm", kernel, dim3(unsigned(blocks)), dim3(256), lds, st, p);
}

// Tiles in units of 16 rows of A and of W.
struct Tile {
  int tm, tn;
};
Tile tile_of(bool large, int parts, bool logits) {
  if (!large) return {8, 8};
  return {16, parts == 1 && !logits ? 16 : 8};
}

template <class T, int PARTS, int kEpi>
int launch_mm(CeMmArgs& p, bool large, hipStream_t st) {
  constexpr bool kLogits = kEpi == kStats || kEpi == kGrad;
  const Tile t = tile_of(large, PARTS, kLogits);
  p.stages = p.KC / 2;
  p.ntm = (p.ta + t.tm - 1) / t.tm;
  p.ntn = (p.tw + t.tn - 1) / t.tn;
  p.tile_subs = large ? 1 : 2;
  if constexpr (PARTS == 1) {
    if (!large)
      return launch_items(k_ce_mm<T, 1, kEpi, 8, 8, 2, 4, 2>, p, 2 * kFill, 65536, st);
    if constexpr (kLogits)
      return launch_items(k_ce_mm<T, 1, kEpi, 8, 16, 1, 3, 2>, p, 2 * kFill, 73728, st);
    else
      return launch_items(k_ce_mm<T, 1, kEpi, 16, 16, 2, 4, 1>, p, kFill, 131072, st);
  } else {
    if (!large)
      return launch_items(k_ce_mm<T, 2, kEpi, 8, 8, 2, 4, 1>, p, kFill, 131072, st);
    return launch_items(k_ce_mm<T, 2, kEpi, 8, 16, 1, 3, 1>, p, kFill, 147456, st);
  }
}

int64_t tiles_of(int64_t m, int64_t n, Tile t) { return (m + 16 * t.tm - 1) / (16 * t.tm) * ((n + 16 * t.tn - 1) / (16 * t.tn)); }

// Microseconds of a product of m x n outputs over `columns` in `splits` shares,
// from what the card reaches on many tiles (executed products: 1.1 PF/s on large
// tiles, 0.9 on small ones) and the rounds that the items take, and from what
// the sums of shares, or of pieces (`sums`), write and read at 5 TB/s.  It decides
// between tiles and shares only.  Measured: fp32 logits 1,000 x 10,007 x 361, 316
// large tiles in two rounds, 37.8 us, 632 small ones in three, 31; df 16,320 x
// 512 over 256 columns, two shares of large tiles and their sum, 45 us, whole small
// tiles 24.
double product_us(int64_t m, int64_t n, int64_t columns, int parts, bool logits, bool large, int splits, bool sums) {
  const Tile t = tile_of(large, parts, logits);
  const int64_t hold = parts == 1 && (logits || !large) ? 2 * kFill : kFill;
  const int64_t items = tiles_of(m, n, t) * splits, rounds = (items + hold - 1) / hold;
  const double item = 2.0 * (parts == 1 ? 1 : 3) * t.tm * t.tn * 256.0 * double(columns) / splits;
  return double(rounds) * double(hold) * item / (large ? 1.1e9 : 0.9e9) +
         (sums || splits > 1 ? 8.0 * double(splits) * double(m) * double(n) / 5e6 : 0.0) + (splits > 1 ? 5.0 : 0.0);
}

bool large_logits(int64_t m, int64_t n, int64_t columns, int parts) {
  return product_us(m, n, columns, parts, true, true, 1, false) < product_us(m, n, columns, parts, true, false, 1, false);
}

// How the products with G are shared out, by the first and largest piece:
// whole tiles, or as many shares as fill the card, of either size.
struct Shares {
  bool large;
  int splits;
};
Shares shares_of(int64_t m, int64_t n, int64_t columns, int parts, bool sums) {
  Shares best{};
  double least = 0.0;
  for (const bool large : {true, false}) {
    const int most = choose_splits(tiles_of(m, n, tile_of(large, parts, false)), columns / 64, large || parts == 2 ? kFill : 2 * kFill);
    for (int s = 1;; s = most) {
      const double us = product_us(m, n, columns, parts, false, large, s, sums);
      if (best.splits == 0 || us < least) best = {large, s}, least = us;
      if (s == most) break;
    }
  }
  return best;
}

// One product with G.  `single`: it alone gives the result; else the result
// is the sum of several calls (`add` from the second on), which the one with
// `finish` brings to the output.
template <class T, int PARTS>
int launch_product(CeMmArgs p, const Shares& sh, bool single, bool finish, hipStream_t st) {
  p.splits = sh.splits;
  if (single && p.splits == 1) return launch_mm<T, PARTS, kOut>(p, sh.large, st);
  // A last piece of fewer columns than shares need adds to the first ones only.
  p.splits = std::max(1, std::min(sh.splits, p.KC / 4));
  if (int rc = launch_mm<T, PARTS, kPart>(p, sh.large, st)) return rc;
  if (!finish) return SOMA_OK;
  p.splits = sh.splits;
  const unsigned tiles = unsigned(p.ntm * p.ntn);
  constexpr Tile t = {16, PARTS == 1 ? 16 : 8};           // tile_of(true, PARTS, false)
  if (sh.large) return launch("k_ce_sum", k_ce_sum<T, PARTS, t.tn, t.tm>, dim3(tiles, t.tn * t.tm / 4), dim3(256), 0, st, p);
  return launch("k_ce_sum", k_ce_sum<T, PARTS, 8, 8>, dim3(tiles, 16), dim3(256), 0, st, p);
}

// Packs a, and b as well if it is not NULL, which has as many columns.
template <class T, int PARTS>
int launch_pack(const PackArgs& a, const PackArgs* b, hipStream_t st) {
  const PackPair p{{a, b ? *b : a}, a.np / 64};
  const unsigned blocks = unsigned(p.first + (b ? b->np / 64 : 0));
  return launch("k_ce_pack", k_ce_pack<T, PARTS>, dim3(blocks, unsigned(a.Kp / 64)), dim3(256), 0, st, p);
}

// Partial maxima of each array: a block for every four rows of the larger one.
int maxima_of(const soma_ce_config& c) {
  return int(std::min<int64_t>(kMaxima, up((std::max(c.rows, c.vocab) + 3) / 4, 4)));
}

size_t rows_lds(int width, size_t size, int tiles) { return size_t(up(width, 64)) * 16 * tiles * size; }

// Row tiles of a pass of k_ce_rows, 0: not by it.  Its one or two readings of E
// against a packed copy written and read as well (bf16, 50,257 x 1,024: 64 rows
// 28.9 us, packed 97; 128 rows in two passes 54.7, packed 98).  Of a small head
// nothing is bound by reading, and a second pass costs more than packing: 2,000 x
// 768, 128 rows, 24.8 us, packed 17.3; 16,000 x 512 either way 21.6; 32,000 x 512
// 25.7, packed 39.  fp32 takes 32 rows a pass: its matrix instruction is a
// sixteenth as fast, and bounds 64 in one (107 us, 2 x 32: 103, packed 221).
int rows_of(const soma_ce_config& c, size_t size) {
  int most = size == 2 ? 4 : 2;
  while (most > 0 && rows_lds(c.width, size, most) > kRowsLds) most /= 2;
  if (most == 0 || c.rows > 32 * most) return 0;
  const int passes = c.rows > 16 * most ? 2 : 1;
  if (passes == 2 && int64_t(c.vocab) * c.width * int64_t(size) < kTwiceBytes) return 0;
  int tiles = 1;
  while (16 * tiles * passes < c.rows) tiles *= 2;
  return tiles;
}

template <class T, int RT>
int launch_rows(const RowsArgs& a, int blocks, hipStream_t st) {
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_ce_rows<T, RT>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, int(kRowsLds));
  if (e != hipSuccess) return device_error("hipFuncSetAttribute", e);
  return launch("k_ce_rows", k_ce_rows<T, RT>, dim3(blocks), dim3(64 * kRowsWaves), unsigned(rows_lds(a.K, sizeof(T), RT)), st, a);
}

template <class T, int PARTS>
int loss_typed(const soma_ce_config& c, const void* f, const void* E, const int32_t* targets, float* loss, float* lse,
               char* ws, hipStream_t st) {
  const Sizes s = sizes_of(c, false);
  float2* part = reinterpret_cast<float2*>(ws + s.part);
  float* hit = reinterpret_cast<float*>(ws + s.hit);
  int subs = 0, stride = 0;
  const int tiles = rows_of(c, sizeof(T));
  if (tiles) {
    subs = int(std::min<int64_t>(kRowsBlocks, up(c.vocab, 16) / 16));
    stride = int(up(c.rows, 16));
    for (int r0 = 0; r0 < c.rows; r0 += 16 * tiles) {
      const RowsArgs a{static_cast<const T*>(f) + r0 * c.f_stride, E, c.f_stride, c.e_stride, targets + r0,
                       std::min(c.rows - r0, 16 * tiles), c.vocab, c.width, part + r0, stride, stride - r0,
                       hit + r0};
      int rc = SOMA_OK;
      if (tiles == 1)
        rc = launch_rows<T, 1>(a, subs, st);
      else if (tiles == 2)
        rc = launch_rows<T, 2>(a, subs, st);
      else if constexpr (PARTS == 1)
        rc = launch_rows<T, 4>(a, subs, st);
      if (rc) return rc;
    }
  } else {
    float* maxima = reinterpret_cast<float*>(ws + s.maxima);
    Scales* scales = reinterpret_cast<Scales*>(ws + s.scales);
    uint16_t* fp = reinterpret_cast<uint16_t*>(ws + s.f);
    uint16_t* ep = reinterpret_cast<uint16_t*>(ws + s.e);
    const int nmax = maxima_of(c);
    if (PARTS == 2) {
      const MaxArgs m{f, E, nullptr, targets, c.f_stride, c.e_stride, c.rows, c.vocab, c.width, maxima};
      if (int rc = launch("k_ce_max", k_ce_max<T>, dim3(nmax, 3), dim3(256), 0, st, m, 0)) return rc;
    }
    PackArgs a{};
    a.x = f, a.stride = c.f_stride, a.n = c.rows, a.K = c.width, a.np = int(s.Rp), a.Kp = int(s.Kp);
    a.targets = targets, a.frag = fp, a.maxima = PARTS == 2 ? maxima : nullptr, a.nmax = nmax, a.scales = scales;
    a.V = c.vocab;
    stride = int(s.Rp);
    const int piece = piece_of(c);
    for (int v0 = 0; v0 < c.vocab; v0 += piece) {
      const int n = std::min(piece, c.vocab - v0), np = int(up(n, 128));
      PackArgs b{};
      b.x = static_cast<const T*>(E) + int64_t(v0) * c.e_stride, b.stride = c.e_stride, b.n = n, b.K = c.width;
      b.np = np, b.Kp = int(s.Kp), b.frag = ep, b.maxima = a.maxima, b.nmax = nmax, b.which = 1;
      if (int rc = v0 == 0 ? launch_pack<T, PARTS>(a, &b, st) : launch_pack<T, PARTS>(b, nullptr, st)) return rc;
      CeMmArgs p{};
      p.A = fp, p.W = ep, p.ta = int(s.Rp / 16), p.tw = np / 16, p.KC = int(s.Kp / 32), p.scales = scales;
      p.part = part, p.part_stride = stride, p.sub0 = subs, p.hit = hit, p.targets = targets, p.R = c.rows, p.V = n, p.v0 = v0;
      const bool large = large_logits(s.Rp, np, s.Kp, PARTS);
      p.splits = 1;
      if (int rc = launch_mm<T, PARTS, kStats>(p, large, st)) return rc;
      subs += p.tile_subs * p.ntn;
    }
  }
  const dim3 jgrid((c.rows + 15) / 16);
  if (subs <= 32)
    return launch("k_ce_join", k_ce_join<8>, jgrid, dim3(128), 0, st, part, subs, stride, targets, hit, c.rows, c.vocab, loss, lse);
  return launch("k_ce_join", k_ce_join<64>, jgrid, dim3(1024), 0, st, part, subs, stride, targets, hit, c.rows, c.vocab, loss, lse);
}

template <class T, int PARTS>
int grad_typed(const soma_ce_config& c, const void* f, const void* E, const int32_t* targets, const float* lse,
               const float* w, void* df, void* dE, char* ws, hipStream_t st) {
  const Sizes s = sizes_of(c, true);
  float* maxima = reinterpret_cast<float*>(ws + s.maxima);
  Scales* scales = reinterpret_cast<Scales*>(ws + s.scales);
  RowMeta* meta = reinterpret_cast<RowMeta*>(ws + s.meta);
  auto at = [&](size_t o) { return reinterpret_cast<uint16_t*>(ws + o); };
  const MaxArgs m{f, E, w, targets, c.f_stride, c.e_stride, c.rows, c.vocab, c.width, maxima};
  const int nmax = PARTS == 2 ? maxima_of(c) : 64;
  if (int rc = launch("k_ce_max", k_ce_max<T>, dim3(nmax, PARTS == 2 ? 3 : 1), dim3(256), 0, st, m, PARTS == 2 ? 0 : 2)) return rc;
  PackArgs a{};
  a.x = f, a.stride = c.f_stride, a.n = c.rows, a.K = c.width, a.np = int(s.Rp), a.Kp = int(s.Kp);
  a.targets = targets, a.frag = at(s.f), a.fragT = dE ? at(s.fT) : nullptr, a.maxima = maxima, a.nmax = nmax;
  a.scales = scales, a.meta = meta, a.lse = lse, a.w = w, a.V = c.vocab;
  const Shares of_df = shares_of(s.Rp, s.Kp, s.Vp, PARTS, c.vocab > piece_of(c));
  const int piece = piece_of(c);
  for (int v0 = 0; v0 < c.vocab; v0 += piece) {
    const int n = std::min(piece, c.vocab - v0), np = int(up(n, 128));
    PackArgs b{};
    b.x = static_cast<const T*>(E) + int64_t(v0) * c.e_stride, b.stride = c.e_stride, b.n = n, b.K = c.width;
    b.np = np, b.Kp = int(s.Kp), b.frag = at(s.e), b.fragT = df ? at(s.eT) : nullptr;
    b.maxima = PARTS == 2 ? maxima : nullptr, b.nmax = nmax, b.which = 1;
    if (int rc = v0 == 0 ? launch_pack<T, PARTS>(a, &b, st) : launch_pack<T, PARTS>(b, nullptr, st)) return rc;
    CeMmArgs p{};
    p.A = at(s.f), p.W = at(s.e), p.ta = int(s.Rp / 16), p.tw = np / 16, p.KC = int(s.Kp / 32), p.scales = scales;
    p.meta = meta, p.G = at(s.G), p.GT = at(s.GT), p.V = n, p.v0 = v0;
    p.splits = 1;
    if (int rc = launch_mm<T, PARTS, kGrad>(p, large_logits(s.Rp, np, s.Kp, PARTS), st)) return rc;
    if (df) {
      CeMmArgs q{};
      q.A = at(s.G), q.W = at(s.eT), q.ta = int(s.Rp / 16), q.tw = int(s.Kp / 16), q.KC = np / 32, q.scales = scales;
      q.out = df, q.M = c.rows, q.N = c.width, q.acc = reinterpret_cast<float4*>(ws + s.accf), q.add = v0 > 0;
      if (int rc = launch_product<T, PARTS>(q, of_df, c.vocab <= piece, v0 + piece >= c.vocab, st)) return rc;
    }
    if (dE) {
      CeMmArgs q{};
      q.A = at(s.GT), q.W = at(s.fT), q.ta = np / 16, q.tw = int(s.Kp / 16), q.KC = int(s.Rp / 32), q.scales = scales;
      q.out = static_cast<T*>(dE) + int64_t(v0) * c.width, q.M = n, q.N = c.width, q.is_de = 1;
      q.acc = reinterpret_cast<float4*>(ws + s.acce);
      if (int rc = launch_product<T, PARTS>(q, shares_of(np, s.Kp, s.Rp, PARTS, false), true, true, st)) return rc;
    }
  }
  return SOMA_OK;
}

}  // namespace
}  // namespace soma

using namespace soma;

extern "C" {

int soma_ce_workspace_size(const soma_ce_config* cfg, int grad, size_t* bytes) {
  if (int rc = check_ce(cfg)) return rc;
  if (!bytes) return set_error(SOMA_EINVAL, "bytes is NULL");
  *bytes = sizes_of(*cfg, false).total;
  if (grad) *bytes = std::max(*bytes, sizes_of(*cfg, true).total);
  return set_ok();
}

int soma_ce_loss(const soma_ce_config* cfg, const void* f, const void* E, const int32_t* targets, float* loss, float* lse,
                 void* workspace, size_t ws_bytes, void* stream) {
  if (int rc = check_ce(cfg)) return rc;
  const soma_ce_config& c = *cfg;
  if (c.rows == 0) return set_ok();
  if (!f || !E || !targets || (!loss && !lse)) return set_error(SOMA_EINVAL, "NULL device pointer");
  const size_t e = type_size(c.type);
  if (!is_aligned(f, e) || !is_aligned(E, e) || !is_aligned(targets, 4) || !is_aligned(loss, 4) || !is_aligned(lse, 4))
    return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  if (int rc = check_workspace(workspace, ws_bytes, sizes_of(c, false).total)) return rc;
  char* ws = static_cast<char*>(workspace);
  const hipStream_t st = stream_of(stream);
  if (int rc = c.type == SOMA_FLOAT ? loss_typed<float, 2>(c, f, E, targets, loss, lse, ws, st)
                                    : loss_typed<bf16, 1>(c, f, E, targets, loss, lse, ws, st))
    return rc;
  return set_ok();
}

int soma_ce_grad(const soma_ce_config* cfg, const void* f, const void* E, const int32_t* targets, const float* lse,
                 const float* grad_loss, void* df, void* dE, void* workspace, size_t ws_bytes, void* stream) {
  if (int rc = check_ce(cfg)) return rc;
  const soma_ce_config& c = *cfg;
  const size_t e = type_size(c.type);
  if (c.rows > 0 && !df && !dE) return set_error(SOMA_EINVAL, "neither df nor dE is wanted");   // of no rows, df has no address
  if (c.rows > 0 && (!f || !E || !targets || !lse || !grad_loss)) return set_error(SOMA_EINVAL, "NULL device pointer");
  if (!is_aligned(f, e) || !is_aligned(E, e) || !is_aligned(targets, 4) || !is_aligned(lse, 4) ||
      !is_aligned(grad_loss, 4))
    return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  if (!is_aligned(df, 16) || !is_aligned(dE, 16)) return set_error(SOMA_EINVAL, "df and dE must be 16-byte aligned");
  if (int rc = check_workspace(workspace, ws_bytes, sizes_of(c, true).total)) return rc;
  const hipStream_t st = stream_of(stream);
  if (c.rows == 0) {                      // no row: dE is a sum of nothing
    if (dE) {
      const int64_t halves = int64_t(c.vocab) * c.width * int64_t(e) / 2;
      if (int rc = launch("k_ce_zero", k_ce_zero, dim3(1024), dim3(256), 0, st, static_cast<uint16_t*>(dE), halves)) return rc;
    }
    return set_ok();
  }
  char* ws = static_cast<char*>(workspace);
  if (int rc = c.type == SOMA_FLOAT ? grad_typed<float, 2>(c, f, E, targets, lse, grad_loss, df, dE, ws, st)
                                    : grad_typed<bf16, 1>(c, f, E, targets, lse, grad_loss, df, dE, ws, st))
    return rc;
  return set_ok();
}

}  // extern "C"
