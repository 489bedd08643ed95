// soma_norm.hip -- dropout from the counter-based generator, and the root-mean-square
// norm with the residual's addition:
//   total = residual + drop(x),   y = gain total / sqrt(mean(total^2) + eps),
// forward (y in fp32, bf16 or e4m3 codes with a scale for each row) and backward.
//
// A lane works on groups of eight elements, i = 8 b .. 8 b + 7 of the array as if its
// rows lay side by side, which are one Philox block's (16 bits an element) and, where
// rows do lie so, 16 or 32 aligned bytes whatever the width: only the groups at a row's
// two ends are stored element by element.  The mask is formed again wherever it is needed.
//
// Norm: a row is one wave's (up to 2,048 columns; backward 1,024), or a block's of up to
// 1,024 lanes, and stays in registers between its sum of squares and its output; each array is
// read or written once.  Bound by memory, with dropout beside Philox's multiplications
// (20 of 32 x 32 bits for eight elements).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "soma.h"
#include "soma_eights.hpp"
#include "soma_host.hpp"
#include "soma_rng.hpp"
#include "soma_types.hpp"

namespace soma {
namespace {

// What decides which elements are kept.
struct Drop {
  uint64_t seed, step;
  const uint64_t* step_dev;   // added to step, or NULL
  uint32_t layer, cut;        // an element whose field is below `cut` is dropped
  float scale;                // of what is kept
};

// Key and counter words of a launch.
struct Stream {
  uint2 key;
  uint32_t layer, step, cut;
  float scale;
  __device__ __forceinline__ explicit Stream(const Drop& d) {
    const uint64_t s = d.step + (d.step_dev ? *d.step_dev : 0);
    key = stream_key(d.seed, s);
    layer = d.layer, step = static_cast<uint32_t>(s), cut = d.cut, scale = d.scale;
  }
  // x, kept and scaled or 0: what is dropped is 0 whatever it was.
  __device__ __forceinline__ void apply(int64_t block, float (&x)[8]) const {
    const uint4 w = philox4x32_10(make_uint4(static_cast<uint32_t>(block), layer, step, static_cast<uint32_t>(block >> 32)), key);
    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t field = i & 1 ? word[i / 2] >> 16 : word[i / 2] & 0xFFFFu;
      x[i] = field >= cut ? x[i] * scale : 0.0f;
    }
  }
};

// Elements lo to hi - 1 of the eight at p + at.  Where groups are aligned (vec) all eight
// are read at once, also at a row's two ends (what is around, not zeros then, belongs to
// the rows before and behind), but for the last row (`last`).  Rows so narrow that a group
// reaches past the next one are never `vec`.
template <class T>
__device__ __forceinline__ void load_eight(const T* p, int64_t at, bool vec, bool last, int lo, int hi, float (&x)[8]) {
  if (reads_whole(vec, last, lo, hi)) {
    if constexpr (sizeof(T) == 2) {
      const uint4 u = *reinterpret_cast<const uint4*>(p + at);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    } else {
      const float4 a = load_four(p + at), b = load_four(p + at + 4);
      x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i >= lo && i < hi ? load_value(p + at + i) : 0.0f;
  }
}
// Zeros around them (without a branch, which would part the loads of several groups:
// 16,384 rows of 4,096 in codes 103 us for 96).
__device__ __forceinline__ void clear_around(int lo, int hi, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = static_cast<unsigned>(i - lo) < static_cast<unsigned>(hi - lo) ? x[i] : 0.0f;
}
// Those elements, and nothing around them.
template <class T>
__device__ __forceinline__ void store_eight(T* p, int64_t at, bool vec, int lo, int hi, const float (&x)[8]) {
  if (vec && lo == 0 && hi == 8) {
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint4*>(p + at) =
          make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
    } else {
      store_four(p + at, make_float4(x[0], x[1], x[2], x[3]));
      store_four(p + at + 4, make_float4(x[4], x[5], x[6], x[7]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= lo && i < hi) store_value(p + at + i, x[i]);
  }
}

struct DropArgs {
  const void *x, *residual;
  void* y;
  int64_t x_stride, residual_stride, rows, width, groups;   // groups of a row at the most
  int x_vec, residual_vec, y_vec;
  Drop drop;
};

// A lane a group.  65,536 rows of 1,024 in bf16, added to a residual: 70 us, 402 MB at 5.8
// TB/s (a copy's rate from memory would take 78: some of it lies in the caches).
template <class T, bool kDrop>
__global__ __launch_bounds__(256) void k_dropout(const DropArgs a) {
  const Stream s(a.drop);
  const int64_t u = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t row = a.rows == 1 ? 0 : u / a.groups;
  if (row >= a.rows) return;
  const Eight g(row, a.width, u - row * a.groups);
  if (g.hi <= g.lo) return;
  const bool last = row + 1 == a.rows;
  float x[8], r[8];
  load_eight(static_cast<const T*>(a.x), row * a.x_stride + g.col, a.x_vec, last, g.lo, g.hi, x);
  if (a.residual) load_eight(static_cast<const T*>(a.residual), row * a.residual_stride + g.col, a.residual_vec, last, g.lo, g.hi, r);
  if constexpr (kDrop) s.apply(g.block, x);
  if (a.residual) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = r[i] + x[i];
  }
  store_eight(static_cast<T*>(a.y), row * a.width + g.col, a.y_vec, g.lo, g.hi, x);
}

// A block's threads, and its rows, where kLanes of them share one.
constexpr int threads_of(int lanes) { return lanes == 64 ? 256 : lanes; }
constexpr int rows_of(int lanes) { return lanes == 64 ? 4 : 1; }

// Sum, or largest value, over the lanes that share a row, in every one of them.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}
template <int kLanes, bool kMax>
__device__ __forceinline__ float over_row(float v, float* lds) {
  v = kMax ? wave_max(v) : wave_sum(v);
  if constexpr (kLanes > 64) {
    constexpr int kW = kLanes / 64;
    __syncthreads();                        // lds has been read
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < kW; ++w) v = kMax ? fmaxf(v, lds[w]) : v + lds[w];
  }
  return v;
}

// Two sums at once.
template <int kLanes>
__device__ __forceinline__ void over_row(float& a, float& b, float* lds) {
  a = wave_sum(a), b = wave_sum(b);
  if constexpr (kLanes > 64) {
    constexpr int kW = kLanes / 64;
    __syncthreads();                        // lds has been read
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a, lds[kW + (threadIdx.x >> 6)] = b;
    __syncthreads();
    a = lds[0], b = lds[kW];
#pragma unroll
    for (int w = 1; w < kW; ++w) a += lds[w], b += lds[kW + w];
  }
}

struct NormArgs {
  const void *x, *residual, *dy, *dtotal;
  const float* gain;
  void *total, *y, *dresidual, *dx;
  float* scales;              // forward into codes
  float* partial;             // backward: [blocks][width], or NULL
  int64_t x_stride, residual_stride;
  int first, rows, width;     // rows from `first` on (forward)
  int x_vec, residual_vec, total_vec, y_vec, dy_vec, dtotal_vec, dresidual_vec, dx_vec;
  float eps;
  Drop drop;
};

// The gain of a group's columns, 0 outside.  (Loads of 16 bytes take a float's alignment.)
__device__ __forceinline__ void load_gain(const float* gain, int width, int col, int lo, int hi, float (&g)[8]) {
  typedef float Four __attribute__((ext_vector_type(4), aligned(4)));
  if (lo == 0 && hi == 8) {
    const Four a = *reinterpret_cast<const Four*>(gain + col), b = *reinterpret_cast<const Four*>(gain + col + 4);
    g[0] = a[0], g[1] = a[1], g[2] = a[2], g[3] = a[3], g[4] = b[0], g[5] = b[1], g[6] = b[2], g[7] = b[3];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = gain[min(max(col + i, 0), width - 1)];
    clear_around(lo, hi, g);
  }
}

// T: x and y; S: residual and total; kLanes lanes a row, kGroups groups a lane; kRagged:
// the width is no multiple of 8, and groups lie across the rows' ends.
// 16,384 rows of 4,096 in bf16 with codes: 91 us, 470 MB at 5.15 TB/s; 65,536 of 512, bf16
// with fp32 sums and dropout: 71 us, 403 MB at 5.7.  Ragged widths fall behind where the
// caches hold nothing of the inputs: 22,000 of 361 in fp32 34 to 36 us, 127 MB at 3.6 (25
// where they do; of 360 30 and 22), 8,192 of 4,099 in bf16 66 us (52; of 4,096 54 and 42).
// Rows' ends read one element at a time took 30 for those 25, and 107 for the 52.
template <class T, class S, int kLanes, int kGroups, bool kCodes, bool kRagged>
__global__ __launch_bounds__(threads_of(kLanes)) void k_norm_forward(const NormArgs a) {
  __shared__ float lds[16];
  constexpr int kRows = rows_of(kLanes);
  const int lane = threadIdx.x % kLanes, row = a.first + static_cast<int>(blockIdx.x * kRows + threadIdx.x / kLanes);
  if (row >= a.rows) return;                // whole waves, or the block
  const bool last = row + 1 == a.rows;
  const Stream s(a.drop);
  float t[kGroups][8];
  float sum = 0.0f;
#pragma unroll
  for (int k = 0; k < kGroups; ++k) {
    const Group<kLanes, kRagged> g(row, a.width, lane, k);
    if (g.hi <= g.lo) {
#pragma unroll
      for (int i = 0; i < 8; ++i) t[k][i] = 0.0f;
      continue;
    }
    load_eight(static_cast<const T*>(a.x), row * a.x_stride + g.col, a.x_vec, last, g.lo, g.hi, t[k]);
    if (a.residual) {
      float r[8];
      load_eight(static_cast<const S*>(a.residual), row * a.residual_stride + g.col, a.residual_vec, last, g.lo, g.hi, r);
      if (a.drop.cut) s.apply(g.block, t[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) t[k][i] = r[i] + t[k][i];
    } else if (a.drop.cut) {
      s.apply(g.block, t[k]);
    }
    if constexpr (kRagged) clear_around(g.lo, g.hi, t[k]);
    if (a.total)
      store_eight(static_cast<S*>(a.total), static_cast<int64_t>(row) * a.width + g.col, a.total_vec, g.lo, g.hi, t[k]);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += t[k][i] * t[k][i];
  }
  const float inv = 1.0f / sqrtf(over_row<kLanes, false>(sum, lds) / static_cast<float>(a.width) + a.eps);
  float top = 0.0f;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < kGroups; ++k) {
    const Group<kLanes, kRagged> g(row, a.width, lane, k);
    if (g.hi <= g.lo) continue;
    float gain[8];
    load_gain(a.gain, a.width, g.col, g.lo, g.hi, gain);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      t[k][i] = t[k][i] * inv * gain[i];
      if (kCodes && i >= g.lo && i < g.hi) {
        top = fmaxf(top, fabsf(t[k][i]));
        bad |= t[k][i] != t[k][i];
      }
    }
    if constexpr (!kCodes)
      store_eight(static_cast<T*>(a.y), static_cast<int64_t>(row) * a.width + g.col, a.y_vec, g.lo, g.hi, t[k]);
  }
  if constexpr (kCodes) {
    top = over_row<kLanes, true>(top, lds);
    const float nan = over_row<kLanes, true>(bad ? 1.0f : 0.0f, lds);
    // (a scale below the normal numbers has no reciprocal: such a row's is the least of them)
    const bool tiny = top > 0.0f && top < 448.0f * 0x1p-126f;
    const float up = tiny ? 0x1p126f : top > 0.0f ? 448.0f / top : 0.0f;
    if (lane == 0) a.scales[row] = nan > 0.0f ? __uint_as_float(0x7FC00000u) : tiny ? 0x1p-126f : top * (1.0f / 448.0f);
    uint8_t* const y = static_cast<uint8_t*>(a.y) + static_cast<int64_t>(row) * a.width;
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      const Group<kLanes, kRagged> g(row, a.width, lane, k);
      if (g.hi <= g.lo) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) t[k][i] *= up;
      int lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[k][0], t[k][1], 0, false);
      lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[k][2], t[k][3], lo, true);
      int hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[k][4], t[k][5], 0, false);
      hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[k][6], t[k][7], hi, true);
      if (a.y_vec && g.lo == 0 && g.hi == 8) {
        *reinterpret_cast<uint2*>(y + g.col) = make_uint2(lo, hi);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i >= g.lo && i < g.hi) y[g.col + i] = static_cast<uint8_t>((i < 4 ? lo : hi) >> (8 * (i & 3)));
      }
    }
  }
}

// With n = total / rms, h = dy gain:  dresidual = dtotal + (h - n mean(h n)) / rms,
// dx = drop(dresidual), dgain = sum over rows of dy n.  Blocks walk over rows, a multiple
// of 8 apart, so that whatever the width a lane's columns are the same in every row and
// their sums stay in registers.  65,536 rows of 512 (bf16, fp32 sums, dropout): 112 to
// 119 us, 537 MB at 4.5 to 4.8 TB/s; 22,000 of 361 in fp32: 45 us, 159 MB at 3.5 (31 where
// the caches hold a part of the inputs).
template <class T, class S, int kLanes, int kGroups, bool kRagged>
__global__ __launch_bounds__(threads_of(kLanes)) void k_norm_backward(const NormArgs a) {
  constexpr int kRows = rows_of(kLanes);
  __shared__ float lds[32];
  extern __shared__ float sums[];           // kRows > 1: [kRows][width], eight columns nine apart
  const int lane = threadIdx.x % kLanes, mine = threadIdx.x / kLanes;
  const int line = a.width + a.width / 8 + 1;
  float* const own = sums + mine * line;
  const Stream s(a.drop);
  float part[kGroups][8];
#pragma unroll
  for (int k = 0; k < kGroups; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) part[k][i] = 0.0f;
  for (int row = blockIdx.x * kRows + mine; row < a.rows; row += gridDim.x * kRows) {
    const int64_t at = static_cast<int64_t>(row) * a.width;
    const bool last = row + 1 == a.rows;
    float t[kGroups][8], h[kGroups][8];
    float squares = 0.0f, dot = 0.0f;
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      const Group<kLanes, kRagged> g(row, a.width, lane, k);
      if (g.hi <= g.lo) continue;
      load_eight(static_cast<const S*>(a.total), at + g.col, a.total_vec, last, g.lo, g.hi, t[k]);
      load_eight(static_cast<const T*>(a.dy), at + g.col, a.dy_vec, last, g.lo, g.hi, h[k]);
      float gain[8];
      load_gain(a.gain, a.width, g.col, g.lo, g.hi, gain);
      if constexpr (kRagged) {
        clear_around(g.lo, g.hi, t[k]);
        clear_around(g.lo, g.hi, h[k]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        squares += t[k][i] * t[k][i];
        dot += h[k][i] * gain[i] * t[k][i];
      }
    }
    over_row<kLanes>(squares, dot, lds);
    const float n = static_cast<float>(a.width), inv = 1.0f / sqrtf(squares / n + a.eps);
    const float mean = dot * inv / n;       // of h n
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      const Group<kLanes, kRagged> g(row, a.width, lane, k);
      if (g.hi <= g.lo) continue;
      float gain[8], d[8];
      load_gain(a.gain, a.width, g.col, g.lo, g.hi, gain);
      // (not kept in registers, of which 16 waves have 128 each)
      if constexpr (kLanes == 1024) {
        load_eight(static_cast<const T*>(a.dy), at + g.col, a.dy_vec, last, g.lo, g.hi, h[k]);
        if constexpr (kRagged) clear_around(g.lo, g.hi, h[k]);
      }
      if (a.dtotal) {
        load_eight(static_cast<const S*>(a.dtotal), at + g.col, a.dtotal_vec, last, g.lo, g.hi, d);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = t[k][i] * inv;
        part[k][i] += h[k][i] * x;
        d[i] += inv * (h[k][i] * gain[i] - x * mean);
      }
      if (a.dresidual) store_eight(static_cast<S*>(a.dresidual), at + g.col, a.dresidual_vec, g.lo, g.hi, d);
      if (a.dx) {
        if (a.drop.cut) s.apply(g.block, d);
        store_eight(static_cast<T*>(a.dx), at + g.col, a.dx_vec, g.lo, g.hi, d);
      }
    }
  }
  if (!a.partial) return;
  float* const out = a.partial + static_cast<int64_t>(blockIdx.x) * a.width;
#pragma unroll
  for (int k = 0; k < kGroups; ++k) {
    const Group<kLanes, kRagged> g(blockIdx.x * kRows + mine, a.width, lane, k);
    if (g.hi <= g.lo) continue;
    if constexpr (kRows == 1) {
      store_eight(out, g.col, a.width % 8 == 0, g.lo, g.hi, part[k]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i >= g.lo && i < g.hi) own[g.col + i + (g.col + i) / 8] = part[k][i];
    }
  }
  if constexpr (kRows > 1) {
    __syncthreads();
    for (int c = threadIdx.x; c < a.width; c += kLanes * kRows) {
      float x = sums[c + c / 8];
#pragma unroll
      for (int r = 1; r < kRows; ++r) x += sums[r * line + c + c / 8];
      out[c] = x;
    }
  }
}

// dgain: the blocks' sums, 16 waves a block of 64 columns: latency, 6 us.
__global__ __launch_bounds__(1024) void k_norm_gain(const float* partial, int blocks, int width, float* dgain) {
  __shared__ float sums[16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
  float x = 0.0f;
  if (c < width) {
    // sixteen on their way at once
    for (int b0 = w; b0 < blocks; b0 += 256) {
      float p[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) p[k] = b0 + 16 * k < blocks ? partial[static_cast<int64_t>(b0 + 16 * k) * width + c] : 0.0f;
#pragma unroll
      for (int k = 0; k < 16; ++k) x += p[k];
    }
  }
  sums[w][threadIdx.x & 63] = x;
  __syncthreads();
  if (w == 0 && c < width) {
#pragma unroll
    for (int i = 1; i < 16; ++i) x += sums[i][threadIdx.x];
    dgain[c] = x;
  }
}

// ---------------------------------------------------------------------------
// Host

constexpr int kMostWidth = 1 << 14;

int fill_drop(const soma_drop* d, Drop* out) {
  *out = Drop{};
  out->scale = 1.0f;
  if (!d) return SOMA_OK;
  if (d->reserved) return set_error(SOMA_EINVAL, "reserved must be 0");
  if (!(d->p >= 0.0 && d->p < 1.0)) return set_error(SOMA_EINVAL, "p must be in [0, 1)");
  const long cut = lrint(d->p * 65536.0);
  if (cut > 65535) return set_error(SOMA_EINVAL, "p %g leaves less than 1 of 65,536 elements", d->p);
  if (!is_aligned(d->step_dev, 8)) return set_error(SOMA_EINVAL, "step_dev is not aligned to its element");
  out->seed = d->seed, out->step = d->step, out->step_dev = d->step_dev, out->layer = d->layer;
  out->cut = static_cast<uint32_t>(cut);
  out->scale = static_cast<float>(65536.0 / (65536 - cut));
  return SOMA_OK;
}

bool in_eights(const void* p, int64_t stride, int64_t width, size_t e) { return soma::in_eights(is_aligned(p, 16), stride, width, e); }

int check_norm(const soma_norm_config* cfg) {
  if (!cfg) return set_error(SOMA_EINVAL, "cfg is NULL");
  const soma_norm_config& c = *cfg;
  if (c.reserved) return set_error(SOMA_EINVAL, "reserved must be 0");
  if (!is_type(c.type) || !is_type(c.sum_type)) return set_error(SOMA_EINVAL, "a type is none of enum soma_type");
  if (c.type == SOMA_FLOAT && c.sum_type == SOMA_BFLOAT) return set_error(SOMA_EINVAL, "sums in bf16 of an fp32 branch");
  if (c.rows < 0 || c.rows > (1 << 30)) return set_error(SOMA_ESHAPE, "rows %d is out of range", c.rows);
  if (c.width < 1 || c.width > kMostWidth) return set_error(SOMA_ESHAPE, "width %d is out of range", c.width);
  if (!(c.eps >= 0.0f) || std::isinf(c.eps)) return set_error(SOMA_EINVAL, "eps must be finite and not negative");
  if (c.x_stride < c.width || c.residual_stride < c.width) return set_error(SOMA_ESHAPE, "a row stride is shorter than its row");
  if (c.x_stride > (int64_t{1} << 32) || c.residual_stride > (int64_t{1} << 32))
    return set_error(SOMA_ESHAPE, "a row stride is out of range");
  return SOMA_OK;
}

int lanes_of(int width) {
  const int64_t g = groups_of(width);
  return g <= 128 ? 64 : g <= 256 ? 128 : g <= 512 ? 256 : g <= 1024 ? 512 : 1024;
}
// Blocks of the backward pass: a block a row, or a multiple of eight, up to 1,024 of 64
// lanes a row (512, 1,024 and 2,048: 22,000 rows of 361 in fp32, from the caches, both passes
// 70, 63 and 70 us, 65,536 of 512 in bf16 199, 193 and 199), of more lanes as many lanes in
// all: 2,048 of 128, 1,024 of 256, at least 512.
int backward_blocks(const soma_norm_config& c) {
  const int lanes = lanes_of(c.width), rows = rows_of(lanes);
  return std::max(1, std::min((c.rows + rows - 1) / rows, lanes == 64 ? 1024 : std::max(512, (1 << 18) / lanes)));
}

template <class T, class S, int kLanes, int kGroups, bool kCodes, bool kRagged>
int forward_in(NormArgs a, hipStream_t st) {
  constexpr int kRows = rows_of(kLanes), kMost = static_cast<int>(kMostThreads / 2 / kLanes);
  for (; a.first < a.rows; a.first += kMost)
    if (int rc = launch("k_norm_forward", k_norm_forward<T, S, kLanes, kGroups, kCodes, kRagged>,
                        dim3((std::min(a.rows - a.first, kMost) + kRows - 1) / kRows), dim3(threads_of(kLanes)), 0, st, a))
      return rc;
  return SOMA_OK;
}
template <class T, class S, int kLanes, int kGroups, bool kCodes>
int forward_as(const NormArgs& a, hipStream_t st) {
  return a.width % 8 ? forward_in<T, S, kLanes, kGroups, kCodes, true>(a, st) : forward_in<T, S, kLanes, kGroups, kCodes, false>(a, st);
}
template <class T, class S, int kLanes, int kGroups>
int backward_as(const NormArgs& a, int blocks, hipStream_t st) {
  constexpr int kRows = rows_of(kLanes);
  const unsigned lds = kRows == 1 ? 0 : sizeof(float) * kRows * (a.width + a.width / 8 + 1);
  const auto kernel = a.width % 8 ? k_norm_backward<T, S, kLanes, kGroups, true> : k_norm_backward<T, S, kLanes, kGroups, false>;
  return launch("k_norm_backward", kernel, dim3(blocks), dim3(threads_of(kLanes)), lds, st, a);
}

// f(lanes, groups) with the instance for this width.  Two groups a lane leave the
// backward pass registers for twice the waves: 20,000 rows of 1,536 in bf16 84 us, four
// groups in a wave 101; 8,192 of 5,120 117, four groups in 256 lanes 160.  (Forward 1,536:
// 37 both ways, 1,100: 38 and 36; 5,120 in fp32: 139 and 153.)
template <bool kForward, class F>
int by_width(int width, F f) {
  const int64_t g = groups_of(width);
  using std::integral_constant;
#define SOMA_NORM(l, n) f(integral_constant<int, l>{}, integral_constant<int, n>{})
  if (g <= 64) return SOMA_NORM(64, 1);
  if (g <= 128) return SOMA_NORM(64, 2);
  if (g <= 256) {
    if constexpr (kForward) return SOMA_NORM(64, 4);
    else return SOMA_NORM(128, 2);
  }
  if (g <= 512) return SOMA_NORM(256, 2);
  if (g <= 1024) return SOMA_NORM(512, 2);
  return SOMA_NORM(1024, 3);
#undef SOMA_NORM
}

// f(T, S) with the types of this configuration.
template <class F>
int by_type(const soma_norm_config& c, F f) {
  if (c.type == SOMA_FLOAT) return f(float{}, float{});
  return c.sum_type == SOMA_FLOAT ? f(bf16{}, float{}) : f(bf16{}, bf16{});
}

int norm_forward(const soma_norm_config* cfg, const void* x, const void* residual, const float* gain, const soma_drop* drop,
                 void* total, void* y, float* scales, bool codes, void* stream) {
  if (int rc = check_norm(cfg)) return rc;
  const soma_norm_config& c = *cfg;
  const size_t e = type_size(c.type), f = type_size(c.sum_type), out = codes ? 1 : e;
  NormArgs a{};
  if (int rc = fill_drop(drop, &a.drop)) return rc;
  if (!gain || (c.rows > 0 && (!x || !y || (codes && !scales)))) return set_error(SOMA_EINVAL, "NULL device pointer");
  if (!is_aligned(x, e) || !is_aligned(residual, f) || !is_aligned(total, f) || !is_aligned(y, out) || !is_aligned(gain, 4) ||
      !is_aligned(scales, 4))
    return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  const bool in_place = residual && total == residual && (c.residual_stride == c.width || c.rows == 1);
  if (!are_apart({span_of(total, c.rows, c.width, c.width, f), span_of(y, c.rows, c.width, c.width, out),
                  span_of(scales, c.rows, 1, 1, 4)},
                 {span_of(x, c.rows, c.width, c.x_stride, e), {gain, sizeof(float) * c.width},
                  span_of(in_place ? nullptr : residual, c.rows, c.width, c.residual_stride, f),
                  {a.drop.step_dev, sizeof(uint64_t)}}))
    return set_error(SOMA_EINVAL, "an output overlaps another array");
  if (c.rows == 0) return set_ok();
  a.x = x, a.residual = residual, a.gain = gain, a.total = total, a.y = y, a.scales = scales;
  a.x_stride = c.x_stride, a.residual_stride = c.residual_stride;
  a.rows = c.rows, a.width = c.width, a.eps = c.eps;
  a.x_vec = in_eights(x, c.x_stride, c.width, e);
  a.residual_vec = in_eights(residual, c.residual_stride, c.width, f);
  a.total_vec = is_aligned(total, 16);
  a.y_vec = is_aligned(y, codes ? 8 : 16);
  const hipStream_t st = stream_of(stream);
  const int rc = by_type(c, [&](auto t, auto s) {
    return by_width<true>(c.width, [&](auto lanes, auto groups) {
      return codes ? forward_as<decltype(t), decltype(s), lanes(), groups(), true>(a, st)
                   : forward_as<decltype(t), decltype(s), lanes(), groups(), false>(a, st);
    });
  });
  return rc ? rc : set_ok();
}

}  // namespace
}  // namespace soma

using namespace soma;

extern "C" {

int soma_dropout(const soma_dropout_config* cfg, const void* x, const void* residual, const soma_drop* drop, void* y,
                 void* stream) {
  if (!cfg) return set_error(SOMA_EINVAL, "cfg is NULL");
  const soma_dropout_config& c = *cfg;
  if (c.reserved) return set_error(SOMA_EINVAL, "reserved must be 0");
  if (!is_type(c.type)) return set_error(SOMA_EINVAL, "type %d is none of enum soma_type", c.type);
  if (c.rows < 0 || c.rows > (1 << 30)) return set_error(SOMA_ESHAPE, "rows %d is out of range", c.rows);
  if (c.width < 1 || c.width > (1 << 20)) return set_error(SOMA_ESHAPE, "width %d is out of range", c.width);
  if (static_cast<int64_t>(c.rows) * c.width > int64_t{1} << 34) return set_error(SOMA_ESHAPE, "more than 2^34 elements");
  if (c.x_stride < c.width || c.residual_stride < c.width) return set_error(SOMA_ESHAPE, "a row stride is shorter than its row");
  if (c.x_stride > (int64_t{1} << 32) || c.residual_stride > (int64_t{1} << 32))
    return set_error(SOMA_ESHAPE, "a row stride is out of range");
  const size_t e = type_size(c.type);
  DropArgs a{};
  if (int rc = fill_drop(drop, &a.drop)) return rc;
  if (c.rows > 0 && (!x || !y)) return set_error(SOMA_EINVAL, "NULL device pointer");
  if (!is_aligned(x, e) || !is_aligned(residual, e) || !is_aligned(y, e))
    return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  const auto place = [&](const void* p, int64_t stride) { return p == y && (stride == c.width || c.rows == 1); };
  if (!are_apart({span_of(y, c.rows, c.width, c.width, e)},
                 {span_of(place(x, c.x_stride) ? nullptr : x, c.rows, c.width, c.x_stride, e),
                  span_of(place(residual, c.residual_stride) ? nullptr : residual, c.rows, c.width, c.residual_stride, e),
                  {a.drop.step_dev, sizeof(uint64_t)}}))
    return set_error(SOMA_EINVAL, "an output overlaps another array");
  if (c.rows == 0) return set_ok();
  a.x = x, a.residual = residual, a.y = y;
  a.rows = c.rows, a.width = c.width, a.x_stride = c.x_stride, a.residual_stride = c.residual_stride;
  if (c.x_stride == c.width && (!residual || c.residual_stride == c.width)) a.width *= a.rows, a.x_stride = a.residual_stride = a.width, a.rows = 1;
  a.groups = a.rows == 1 ? (a.width + 7) / 8 : groups_of(a.width);
  a.x_vec = in_eights(x, a.x_stride, a.width, e);
  a.residual_vec = in_eights(residual, a.residual_stride, a.width, e);
  a.y_vec = is_aligned(y, 16);
  const int64_t blocks = (a.rows * a.groups + 255) / 256;   // (of 2^34 elements at the most: fewer than 2^24)
  const auto kernel = c.type == SOMA_FLOAT ? (a.drop.cut ? k_dropout<float, true> : k_dropout<float, false>)
                                           : (a.drop.cut ? k_dropout<bf16, true> : k_dropout<bf16, false>);
  if (int rc = launch("k_dropout", kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream_of(stream), a)) return rc;
  return set_ok();
}

int soma_norm_workspace_size(const soma_norm_config* cfg, size_t* bytes) {
  if (int rc = check_norm(cfg)) return rc;
  if (!bytes) return set_error(SOMA_EINVAL, "bytes is NULL");
  *bytes = up256(sizeof(float) * backward_blocks(*cfg) * cfg->width);
  return set_ok();
}

int soma_norm_forward(const soma_norm_config* cfg, const void* x, const void* residual, const float* gain,
                      const soma_drop* drop, void* total, void* y, void* stream) {
  return norm_forward(cfg, x, residual, gain, drop, total, y, nullptr, false, stream);
}

int soma_norm_forward_codes(const soma_norm_config* cfg, const void* x, const void* residual, const float* gain,
                            const soma_drop* drop, void* total, void* codes, float* scales, void* stream) {
  return norm_forward(cfg, x, residual, gain, drop, total, codes, scales, true, stream);
}

int soma_norm_backward(const soma_norm_config* cfg, const void* total, const float* gain, const void* dy, const void* dtotal,
                       const soma_drop* drop, void* dresidual, void* dx, float* dgain, void* workspace, size_t ws_bytes,
                       void* stream) {
  if (int rc = check_norm(cfg)) return rc;
  const soma_norm_config& c = *cfg;
  const size_t e = type_size(c.type), f = type_size(c.sum_type);
  NormArgs a{};
  if (int rc = fill_drop(drop, &a.drop)) return rc;
  if (!gain || (c.rows > 0 && (!total || !dy)) || (!dresidual && !dx && !dgain && c.rows > 0))
    return set_error(SOMA_EINVAL, "NULL device pointer");
  if (!is_aligned(total, f) || !is_aligned(dy, e) || !is_aligned(dtotal, f) || !is_aligned(dresidual, f) || !is_aligned(dx, e) ||
      !is_aligned(gain, 4) || !is_aligned(dgain, 4))
    return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  const auto rows = [&](const void* p, size_t size) { return span_of(p, c.rows, c.width, c.width, size); };
  if (!are_apart({rows(dresidual, f), rows(dx, e), {dgain, sizeof(float) * c.width}},
                 {rows(total, f), rows(dy, e), rows(dresidual && dtotal == dresidual ? nullptr : dtotal, f),
                  {gain, sizeof(float) * c.width}, {a.drop.step_dev, sizeof(uint64_t)}}))
    return set_error(SOMA_EINVAL, "an output overlaps another array");
  const int blocks = backward_blocks(c);
  if (dgain)
    if (int rc = check_workspace(workspace, ws_bytes, up256(sizeof(float) * blocks * c.width))) return rc;
  a.total = const_cast<void*>(total), a.gain = gain, a.dy = dy, a.dtotal = dtotal, a.dresidual = dresidual, a.dx = dx;
  a.partial = dgain ? static_cast<float*>(workspace) : nullptr;
  a.rows = c.rows, a.width = c.width, a.eps = c.eps;
  a.total_vec = in_eights(total, c.width, c.width, f), a.dy_vec = in_eights(dy, c.width, c.width, e);
  a.dtotal_vec = in_eights(dtotal, c.width, c.width, f);
  a.dresidual_vec = is_aligned(dresidual, 16), a.dx_vec = is_aligned(dx, 16);
  const hipStream_t st = stream_of(stream);
  if (int rc = by_type(c, [&](auto t, auto s) {
        return by_width<false>(c.width, [&](auto lanes, auto groups) {
          return backward_as<decltype(t), decltype(s), lanes(), groups()>(a, blocks, st);
        });
      }))
    return rc;
  if (dgain)
    if (int rc = launch("k_norm_gain", k_norm_gain, dim3((c.width + 63) / 64), dim3(1024), 0, st,
                        static_cast<const float*>(workspace), blocks, c.width, dgain))
      return rc;
  return set_ok();
}

}  // extern "C"
