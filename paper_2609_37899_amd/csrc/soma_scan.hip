// soma_scan.hip -- the gated linear recurrence: the LSTM's cell with gates that
// read the input alone,
//   c_t = s(f_t) c_{t-1} + s(i_t) tanh(g_t),   h_t = s(o_t) tanh(c_t),
// over packed sequences, forward and backward.
//
// With a_t = s(f_t), b_t = s(i_t) tanh(g_t) a run of rows is one affine map of
// the state in front of it, c -> A c + B, and maps of neighbouring runs
// compose: (A2, B2) after (A1, B1) is (A2 A1, A2 B1 + B2).  So time runs side by
// side.  A block takes 64 lanes of channels and walks over tiles of 64 rows: its 8
// waves hold 8 rows each in registers, form the map of their rows, exchange the
// maps through LDS and start from the state that the earlier waves' maps give.
// The gates are read once; the next tile's are on their way meanwhile.  The
// state in front of every 64th row is kept for the backward pass, which forms the
// cells of a tile again from it (1/64 of a state array instead of a whole one).
//
// Backward, with u_t = dh_t s(o_t) (1 - tanh^2 c_t), the gradient of a cell is
// l_t = u_t + q_{t+1}, and what it passes on is q_t = s(f_t) l_t: the same affine
// maps from the last row to the first, q -> A q + B.
//
// Work is split by sequence and channels where that fills the card.  Else the
// rows are cut into pieces of whole tiles: a first launch forms the map of every
// piece, and each block of the second starts from the maps of the pieces in front
// of it.  That reads the gates twice (the second time largely from the last-level
// cache), and is bound by memory like the first way.
#include <hip/hip_runtime.h>

#include <cmath>

#include "soma.h"
#include "soma_host.hpp"
#include "soma_types.hpp"

namespace soma {
namespace {

constexpr int kTile = 64;             // rows of a tile: SOMA_SCAN_BLOCK
constexpr int kWaves = 8;
constexpr int kRows = kTile / kWaves; // rows of a wave
constexpr float kL2e = 1.4426950408889634f;
static_assert(kTile == SOMA_SCAN_BLOCK, "the states' spacing is part of the interface");

struct ScanArgs {
  const void* gates;
  int64_t gate_stride;      // elements between rows
  const void* dh;           // backward
  void* out;                // h [rows][H], or dgates [rows][4H]
  const int32_t* offsets;   // [S + 1], or NULL: `length` rows each
  const float* c0;          // [S][H] or NULL: zeros
  float* last;              // forward: cT [S][H]; backward: dc0 [S][H]; or NULL
  const float* dcT;         // backward: [S][H] or NULL: zeros
  float* states;            // [ceil(rows / 64)][H]: the state in front of row 64 j; or NULL
  float* start;             // pieces: c0 as it was (cT may be the same array), [S][H]
  float2* maps;             // pieces: [pieces][H]
  int rows, H, S, length;
  int piece;                // rows of a piece, a multiple of 64 (0: split by sequence)
};

// An affine map x -> a x + b of the state.  a < 0 marks a map that forgets x
// (a sequence starts inside): 0 * x would let another sequence's NaN through.
__device__ __forceinline__ float apply_map(float2 m, float x) {
  return m.x < 0.0f ? m.y : __builtin_fmaf(m.x, x, m.y);
}

__device__ __forceinline__ float sigmoid(float x) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kL2e * x));
}
__device__ __forceinline__ float tanh_of(float x) {
  const float e = __builtin_amdgcn_exp2f(-2.0f * kL2e * __builtin_fabsf(x));
  return __builtin_copysignf((1.0f - e) * __builtin_amdgcn_rcpf(1.0f + e), x);
}

// VEC neighbouring channels of a row as 32 bits (bf16 pair, fp32, or one bf16).
template <class T, int VEC>
struct Lane;
template <>
struct Lane<float, 1> {
  typedef float raw;
  static __device__ __forceinline__ raw load(const void* p, int64_t i) { return static_cast<const float*>(p)[i]; }
  static __device__ __forceinline__ float get(raw r, int) { return r; }
  static __device__ __forceinline__ void store(void* p, int64_t i, const float (&x)[1]) { static_cast<float*>(p)[i] = x[0]; }
};
template <>
struct Lane<bf16, 1> {
  typedef uint16_t raw;
  static __device__ __forceinline__ raw load(const void* p, int64_t i) { return static_cast<const uint16_t*>(p)[i]; }
  static __device__ __forceinline__ float get(raw r, int) { return from_bf16(r); }
  static __device__ __forceinline__ void store(void* p, int64_t i, const float (&x)[1]) {
    store_value(static_cast<bf16*>(p) + i, x[0]);
  }
};
template <>
struct Lane<bf16, 2> {
  typedef uint32_t raw;
  static __device__ __forceinline__ raw load(const void* p, int64_t i) {
    return *reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p) + i);
  }
  static __device__ __forceinline__ float get(raw r, int v) {
    return __uint_as_float(v ? r & 0xFFFF0000u : r << 16);
  }
  static __device__ __forceinline__ void store(void* p, int64_t i, const float (&x)[2]) {
    *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p) + i) = bf16_pair(x[0], x[1]);
  }
};

__device__ __forceinline__ int clamp_row(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// First row of sequence s (s = S: the end of the last), within [0, rows]
// whatever the offsets say.
__device__ __forceinline__ int first_row(const ScanArgs& a, int s) {
  if (!a.offsets) return s * a.length;
  return clamp_row(a.offsets[s], 0, a.rows);
}

// The sequence that row r belongs to: the last one that starts at or before it.
__device__ __forceinline__ int sequence_of(const ScanArgs& a, int r) {
  if (!a.offsets) return r / a.length;
  int lo = 0, hi = a.S - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (first_row(a, mid) <= r)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// This block's channels.
template <int VEC>
struct Channels {
  int ch;
  bool on;
  __device__ __forceinline__ explicit Channels(const ScanArgs& a)
      : ch((blockIdx.x * 64 + (threadIdx.x & 63)) * VEC), on(ch < a.H) {}
};

template <int VEC>
__device__ __forceinline__ void load_state(const float* p, int64_t row, const ScanArgs& a, const Channels<VEC>& c,
                                           float (&x)[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) x[v] = p && c.on ? p[row * a.H + c.ch + v] : 0.0f;
}
template <int VEC>
__device__ __forceinline__ void store_state(float* p, int64_t row, const ScanArgs& a, const Channels<VEC>& c,
                                            const float (&x)[VEC]) {
  if (p && c.on) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) p[row * a.H + c.ch + v] = x[v];
  }
}

// A run of rows of one sequence inside one tile.
struct Run {
  int lo, hi;      // rows lo .. hi - 1
  __device__ __forceinline__ int base() const { return lo & ~(kTile - 1); }
};

// The maps of a tile's waves, exchanged through LDS (two buffers in turn, so
// that one barrier a tile is enough).
template <int VEC>
struct Exchange {
  float2 m[2][kWaves][64 * VEC];
};

// ---------------------------------------------------------------------------
// Forward.  kMaps: only the map of the rows (piece mode's first launch).
// ---------------------------------------------------------------------------
template <class T, int VEC, bool kMaps>
struct Forward {
  typedef Lane<T, VEC> L;
  const ScanArgs& a;
  Channels<VEC> c;
  Exchange<VEC>& x;
  int wave, lane, buf = 0;

  __device__ __forceinline__ Forward(const ScanArgs& a_, Exchange<VEC>& x_)
      : a(a_), c(a_), x(x_), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), lane(threadIdx.x & 63) {}

  struct Raw {
    typename L::raw g[4][kRows];
  };

  __device__ __forceinline__ void load(const Run& r, Raw& raw) const {
    const int row0 = r.base() + wave * kRows;
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int row = row0 + u;
      if (c.on && row >= r.lo && row < r.hi) {
        const int64_t at = int64_t(row) * a.gate_stride + c.ch;
#pragma unroll
        for (int k = 0; k < (kMaps ? 3 : 4); ++k) raw.g[k][u] = L::load(a.gates, at + int64_t(k) * a.H);
      }
    }
  }

  // Advances the state (or, for kMaps, the map (A, state)) over a run.
  __device__ __forceinline__ void advance(const Run& r, const Raw& raw, float (&state)[VEC], float (&A)[VEC]) {
    const int row0 = r.base() + wave * kRows;
    float pa[kRows][VEC], pb[kRows][VEC];     // the map of the wave's rows up to each
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float ma = 1.0f, mb = 0.0f;
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int row = row0 + u;
        if (row >= r.lo && row < r.hi) {      // wave-uniform
          const float fa = sigmoid(L::get(raw.g[1][u], v));
          const float b = sigmoid(L::get(raw.g[0][u], v)) * tanh_of(L::get(raw.g[2][u], v));
          ma *= fa;
          mb = __builtin_fmaf(fa, mb, b);
        }
        pa[u][v] = ma;
        pb[u][v] = mb;
      }
      x.m[buf][wave][lane * VEC + v] = make_float2(ma, mb);
    }
    __syncthreads();
    float in[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float s = state[v];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        if (w == wave) in[v] = s;
        const float2 m = x.m[buf][w][lane * VEC + v];
        s = __builtin_fmaf(m.x, s, m.y);
        if constexpr (kMaps) A[v] = A[v] < 0.0f ? A[v] : A[v] * m.x;
      }
      state[v] = s;
    }
    buf ^= 1;
    if constexpr (!kMaps) {
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int row = row0 + u;
        if (c.on && row >= r.lo && row < r.hi) {
          float h[VEC];
#pragma unroll
          for (int v = 0; v < VEC; ++v) {
            const float cell = __builtin_fmaf(pa[u][v], in[v], pb[u][v]);
            h[v] = sigmoid(L::get(raw.g[3][u], v)) * tanh_of(cell);
          }
          L::store(a.out, int64_t(row) * a.H + c.ch, h);
        }
      }
    }
  }
};

// Rows [lo, hi) of sequence s from `state`, which is left as the state behind
// them.  (kMaps: A is the map's factor.)
template <class T, int VEC, bool kMaps>
__device__ __forceinline__ void forward_rows(Forward<T, VEC, kMaps>& f, int lo, int hi, float (&state)[VEC],
                                             float (&A)[VEC]) {
  typedef typename Forward<T, VEC, kMaps>::Raw Raw;
  if (lo >= hi) return;
  Run r{lo, min(hi, (lo & ~(kTile - 1)) + kTile)};
  Raw raw;
  f.load(r, raw);
  for (;;) {
    const Run next{r.hi, min(hi, r.hi + kTile)};
    Raw ahead;
    if (next.lo < hi) f.load(next, ahead);
    if constexpr (!kMaps)
      if (f.wave == 0 && (r.lo & (kTile - 1)) == 0) store_state<VEC>(f.a.states, r.lo / kTile, f.a, f.c, state);
    f.advance(r, raw, state, A);
    if (next.lo >= hi) break;
    r = next;
    raw = ahead;
  }
}

template <class T, int VEC>
__global__ __launch_bounds__(64 * kWaves) void k_scan_forward(ScanArgs a) {
  __shared__ Exchange<VEC> x;
  Forward<T, VEC, false> f(a, x);
  float state[VEC], unused[VEC];
  if (a.piece == 0) {
    const int s = blockIdx.y;
    const int lo = first_row(a, s), hi = clamp_row(first_row(a, s + 1), lo, a.rows);
    load_state<VEC>(a.c0, s, a, f.c, state);
    forward_rows(f, lo, hi, state, unused);
    if (f.wave == 0) store_state<VEC>(a.last, s, a, f.c, state);
    return;
  }
  // Rows [lo, hi) of all sequences together.
  const int p = blockIdx.y, begin = first_row(a, 0), end = clamp_row(first_row(a, a.S), begin, a.rows);
  int lo = max(p * a.piece, begin);
  const int hi = static_cast<int>(min(int64_t(p + 1) * a.piece, int64_t(end)));
  if (p == 0 && f.wave == 0 && a.last)        // sequences without a row keep their state
    for (int s = 0; s < a.S; ++s)
      if (first_row(a, s + 1) <= first_row(a, s)) {
        load_state<VEC>(a.start, s, a, f.c, state);
        store_state<VEC>(a.last, s, a, f.c, state);
      }
  if (lo >= hi) return;
  int s = sequence_of(a, lo);
  if (first_row(a, s) == lo) {
    load_state<VEC>(a.start, s, a, f.c, state);
  } else {
#pragma unroll
    for (int v = 0; v < VEC; ++v) state[v] = 0.0f;
    for (int q = 0; q < p; ++q)
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        if (f.c.on) state[v] = apply_map(a.maps[int64_t(q) * a.H + f.c.ch + v], state[v]);
  }
  for (;;) {
    const int to = clamp_row(first_row(a, s + 1), lo, hi);
    forward_rows(f, lo, to, state, unused);
    if (f.wave == 0 && to == first_row(a, s + 1) && to > first_row(a, s)) store_state<VEC>(a.last, s, a, f.c, state);
    lo = to;
    if (lo >= hi || s + 1 >= a.S) break;
    ++s;
    if (first_row(a, s) == lo && first_row(a, s + 1) > lo) load_state<VEC>(a.start, s, a, f.c, state);
  }
}

// Piece mode's first launch: the map of every piece's rows, and the initial
// states as they are now (the second launch may overwrite them with the last).
template <class T, int VEC>
__global__ __launch_bounds__(64 * kWaves) void k_scan_forward_maps(ScanArgs a) {
  __shared__ Exchange<VEC> x;
  Forward<T, VEC, true> f(a, x);
  float state[VEC], A[VEC];
  const int p = blockIdx.y, begin = first_row(a, 0), end = clamp_row(first_row(a, a.S), begin, a.rows);
  if (f.wave == 0)
    for (int s = p; s < a.S; s += gridDim.y) {
      load_state<VEC>(a.c0, s, a, f.c, state);
      store_state<VEC>(a.start, s, a, f.c, state);
    }
  const int lo = max(p * a.piece, begin);
  const int hi = static_cast<int>(min(int64_t(p + 1) * a.piece, int64_t(end)));
#pragma unroll
  for (int v = 0; v < VEC; ++v) A[v] = 1.0f, state[v] = 0.0f;
  if (lo < hi) {
    // Only the rows from the last start on matter.
    const int s = sequence_of(a, hi - 1), from = first_row(a, s);
    if (from >= lo) {
      load_state<VEC>(a.c0, s, a, f.c, state);
#pragma unroll
      for (int v = 0; v < VEC; ++v) A[v] = -1.0f;
    }
    forward_rows(f, max(lo, from), hi, state, A);
  }
  if (f.wave == 0 && f.c.on)
#pragma unroll
    for (int v = 0; v < VEC; ++v) a.maps[int64_t(p) * a.H + f.c.ch + v] = make_float2(A[v], state[v]);
}

// ---------------------------------------------------------------------------
// Backward.
// ---------------------------------------------------------------------------
template <class T, int VEC, bool kMaps>
struct Backward {
  typedef Lane<T, VEC> L;
  const ScanArgs& a;
  Channels<VEC> c;
  Exchange<VEC>&x, &y;
  int wave, lane, buf = 0;

  __device__ __forceinline__ Backward(const ScanArgs& a_, Exchange<VEC>& x_, Exchange<VEC>& y_)
      : a(a_), c(a_), x(x_), y(y_), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), lane(threadIdx.x & 63) {}

  struct Raw {
    typename L::raw g[5][kRows];
    float entry[VEC];      // the state in front of the run
  };

  __device__ __forceinline__ void load(const Run& r, int s, int first, Raw& raw) const {
    const int row0 = r.base() + wave * kRows;
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int row = row0 + u;
      if (c.on && row >= r.lo && row < r.hi) {
        const int64_t at = int64_t(row) * a.gate_stride + c.ch;
#pragma unroll
        for (int k = 0; k < 4; ++k) raw.g[k][u] = L::load(a.gates, at + int64_t(k) * a.H);
        raw.g[4][u] = L::load(a.dh, int64_t(row) * a.H + c.ch);
      }
    }
    if (r.lo == first)
      load_state<VEC>(a.c0, s, a, c, raw.entry);
    else
      load_state<VEC>(a.states, r.lo / kTile, a, c, raw.entry);
  }

  // From q = the gradient that the rows behind pass on to the one that this
  // run passes on (or, for kMaps, the map (A, q)).
  __device__ __forceinline__ void advance(const Run& r, const Raw& raw, float (&q)[VEC], float (&A)[VEC]) {
    const int row0 = r.base() + wave * kRows;
    float f[kRows][VEC], cell[kRows][VEC], before[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float ma = 1.0f, mb = 0.0f;
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int row = row0 + u;
        if (row >= r.lo && row < r.hi) {
          f[u][v] = sigmoid(L::get(raw.g[1][u], v));
          cell[u][v] = sigmoid(L::get(raw.g[0][u], v)) * tanh_of(L::get(raw.g[2][u], v));
          ma *= f[u][v];
          mb = __builtin_fmaf(f[u][v], mb, cell[u][v]);
        }
      }
      x.m[buf][wave][lane * VEC + v] = make_float2(ma, mb);
    }
    __syncthreads();
    float pq[kRows][VEC];                  // q in front of each row, from 0 behind the wave's last
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float s = raw.entry[v];
#pragma unroll
      for (int w = 0; w < kWaves - 1; ++w)
        if (w < wave) {
          const float2 m = x.m[buf][w][lane * VEC + v];
          s = __builtin_fmaf(m.x, s, m.y);
        }
      before[v] = s;
      float u_of[kRows];
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int row = row0 + u;
        if (row >= r.lo && row < r.hi) {
          s = __builtin_fmaf(f[u][v], s, cell[u][v]);
          cell[u][v] = s;
          const float t = tanh_of(s);
          u_of[u] = L::get(raw.g[4][u], v) * sigmoid(L::get(raw.g[3][u], v)) * (1.0f - t * t);
        }
      }
      float ma = 1.0f, mb = 0.0f;
#pragma unroll
      for (int u = kRows - 1; u >= 0; --u) {
        const int row = row0 + u;
        pq[u][v] = 0.0f;
        if (row >= r.lo && row < r.hi) {
          pq[u][v] = mb + u_of[u];         // l of the row, without what comes from behind the wave
          mb = f[u][v] * pq[u][v];
          ma *= f[u][v];
        }
      }
      y.m[buf][wave][lane * VEC + v] = make_float2(ma, mb);
    }
    __syncthreads();
    float in[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float s = q[v];
#pragma unroll
      for (int w = kWaves - 1; w >= 0; --w) {
        if (w == wave) in[v] = s;
        const float2 m = y.m[buf][w][lane * VEC + v];
        s = __builtin_fmaf(m.x, s, m.y);
        if constexpr (kMaps) A[v] = A[v] < 0.0f ? A[v] : A[v] * m.x;
      }
      q[v] = s;
    }
    buf ^= 1;
    if constexpr (!kMaps) {
      float fac[VEC];                      // product of the f of the rows behind
#pragma unroll
      for (int v = 0; v < VEC; ++v) fac[v] = in[v];
#pragma unroll
      for (int u = kRows - 1; u >= 0; --u) {
        const int row = row0 + u;
        if (row >= r.lo && row < r.hi) {
          float d[4][VEC];
#pragma unroll
          for (int v = 0; v < VEC; ++v) {
            const float l = pq[u][v] + fac[v];
            fac[v] *= f[u][v];
            const float i = sigmoid(L::get(raw.g[0][u], v)), g = tanh_of(L::get(raw.g[2][u], v));
            const float o = sigmoid(L::get(raw.g[3][u], v)), t = tanh_of(cell[u][v]);
            const float prev = u > 0 && row > r.lo ? cell[u > 0 ? u - 1 : 0][v] : before[v];
            d[0][v] = l * g * (i * (1.0f - i));
            d[1][v] = l * prev * (f[u][v] * (1.0f - f[u][v]));
            d[2][v] = l * i * (1.0f - g * g);
            d[3][v] = L::get(raw.g[4][u], v) * t * (o * (1.0f - o));
          }
          if (c.on) {
            const int64_t at = int64_t(row) * 4 * a.H + c.ch;
#pragma unroll
            for (int k = 0; k < 4; ++k) L::store(a.out, at + int64_t(k) * a.H, d[k]);
          }
        }
      }
    }
  }
};

// Rows [lo, hi) of sequence s (which starts at row `first`), last to first.
template <class T, int VEC, bool kMaps>
__device__ __forceinline__ void backward_rows(Backward<T, VEC, kMaps>& b, int lo, int hi, int s, int first,
                                              float (&q)[VEC], float (&A)[VEC]) {
  typedef typename Backward<T, VEC, kMaps>::Raw Raw;
  if (lo >= hi) return;
  Run r{max(lo, (hi - 1) & ~(kTile - 1)), hi};
  Raw raw;
  b.load(r, s, first, raw);
  for (;;) {
    const Run next{max(lo, r.lo - kTile), r.lo};
    Raw ahead;
    if (next.hi > lo) b.load(next, s, first, ahead);
    b.advance(r, raw, q, A);
    if (next.hi <= lo) break;
    r = next;
    raw = ahead;
  }
}

template <class T, int VEC>
__global__ __launch_bounds__(64 * kWaves) void k_scan_backward(ScanArgs a) {
  __shared__ Exchange<VEC> x, y;
  Backward<T, VEC, false> b(a, x, y);
  float q[VEC], unused[VEC];
  if (a.piece == 0) {
    const int s = blockIdx.y;
    const int lo = first_row(a, s), hi = clamp_row(first_row(a, s + 1), lo, a.rows);
    load_state<VEC>(a.dcT, s, a, b.c, q);
    backward_rows(b, lo, hi, s, lo, q, unused);
    if (b.wave == 0) store_state<VEC>(a.last, s, a, b.c, q);
    return;
  }
  const int p = blockIdx.y, begin = first_row(a, 0), end = clamp_row(first_row(a, a.S), begin, a.rows);
  const int lo = max(p * a.piece, begin);
  int hi = static_cast<int>(min(int64_t(p + 1) * a.piece, int64_t(end)));
  if (p == 0 && b.wave == 0 && a.last)
    for (int s = 0; s < a.S; ++s)
      if (first_row(a, s + 1) <= first_row(a, s)) {
        load_state<VEC>(a.start, s, a, b.c, q);
        store_state<VEC>(a.last, s, a, b.c, q);
      }
  if (lo >= hi) return;
  int s = sequence_of(a, hi - 1);
  if (first_row(a, s + 1) == hi) {
    load_state<VEC>(a.start, s, a, b.c, q);
  } else {
#pragma unroll
    for (int v = 0; v < VEC; ++v) q[v] = 0.0f;
    for (int n = static_cast<int>(gridDim.y) - 1; n > p; --n)
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        if (b.c.on) q[v] = apply_map(a.maps[int64_t(n) * a.H + b.c.ch + v], q[v]);
  }
  for (;;) {
    const int first = first_row(a, s), from = max(first, lo);
    backward_rows(b, from, hi, s, first, q, unused);
    if (b.wave == 0 && from == first && from < hi) store_state<VEC>(a.last, s, a, b.c, q);
    hi = from;
    if (hi <= lo) break;
    s = sequence_of(a, hi - 1);
    load_state<VEC>(a.start, s, a, b.c, q);
  }
}

template <class T, int VEC>
__global__ __launch_bounds__(64 * kWaves) void k_scan_backward_maps(ScanArgs a) {
  __shared__ Exchange<VEC> x, y;
  Backward<T, VEC, true> b(a, x, y);
  float q[VEC], A[VEC];
  const int p = blockIdx.y, begin = first_row(a, 0), end = clamp_row(first_row(a, a.S), begin, a.rows);
  if (b.wave == 0)
    for (int s = p; s < a.S; s += gridDim.y) {
      load_state<VEC>(a.dcT, s, a, b.c, q);
      store_state<VEC>(a.start, s, a, b.c, q);
    }
  const int lo = max(p * a.piece, begin);
  const int hi = static_cast<int>(min(int64_t(p + 1) * a.piece, int64_t(end)));
#pragma unroll
  for (int v = 0; v < VEC; ++v) A[v] = 1.0f, q[v] = 0.0f;
  if (lo < hi) {
    // Only the rows up to the end of the sequence that the piece begins in
    // matter to the pieces in front of it.
    const int s = sequence_of(a, lo), first = first_row(a, s), to = first_row(a, s + 1);
    if (first == lo) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) A[v] = -1.0f;   // nothing is passed on
    } else {
      if (to <= hi) {
        load_state<VEC>(a.dcT, s, a, b.c, q);
#pragma unroll
        for (int v = 0; v < VEC; ++v) A[v] = -1.0f;
      }
      backward_rows(b, lo, min(hi, to), s, first, q, A);
    }
  }
  if (b.wave == 0 && b.c.on)
#pragma unroll
    for (int v = 0; v < VEC; ++v) a.maps[int64_t(p) * a.H + b.c.ch + v] = make_float2(A[v], q[v]);
}

// ---------------------------------------------------------------------------
// One row for every sequence: a cell each, nothing to scan.
// ---------------------------------------------------------------------------
template <class T>
__global__ __launch_bounds__(256) void k_scan_step(const T* gates, int64_t gate_stride, const float* c0, float* cT, T* h,
                                                   int H) {
  const int ch = blockIdx.x * 256 + threadIdx.x;
  if (ch >= H) return;
  const T* g = gates + blockIdx.y * gate_stride + ch;
  const int64_t i = int64_t(blockIdx.y) * H + ch;
  const float gi = load_value(g), gf = load_value(g + H), gg = load_value(g + 2 * int64_t(H)),
              go = load_value(g + 3 * int64_t(H));
  const float c = __builtin_fmaf(sigmoid(gf), c0 ? c0[i] : 0.0f, sigmoid(gi) * tanh_of(gg));
  cT[i] = c;
  store_value(h + i, sigmoid(go) * tanh_of(c));
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
constexpr int kMostPieces = 256;

int check_shape(const soma_scan_config* c) {
  if (!c) return set_error(SOMA_EINVAL, "cfg is NULL");
  if (!is_type(c->type)) return set_error(SOMA_EINVAL, "unknown type %d", c->type);
  if (c->rows < 0 || c->rows > (1 << 30)) return set_error(SOMA_ESHAPE, "rows must be in [0, 2^30]");
  if (c->width < 1 || c->width > (1 << 20)) return set_error(SOMA_ESHAPE, "width must be in [1, 2^20]");
  if (c->sequences < 1 || c->sequences > 65535) return set_error(SOMA_ESHAPE, "sequences must be in [1, 65535]");
  if (c->gate_stride < 4 * int64_t(c->width) || c->gate_stride > (int64_t(1) << 32))
    return set_error(SOMA_ESHAPE, "gate_stride must be at least 4 width");
  return SOMA_OK;
}

int vec_of(const soma_scan_config& c) { return c.type == SOMA_BFLOAT && c.width % 2 == 0 && c.gate_stride % 2 == 0 ? 2 : 1; }

int groups_of(const soma_scan_config& c, int vec) { return (c.width + 64 * vec - 1) / (64 * vec); }

// Rows of a piece, or 0: split by sequence.  A block for every sequence and
// group of channels reads its gates once; it is the better way where those
// blocks fill the card's 256 compute units.  Below that the rows are cut into
// about 512 blocks' pieces, at least one tile each.
int piece_rows(const soma_scan_config& c, int vec) {
  const int groups = groups_of(c, vec);
  if (int64_t(c.sequences) * groups >= 256) return 0;
  const int64_t tiles = (int64_t(c.rows) + kTile - 1) / kTile;
  int64_t pieces = 512 / groups;
  pieces = pieces < 1 ? 1 : (pieces > kMostPieces ? kMostPieces : pieces);
  if (pieces <= c.sequences || tiles <= c.sequences) return 0;
  const int64_t each = (tiles + pieces - 1) / pieces;
  return static_cast<int>(each * kTile);
}

size_t scan_workspace(const soma_scan_config& c) {
  return up256(size_t(kMostPieces) * c.width * sizeof(float2)) + up256(size_t(c.sequences) * c.width * sizeof(float));
}

// The pieces' share of the arguments; returns the grid's second dimension.
int split(const soma_scan_config& c, int vec, void* ws, ScanArgs* a) {
  a->piece = piece_rows(c, vec);
  if (a->piece == 0) return c.sequences;
  a->maps = static_cast<float2*>(ws);
  a->start = reinterpret_cast<float*>(static_cast<char*>(ws) + up256(size_t(kMostPieces) * c.width * sizeof(float2)));
  return (c.rows + a->piece - 1) / a->piece;
}

int fill(const soma_scan_config& c, const void* gates, const int32_t* offsets, const float* c0, ScanArgs* a) {
  if (!offsets && c.rows % c.sequences)
    return set_error(SOMA_ESHAPE, "without offsets rows must be a multiple of sequences");
  if (!is_aligned(offsets, 4) || !is_aligned(c0, 4)) return set_error(SOMA_EINVAL, "misaligned pointer");
  a->gates = gates;
  a->gate_stride = c.gate_stride;
  a->offsets = offsets;
  a->c0 = c0;
  a->rows = c.rows;
  a->H = c.width;
  a->S = c.sequences;
  a->length = c.rows / c.sequences;
  if (!offsets && a->length == 0) a->length = 1;       // rows == 0: every sequence is empty (first_row is clamped)
  return SOMA_OK;
}

}  // namespace
}  // namespace soma

using namespace soma;

extern "C" {

int soma_scan_workspace_size(const soma_scan_config* cfg, size_t* bytes) {
  if (int rc = check_shape(cfg)) return rc;
  if (!bytes) return set_error(SOMA_EINVAL, "bytes is NULL");
  *bytes = scan_workspace(*cfg);
  return set_ok();
}

int soma_scan_forward(const soma_scan_config* cfg, const void* gates, const int32_t* offsets, const float* c0, void* h,
                      float* cT, float* states, void* workspace, size_t ws_bytes, void* stream) {
  if (int rc = check_shape(cfg)) return rc;
  const soma_scan_config& c = *cfg;
  const size_t e = type_size(c.type);
  if (c.rows > 0 && (!gates || !h)) return set_error(SOMA_EINVAL, "NULL device pointer");
  if (!is_aligned(gates, e) || !is_aligned(h, e) || !is_aligned(cT, 4) || !is_aligned(states, 4))
    return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  if (int rc = check_workspace(workspace, ws_bytes, scan_workspace(c))) return rc;
  ScanArgs a{};
  if (int rc = fill(c, gates, offsets, c0, &a)) return rc;
  a.out = h;
  a.last = cT;
  a.states = states;
  const int vec = vec_of(c) == 2 && is_aligned(gates, 4) && is_aligned(h, 4) ? 2 : 1;
  const dim3 grid(groups_of(c, vec), split(c, vec, workspace, &a)), block(64 * kWaves);
  const hipStream_t st = stream_of(stream);
  if (a.piece) {
    if (c.type == SOMA_FLOAT)
      hipLaunchKernelGGL((k_scan_forward_maps<float, 1>), grid, block, 0, st, a);
    else if (vec == 2)
      hipLaunchKernelGGL((k_scan_forward_maps<bf16, 2>), grid, block, 0, st, a);
    else
      hipLaunchKernelGGL((k_scan_forward_maps<bf16, 1>), grid, block, 0, st, a);
    if (int rc = launched("k_scan_forward_maps")) return rc;
  }
  if (c.type == SOMA_FLOAT)
    hipLaunchKernelGGL((k_scan_forward<float, 1>), grid, block, 0, st, a);
  else if (vec == 2)
    hipLaunchKernelGGL((k_scan_forward<bf16, 2>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((k_scan_forward<bf16, 1>), grid, block, 0, st, a);
  if (int rc = launched("k_scan_forward")) return rc;
  return set_ok();
}

int soma_scan_backward(const soma_scan_config* cfg, const void* gates, const int32_t* offsets, const float* c0,
                       const float* states, const void* dh, const float* dcT, void* dgates, float* dc0, void* workspace,
                       size_t ws_bytes, void* stream) {
  if (int rc = check_shape(cfg)) return rc;
  const soma_scan_config& c = *cfg;
  const size_t e = type_size(c.type);
  if (c.rows > 0 && (!gates || !dh || !dgates || !states)) return set_error(SOMA_EINVAL, "NULL device pointer");
  if (!is_aligned(gates, e) || !is_aligned(dh, e) || !is_aligned(dgates, e) || !is_aligned(dcT, 4) ||
      !is_aligned(dc0, 4) || !is_aligned(states, 4))
    return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  if (dgates == gates || (c.rows > 0 && dgates == dh)) return set_error(SOMA_EINVAL, "dgates must be an array of its own");
  if (int rc = check_workspace(workspace, ws_bytes, scan_workspace(c))) return rc;
  ScanArgs a{};
  if (int rc = fill(c, gates, offsets, c0, &a)) return rc;
  a.dh = dh;
  a.out = dgates;
  a.last = dc0;
  a.dcT = dcT;
  a.states = const_cast<float*>(states);
  const int vec =
      vec_of(c) == 2 && is_aligned(gates, 4) && is_aligned(dh, 4) && is_aligned(dgates, 4) ? 2 : 1;
  const dim3 grid(groups_of(c, vec), split(c, vec, workspace, &a)), block(64 * kWaves);
  const hipStream_t st = stream_of(stream);
  if (a.piece) {
    if (c.type == SOMA_FLOAT)
      hipLaunchKernelGGL((k_scan_backward_maps<float, 1>), grid, block, 0, st, a);
    else if (vec == 2)
      hipLaunchKernelGGL((k_scan_backward_maps<bf16, 2>), grid, block, 0, st, a);
    else
      hipLaunchKernelGGL((k_scan_backward_maps<bf16, 1>), grid, block, 0, st, a);
    if (int rc = launched("k_scan_backward_maps")) return rc;
  }
  if (c.type == SOMA_FLOAT)
    hipLaunchKernelGGL((k_scan_backward<float, 1>), grid, block, 0, st, a);
  else if (vec == 2)
    hipLaunchKernelGGL((k_scan_backward<bf16, 2>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((k_scan_backward<bf16, 1>), grid, block, 0, st, a);
  if (int rc = launched("k_scan_backward")) return rc;
  return set_ok();
}

int soma_scan_step(const soma_scan_config* cfg, const void* gates, const float* c0, float* cT, void* h, void* stream) {
  if (int rc = check_shape(cfg)) return rc;
  const soma_scan_config& c = *cfg;
  const size_t e = type_size(c.type);
  if (c.rows != c.sequences) return set_error(SOMA_ESHAPE, "a step takes one row for every sequence");
  if (!gates || !cT || !h) return set_error(SOMA_EINVAL, "NULL device pointer");
  if (!is_aligned(gates, e) || !is_aligned(h, e) || !is_aligned(cT, 4) || !is_aligned(c0, 4))
    return set_error(SOMA_EINVAL, "a pointer is not aligned to its elements");
  const dim3 grid((c.width + 255) / 256, c.sequences), block(256);
  if (c.type == SOMA_FLOAT)
    hipLaunchKernelGGL(k_scan_step<float>, grid, block, 0, stream_of(stream), static_cast<const float*>(gates),
                       c.gate_stride, c0, cT, static_cast<float*>(h), c.width);
  else
    hipLaunchKernelGGL(k_scan_step<bf16>, grid, block, 0, stream_of(stream), static_cast<const bf16*>(gates),
                       c.gate_stride, c0, cT, static_cast<bf16*>(h), c.width);
  if (int rc = launched("k_scan_step")) return rc;
  return set_ok();
}

}  // extern "C"
