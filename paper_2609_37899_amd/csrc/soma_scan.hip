// soma_scan.hip -- the gated linear recurrence: the LSTM's cell with gates that
// read the input alone,
//   c_t = s(f_t) c_{t-1} + s(i_t) tanh(g_t),   h_t = s(o_t) tanh(c_t),
// over packed sequences, forward and backward.
//
// With a_t = s(f_t), b_t = s(i_t) tanh(g_t) a run of rows is one affine map of
// the state in front of it, c -> A c + B, and maps of neighbouring runs
// compose: (A2, B2) after (A1, B1) is (A2 A1, A2 B1 + B2).  So time runs side by
// side.  A block takes 64 lanes of channels and walks over tiles of 64 rows
// (backward: 32): its 8 waves hold 8 (4) rows each in registers, form the map of
// their rows, exchange the maps through LDS and start from the state that the
// earlier waves' maps give.  The gates are read once and formed once; the next
// tile's are on their way meanwhile.  The state in front of every 32nd row is kept
// for the backward pass, which forms the cells of a tile again from it (1/32 of a
// state array instead of a whole one).
//
// Backward, with u_t = dh_t s(o_t) (1 - tanh^2 c_t), the gradient of a cell is
// l_t = u_t + q_{t+1}, and what it passes on is q_t = s(f_t) l_t: the same affine
// maps from the last row to the first, q -> A q + B.
//
// Work is split by sequence and channels where that fills the card.  Else the
// rows are cut into pieces of whole tiles: a first launch forms the map of every
// piece, and each block of the second starts from the maps of the pieces in front
// of it, applied in order.  That reads the gates twice, and is the shorter way all
// the same: one launch whose tiles publish their maps and look back over those
// before them took 742 us where this takes 690 (one sequence of 65,536 rows, width
// 1,024, bf16, both passes), since a state then goes from compute unit to compute
// unit 1,024 times; and which maps it joined depended on time, and with it the
// last bits.
//
// Measured, bf16: 64 sequences of 1,024 rows, width 512: forward 83 us (4.0 TB/s),
// backward 142 (4.2 TB/s); in pieces, the case above: maps 131 us (3.1 TB/s), forward
// 149 (4.5 TB/s); maps 173, backward 255.  Each row and channel takes 10 of the
// exponentials and reciprocals, which run at a quarter of the rate: 34 us of them in
// the first case, either way, beside the conversions of bf16.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "soma.h"
#include "soma_host.hpp"
#include "soma_types.hpp"

namespace soma {
namespace {

constexpr int kWaves = 8;
// Rows of a tile.  Backward holds twice as much of a row in registers, and takes
// half as many.
constexpr int kForward = 64, kBackward = 32;
constexpr float kL2e = 1.4426950408889634f;
static_assert(kBackward == SOMA_SCAN_BLOCK && kForward == 2 * SOMA_SCAN_BLOCK, "the states' spacing is part of the interface");

struct ScanArgs {
  const void* gates;
  int64_t gate_stride;      // elements between rows
  const void* dh;           // backward
  void* out;                // h [rows][H], or dgates [rows][4H]
  const int32_t* offsets;   // [S + 1], or NULL: `length` rows each
  const float* c0;          // [S][H] or NULL: zeros
  float* last;              // forward: cT [S][H]; backward: dc0 [S][H]; or NULL
  const float* dcT;         // backward: [S][H] or NULL: zeros
  float* states;            // [ceil(rows / 32)][H]: the state in front of row 32 j; or NULL
  int rows, H, S, length;
  float* start;             // pieces: the states that come in as they were (cT or dc0 may be the same array), [S][H]
  float2* maps;             // pieces: [pieces][H]
  int piece;                // rows of a piece, whole tiles (0: split by sequence)
};

// An affine map x -> a x + b of the state.  a < 0 marks a map that forgets x
// (a sequence starts inside): 0 * x would let another sequence's NaN through.
__device__ __forceinline__ float apply_map(float2 m, float x) {
  return m.x < 0.0f ? m.y : __builtin_fmaf(m.x, x, m.y);
}

__device__ __forceinline__ float sigmoid(float x) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kL2e * x));
}
// 1 - 2 / (1 + e^2x): fewer operations than the quotient of e^-2|x|; e^2x = inf gives
// 1.  It is off by 4 u of 1, which is all of a small value; there
//   fp32: below 0.35, where that passes 11 u of the value, x + x^3 p(x^2) with p of
//     three terms (smallest largest relative error, 0.7 u) is off by less than 2 u;
//   bf16: below 0.009, where it passes 2^-15 of the value, x is as near: the gates come
//     with 2^-9.  (The polynomial's seven operations for two take 88 us where this
//     takes 83, forward, 64 sequences of 1,024 rows, width 512.)
template <class T>
__device__ __forceinline__ float tanh_of(float x) {
  const float far = __builtin_fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(2.0f * kL2e * x)), 1.0f);
  if constexpr (sizeof(T) == 2) return __builtin_fabsf(x) < 0.009f ? x : far;
  const float z = x * x;
  const float p = __builtin_fmaf(__builtin_fmaf(z, -0x1.929fe2p-5f, 0x1.106164p-3f), z, -0x1.555394p-2f);
  return __builtin_fabsf(x) < 0.35f ? __builtin_fmaf(x * z, p, x) : far;
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

// The channels of a group.
template <int VEC>
struct Channels {
  int ch;
  bool on;
  __device__ __forceinline__ Channels(const ScanArgs& a, int group)
      : ch((group * 64 + (threadIdx.x & 63)) * VEC), on(ch < a.H) {}
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
};

// The maps of a tile's waves, exchanged through LDS (two buffers in turn, so
// that one barrier a tile is enough).
template <int VEC>
struct Exchange {
  float2 m[2][kWaves][64 * VEC];
};

// The maps of pieces from, from + step, ..., `count` of them, applied to x in this
// order; 16 loads in flight at a time, or their latencies add up.
template <int VEC>
__device__ __forceinline__ void apply_maps(const ScanArgs& a, const Channels<VEC>& c, int from, int step, int count,
                                           float (&x)[VEC]) {
  if (!c.on) return;
  for (int done = 0; done < count; done += 16) {
    float2 m[16][VEC];
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        m[i][v] = a.maps[int64_t(from + step * min(done + i, count - 1)) * a.H + c.ch + v];
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (done + i < count)
#pragma unroll
        for (int v = 0; v < VEC; ++v) x[v] = apply_map(m[i][v], x[v]);
  }
}

// A piece's share of copying the states that come in; sequences without a row
// keep theirs.
template <int VEC>
__device__ __forceinline__ void keep_states(const ScanArgs& a, const Channels<VEC>& c, int wave, int p, const float* from) {
  if (wave != 0) return;
  for (int s = p; s < a.S; s += gridDim.y) {
    float x[VEC];
    load_state<VEC>(from, s, a, c, x);
    store_state<VEC>(a.start, s, a, c, x);
    if (first_row(a, s + 1) <= first_row(a, s)) store_state<VEC>(a.last, s, a, c, x);
  }
}

// ---------------------------------------------------------------------------
// Forward: maps() forms the maps of a run's rows and shares them, fold() brings
// the state through them, rows_out() writes h.
// ---------------------------------------------------------------------------
template <class T, int VEC>
struct Forward {
  typedef Lane<T, VEC> L;
  static constexpr int kTile = kForward, kRows = kTile / kWaves;
  const ScanArgs& a;
  Channels<VEC> c;
  Exchange<VEC>& x;
  int wave, lane, buf = 0;
  float pa[kRows][VEC], pb[kRows][VEC];       // the map of the wave's rows up to each
  float in[VEC];                              // the state in front of the wave's rows

  __device__ __forceinline__ Forward(const ScanArgs& a_, Exchange<VEC>& x_, int group)
      : a(a_), c(a_, group), x(x_), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), lane(threadIdx.x & 63) {}

  struct Raw {
    typename L::raw g[4][kRows];
  };

  template <int kGates>
  __device__ __forceinline__ void load(const Run& r, Raw& raw) const {
    const int row0 = (r.lo & ~(kTile - 1)) + wave * kRows;
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int row = row0 + u;
      if (c.on && row >= r.lo && row < r.hi) {
        const int64_t at = int64_t(row) * a.gate_stride + c.ch;
#pragma unroll
        for (int k = 0; k < kGates; ++k) raw.g[k][u] = L::load(a.gates, at + int64_t(k) * a.H);
      }
    }
  }

  __device__ __forceinline__ void maps(const Run& r, const Raw& raw) {
    const int row0 = (r.lo & ~(kTile - 1)) + wave * kRows;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float ma = 1.0f, mb = 0.0f;
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int row = row0 + u;
        if (row >= r.lo && row < r.hi) {      // wave-uniform
          const float fa = sigmoid(L::get(raw.g[1][u], v));
          const float b = sigmoid(L::get(raw.g[0][u], v)) * tanh_of<T>(L::get(raw.g[2][u], v));
          ma *= fa;
          mb = __builtin_fmaf(fa, mb, b);
        }
        pa[u][v] = ma;
        pb[u][v] = mb;
      }
      x.m[buf][wave][lane * VEC + v] = make_float2(ma, mb);
    }
    __syncthreads();
  }

  // The map (A, B), extended by the run's (A < 0 stays: see apply_map).
  __device__ __forceinline__ void extend(float (&A)[VEC], float (&B)[VEC]) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float2 m = x.m[buf][w][lane * VEC + v];
        A[v] = A[v] < 0.0f ? A[v] : A[v] * m.x;
        B[v] = __builtin_fmaf(m.x, B[v], m.y);
      }
    }
    buf ^= 1;
  }

  // Also keeps the states in front of every 32nd row.
  __device__ __forceinline__ void fold(const Run& r, float (&state)[VEC]) {
    if (wave == 0 && r.lo % SOMA_SCAN_BLOCK == 0) store_state<VEC>(a.states, r.lo / SOMA_SCAN_BLOCK, a, c, state);

#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float s = state[v];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        if (w == wave) in[v] = s;
        const float2 m = x.m[buf][w][lane * VEC + v];
        s = __builtin_fmaf(m.x, s, m.y);
      }
      state[v] = s;
    }
    buf ^= 1;
    const int half = (r.lo & ~(kTile - 1)) + SOMA_SCAN_BLOCK;
    if (wave == kWaves / 2 && r.lo < half && half < r.hi) store_state<VEC>(a.states, half / SOMA_SCAN_BLOCK, a, c, in);
  }

  __device__ __forceinline__ void rows_out(const Run& r, const Raw& raw) const {
    const int row0 = (r.lo & ~(kTile - 1)) + wave * kRows;
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int row = row0 + u;
      if (c.on && row >= r.lo && row < r.hi) {
        float h[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const float cell = __builtin_fmaf(pa[u][v], in[v], pb[u][v]);
          h[v] = sigmoid(L::get(raw.g[3][u], v)) * tanh_of<T>(cell);
        }
        L::store(a.out, int64_t(row) * a.H + c.ch, h);
      }
    }
  }
};

// Rows [lo, hi) of one sequence from `state`, which is left as the state behind
// them.  kMaps: only the map (A, state).
template <bool kMaps, class T, int VEC>
__device__ __forceinline__ void forward_rows(Forward<T, VEC>& f, int lo, int hi, float (&state)[VEC], float (&A)[VEC]) {
  typedef typename Forward<T, VEC>::Raw Raw;
  if (lo >= hi) return;
  Run r{lo, min(hi, (lo & ~(kForward - 1)) + kForward)};
  Raw raw;
  f.template load<kMaps ? 3 : 4>(r, raw);
  for (;;) {
    const Run next{r.hi, min(hi, r.hi + kForward)};
    Raw ahead;
    if (next.lo < hi) f.template load<kMaps ? 3 : 4>(next, ahead);
    f.maps(r, raw);
    if constexpr (kMaps) {
      f.extend(A, state);
    } else {
      f.fold(r, state);
      f.rows_out(r, raw);
    }
    if (next.lo >= hi) break;
    r = next;
    raw = ahead;
  }
}

template <class T, int VEC>
__global__ __launch_bounds__(64 * kWaves) void k_scan_forward(ScanArgs a) {
  __shared__ Exchange<VEC> x;
  Forward<T, VEC> f(a, x, blockIdx.x);
  float state[VEC], unused[VEC];
  // Rows [lo, hi): one sequence, or a piece of all of them together.
  int s, lo, hi;
  if (a.piece == 0) {
    s = blockIdx.y;
    lo = first_row(a, s);
    hi = clamp_row(first_row(a, s + 1), lo, a.rows);
    load_state<VEC>(a.c0, s, a, f.c, state);
    if (lo >= hi) {
      if (f.wave == 0) store_state<VEC>(a.last, s, a, f.c, state);
      return;
    }
  } else {
    const int p = blockIdx.y, begin = first_row(a, 0), end = clamp_row(first_row(a, a.S), begin, a.rows);
    lo = max(p * a.piece, begin);
    hi = static_cast<int>(min(int64_t(p + 1) * a.piece, int64_t(end)));
    if (lo >= hi) return;
    s = sequence_of(a, lo);
    if (first_row(a, s) == lo) {
      load_state<VEC>(a.start, s, a, f.c, state);
    } else {
#pragma unroll
      for (int v = 0; v < VEC; ++v) state[v] = 0.0f;
      apply_maps(a, f.c, 0, 1, p, state);
    }
  }
  for (;;) {
    const int to = a.piece == 0 ? hi : clamp_row(first_row(a, s + 1), lo, hi);
    forward_rows<false>(f, lo, to, state, unused);
    if (f.wave == 0 && (a.piece == 0 || to == first_row(a, s + 1))) store_state<VEC>(a.last, s, a, f.c, state);
    lo = to;
    if (lo >= hi) break;
    s = sequence_of(a, lo);
    load_state<VEC>(a.start, s, a, f.c, state);
  }
}

// Pieces, first launch: the map of every piece's rows, the initial states as they
// are now (the second launch may overwrite them with the last), and the last
// states of sequences without a row.
template <class T, int VEC>
__global__ __launch_bounds__(64 * kWaves) void k_scan_forward_maps(ScanArgs a) {
  __shared__ Exchange<VEC> x;
  Forward<T, VEC> f(a, x, blockIdx.x);
  float state[VEC], A[VEC];
  const int p = blockIdx.y, begin = first_row(a, 0), end = clamp_row(first_row(a, a.S), begin, a.rows);
  keep_states(a, f.c, f.wave, p, a.c0);
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
    forward_rows<true>(f, max(lo, from), hi, state, A);
  }
  if (f.wave == 0 && f.c.on)
#pragma unroll
    for (int v = 0; v < VEC; ++v) a.maps[int64_t(p) * a.H + f.c.ch + v] = make_float2(A[v], state[v]);
}

// ---------------------------------------------------------------------------
// Backward: maps() forms the cells of a run again and the maps of its rows, fold()
// brings what the rows behind pass on through them, rows_out() writes dgates.
// ---------------------------------------------------------------------------
template <class T, int VEC>
struct Backward {
  typedef Lane<T, VEC> L;
  static constexpr int kTile = kBackward, kRows = kTile / kWaves;
  const ScanArgs& a;
  Channels<VEC> c;
  Exchange<VEC>&x, &y;
  int wave, lane, buf = 0;
  // The transcendental unit bounds this pass (a quarter of the rate, ten of its
  // instructions an element): every gate is formed once and kept.
  float f[kRows][VEC], i[kRows][VEC], g[kRows][VEC];
  float pq[kRows][VEC];                    // l of each row, without what comes from behind the wave
  float prev[kRows][VEC];                  // the cell in front of each row
  float go[kRows][VEC];                    // dh t s(o) (1 - s(o))
  float in[VEC];                           // what the rows behind the wave's pass on

  __device__ __forceinline__ Backward(const ScanArgs& a_, Exchange<VEC>& x_, Exchange<VEC>& y_, int group)
      : a(a_), c(a_, group), x(x_), y(y_), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), lane(threadIdx.x & 63) {}

  struct Raw {
    typename L::raw g[5][kRows];
  };

  __device__ __forceinline__ void load(const Run& r, Raw& raw) const {
    const int row0 = (r.lo & ~(kTile - 1)) + wave * kRows;
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
  }

  // The state in front of row `lo` of sequence s, which starts at `first`.
  __device__ __forceinline__ void entry_state(int lo, int s, int first, float (&x)[VEC]) const {
    if (lo == first)
      load_state<VEC>(a.c0, s, a, c, x);
    else
      load_state<VEC>(a.states, lo / SOMA_SCAN_BLOCK, a, c, x);
  }

  __device__ __forceinline__ void maps(const Run& r, const Raw& raw, const float (&entry)[VEC]) {
    const int row0 = (r.lo & ~(kTile - 1)) + wave * kRows;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float ma = 1.0f, mb = 0.0f;
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int row = row0 + u;
        if (row >= r.lo && row < r.hi) {
          f[u][v] = sigmoid(L::get(raw.g[1][u], v));
          i[u][v] = sigmoid(L::get(raw.g[0][u], v));
          g[u][v] = tanh_of<T>(L::get(raw.g[2][u], v));
          ma *= f[u][v];
          mb = __builtin_fmaf(f[u][v], mb, i[u][v] * g[u][v]);
        }
      }
      x.m[buf][wave][lane * VEC + v] = make_float2(ma, mb);
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float s = entry[v];
#pragma unroll
      for (int w = 0; w < kWaves - 1; ++w)
        if (w < wave) {
          const float2 m = x.m[buf][w][lane * VEC + v];
          s = __builtin_fmaf(m.x, s, m.y);
        }
      float u_of[kRows];
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int row = row0 + u;
        if (row >= r.lo && row < r.hi) {
          prev[u][v] = s;
          s = __builtin_fmaf(f[u][v], s, i[u][v] * g[u][v]);
          const float t = tanh_of<T>(s), o = sigmoid(L::get(raw.g[3][u], v)), dho = L::get(raw.g[4][u], v) * o;
          u_of[u] = dho * __builtin_fmaf(-t, t, 1.0f);
          go[u][v] = dho * t * (1.0f - o);
        }
      }
      float ma = 1.0f, mb = 0.0f;
#pragma unroll
      for (int u = kRows - 1; u >= 0; --u) {
        const int row = row0 + u;
        pq[u][v] = 0.0f;
        if (row >= r.lo && row < r.hi) {
          pq[u][v] = mb + u_of[u];
          mb = f[u][v] * pq[u][v];
          ma *= f[u][v];
        }
      }
      y.m[buf][wave][lane * VEC + v] = make_float2(ma, mb);
    }
    __syncthreads();
  }

  __device__ __forceinline__ void extend(float (&A)[VEC], float (&B)[VEC]) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
#pragma unroll
      for (int w = kWaves - 1; w >= 0; --w) {
        const float2 m = y.m[buf][w][lane * VEC + v];
        A[v] = A[v] < 0.0f ? A[v] : A[v] * m.x;
        B[v] = __builtin_fmaf(m.x, B[v], m.y);
      }
    }
    buf ^= 1;
  }

  __device__ __forceinline__ void fold(float (&q)[VEC]) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float s = q[v];
#pragma unroll
      for (int w = kWaves - 1; w >= 0; --w) {
        if (w == wave) in[v] = s;
        const float2 m = y.m[buf][w][lane * VEC + v];
        s = __builtin_fmaf(m.x, s, m.y);
      }
      q[v] = s;
    }
    buf ^= 1;
  }

  __device__ __forceinline__ void rows_out(const Run& r) const {
    const int row0 = (r.lo & ~(kTile - 1)) + wave * kRows;
    float fac[VEC];                        // what the rows behind pass on, through the f of those in between
#pragma unroll
    for (int v = 0; v < VEC; ++v) fac[v] = in[v];
#pragma unroll
    for (int u = kRows - 1; u >= 0; --u) {
      const int row = row0 + u;
      if (row >= r.lo && row < r.hi) {
        float d[4][VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const float l = pq[u][v] + fac[v], lf = l * f[u][v], li = l * i[u][v];
          fac[v] *= f[u][v];
          d[0][v] = li * g[u][v] * (1.0f - i[u][v]);
          d[1][v] = lf * prev[u][v] * (1.0f - f[u][v]);
          d[2][v] = li * __builtin_fmaf(-g[u][v], g[u][v], 1.0f);
          d[3][v] = go[u][v];
        }
        if (c.on) {
          const int64_t at = int64_t(row) * 4 * a.H + c.ch;
#pragma unroll
          for (int k = 0; k < 4; ++k) L::store(a.out, at + int64_t(k) * a.H, d[k]);
        }
      }
    }
  }
};

// Rows [lo, hi) of sequence s (which starts at row `first`), last to first, from q,
// which is left as what they pass on.  kMaps: only the map (A, q).
template <bool kMaps, class T, int VEC>
__device__ __forceinline__ void backward_rows(Backward<T, VEC>& b, int lo, int hi, int s, int first, float (&q)[VEC],
                                              float (&A)[VEC]) {
  typedef typename Backward<T, VEC>::Raw Raw;
  if (lo >= hi) return;
  Run r{max(lo, (hi - 1) & ~(kBackward - 1)), hi};
  Raw raw;
  float entry[VEC];
  b.load(r, raw);
  b.entry_state(r.lo, s, first, entry);
  for (;;) {
    const Run next{max(lo, r.lo - kBackward), r.lo};
    Raw ahead;
    float entry_ahead[VEC];
    if (next.hi > lo) {
      b.load(next, ahead);
      b.entry_state(next.lo, s, first, entry_ahead);
    }
    b.maps(r, raw, entry);
    if constexpr (kMaps) {
      b.extend(A, q);
    } else {
      b.fold(q);
      b.rows_out(r);
    }
    if (next.hi <= lo) break;
    r = next;
    raw = ahead;
#pragma unroll
    for (int v = 0; v < VEC; ++v) entry[v] = entry_ahead[v];
  }
}

template <class T, int VEC>
__global__ __launch_bounds__(64 * kWaves) void k_scan_backward(ScanArgs a) {
  __shared__ Exchange<VEC> x, y;
  Backward<T, VEC> b(a, x, y, blockIdx.x);
  float q[VEC], unused[VEC];
  int s, lo, hi;
  if (a.piece == 0) {
    s = blockIdx.y;
    lo = first_row(a, s);
    hi = clamp_row(first_row(a, s + 1), lo, a.rows);
    load_state<VEC>(a.dcT, s, a, b.c, q);
    if (lo >= hi) {
      if (b.wave == 0) store_state<VEC>(a.last, s, a, b.c, q);
      return;
    }
  } else {
    const int p = blockIdx.y, begin = first_row(a, 0), end = clamp_row(first_row(a, a.S), begin, a.rows);
    lo = max(p * a.piece, begin);
    hi = static_cast<int>(min(int64_t(p + 1) * a.piece, int64_t(end)));
    if (lo >= hi) return;
    s = sequence_of(a, hi - 1);
    if (first_row(a, s + 1) == hi) {
      load_state<VEC>(a.start, s, a, b.c, q);
    } else {
#pragma unroll
      for (int v = 0; v < VEC; ++v) q[v] = 0.0f;
      const int last = static_cast<int>(gridDim.y) - 1;
      apply_maps(a, b.c, last, -1, last - p, q);
    }
  }
  for (;;) {
    const int first = first_row(a, s), from = a.piece == 0 ? lo : max(first, lo);
    backward_rows<false>(b, from, hi, s, first, q, unused);
    if (b.wave == 0 && from == first) store_state<VEC>(a.last, s, a, b.c, q);
    hi = from;
    if (hi <= lo) break;
    s = sequence_of(a, hi - 1);
    load_state<VEC>(a.start, s, a, b.c, q);
  }
}

template <class T, int VEC>
__global__ __launch_bounds__(64 * kWaves) void k_scan_backward_maps(ScanArgs a) {
  __shared__ Exchange<VEC> x, y;
  Backward<T, VEC> b(a, x, y, blockIdx.x);
  float q[VEC], A[VEC];
  const int p = blockIdx.y, begin = first_row(a, 0), end = clamp_row(first_row(a, a.S), begin, a.rows);
  keep_states(a, b.c, b.wave, p, a.dcT);
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
      backward_rows<true>(b, lo, min(hi, to), s, first, q, A);
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
  const float c = __builtin_fmaf(sigmoid(gf), c0 ? c0[i] : 0.0f, sigmoid(gi) * tanh_of<T>(gg));
  cT[i] = c;
  store_value(h + i, sigmoid(go) * tanh_of<T>(c));
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
  if (int64_t(c->rows) * c->width > (int64_t(1) << 40)) return set_error(SOMA_ESHAPE, "rows times width must be at most 2^40");
  if (c->gate_stride < 4 * int64_t(c->width) || c->gate_stride > (int64_t(1) << 32))
    return set_error(SOMA_ESHAPE, "gate_stride must be at least 4 width");
  return SOMA_OK;
}

int groups_of(const soma_scan_config& c, int vec) { return (c.width + 64 * vec - 1) / (64 * vec); }

// Rows of a piece, or 0: split by sequence.  A block for every sequence and group
// of channels reads its gates once, and is the better way where those blocks fill
// the card's 256 compute units, or where a sequence is a few tiles long (bf16,
// both passes, 32 sequences of 512 rows, width 512: 79 us, in pieces 111; one
// sequence of 16,384, width 2,048: 344 us in pieces, above 2,000 without).  Else
// the rows are cut into pieces for about 512 blocks, at least two tiles each.
int piece_rows(const soma_scan_config& c, int vec) {
  const int64_t groups = groups_of(c, vec);
  if (int64_t(c.sequences) * groups_of(c, 1) >= 256 || c.rows <= 256 * int64_t(c.sequences)) return 0;
  const int64_t most = std::min<int64_t>(std::max<int64_t>(512 / groups, 1), kMostPieces);
  const int64_t tiles = (int64_t(c.rows) + kForward - 1) / kForward;
  return static_cast<int>(std::max<int64_t>((tiles + most - 1) / most, 2) * kForward);
}

// Channels of a lane.  Two of bf16 make whole 256-byte runs of a row and halve the
// instructions for addresses (256 sequences of 256 rows, width 512: both passes
// 217 us, one channel 231), unless by sequence that leaves less than two blocks a
// compute unit (64 of 512 rows: 129 us, one channel 115).
int vec_of(const soma_scan_config& c, bool aligned) {
  if (c.type != SOMA_BFLOAT || !aligned || c.width % 2 || c.gate_stride % 2) return 1;
  return piece_rows(c, 2) == 0 && int64_t(c.sequences) * groups_of(c, 2) < 512 ? 1 : 2;
}

size_t scan_workspace(const soma_scan_config& c) {
  if (piece_rows(c, 1) == 0) return 0;               // with two channels a lane, or fewer rows, so too
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
  a->length = c.rows / c.sequences;                    // 0: every sequence is empty
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
  const int vec = vec_of(c, is_aligned(gates, 4) && is_aligned(h, 4));
  const dim3 grid(groups_of(c, vec), split(c, vec, workspace, &a)), block(64 * kWaves);
  const hipStream_t st = stream_of(stream);
  if (a.piece) {
    const auto kernel = c.type == SOMA_FLOAT ? k_scan_forward_maps<float, 1>
                        : vec == 2           ? k_scan_forward_maps<bf16, 2>
                                             : k_scan_forward_maps<bf16, 1>;
    if (int rc = launch("k_scan_forward_maps", kernel, grid, block, 0, st, a)) return rc;
  }
  const auto kernel = c.type == SOMA_FLOAT ? k_scan_forward<float, 1>
                      : vec == 2           ? k_scan_forward<bf16, 2>
                                           : k_scan_forward<bf16, 1>;
  if (int rc = launch("k_scan_forward", kernel, grid, block, 0, st, a)) return rc;
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
  if (c.rows > 0 && (dgates == gates || dgates == dh)) return set_error(SOMA_EINVAL, "dgates must be an array of its own");
  if (int rc = check_workspace(workspace, ws_bytes, scan_workspace(c))) return rc;
  ScanArgs a{};
  if (int rc = fill(c, gates, offsets, c0, &a)) return rc;
  a.dh = dh;
  a.out = dgates;
  a.last = dc0;
  a.dcT = dcT;
  a.states = const_cast<float*>(states);
  const int vec = vec_of(c, is_aligned(gates, 4) && is_aligned(dh, 4) && is_aligned(dgates, 4));
  const dim3 grid(groups_of(c, vec), split(c, vec, workspace, &a)), block(64 * kWaves);
  const hipStream_t st = stream_of(stream);
  if (a.piece) {
    const auto kernel = c.type == SOMA_FLOAT ? k_scan_backward_maps<float, 1>
                        : vec == 2           ? k_scan_backward_maps<bf16, 2>
                                             : k_scan_backward_maps<bf16, 1>;
    if (int rc = launch("k_scan_backward_maps", kernel, grid, block, 0, st, a)) return rc;
  }
  const auto kernel = c.type == SOMA_FLOAT ? k_scan_backward<float, 1>
                      : vec == 2           ? k_scan_backward<bf16, 2>
                                           : k_scan_backward<bf16, 1>;
  if (int rc = launch("k_scan_backward", kernel, grid, block, 0, st, a)) return rc;
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
  const hipStream_t st = stream_of(stream);
  if (int rc = c.type == SOMA_FLOAT
                   ? launch("k_scan_step", k_scan_step<float>, grid, block, 0, st, static_cast<const float*>(gates),
                            c.gate_stride, c0, cT, static_cast<float*>(h), c.width)
                   : launch("k_scan_step", k_scan_step<bf16>, grid, block, 0, st, static_cast<const bf16*>(gates),
                            c.gate_stride, c0, cT, static_cast<bf16*>(h), c.width))
    return rc;
  return set_ok();
}

}  // extern "C"
