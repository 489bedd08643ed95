// soma_scan.hip -- the gated linear recurrence: the LSTM's cell with gates that
// read the input alone,
//   c_t = s(f_t) c_{t-1} + s(i_t) tanh(g_t),   h_t = s(o_t) tanh(c_t),
// over packed sequences, forward and backward.
//
// With a_t = s(f_t), b_t = s(i_t) tanh(g_t) a run of rows is one affine map of
// the state in front of it, c -> A c + B, and maps of neighbouring runs
// compose: (A2, B2) after (A1, B1) is (A2 A1, A2 B1 + B2).  So time runs side by
// side.  A block takes 64 lanes of channels and walks over tiles of 64 rows (backward: 32): its 8
// waves hold 8 (4) rows each in registers, form the map of their rows, exchange the
// maps through LDS and start from the state that the earlier waves' maps give.
// The gates are read once; the next tile's are on their way meanwhile.  The
// state in front of every 64th row is kept for the backward pass, which forms the
// cells of a tile again from it (1/64 of a state array instead of a whole one).
//
// Backward, with u_t = dh_t s(o_t) (1 - tanh^2 c_t), the gradient of a cell is
// l_t = u_t + q_{t+1}, and what it passes on is q_t = s(f_t) l_t: the same affine
// maps from the last row to the first, q -> A q + B.
//
// Work is split by sequence and channels where that fills the card.  Else tiles are
// dealt out one by one, in order (a counter), to blocks that publish their tile's
// map, look back over the maps before it until they meet a state, publish the
// state behind their own tile, and write their rows: the gates are still read
// once, and a tile waits only for tiles that were dealt out earlier, so that some
// block can always go on.  Values travel between compute units as 32- and 64-bit
// words of agent scope that are their own flags (a word of ones: not there yet).
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
  // tiles dealt out one by one
  unsigned* ticket;         // the counter
  struct TileInfo* info;    // [tiles]
  uint64_t* maps;           // [tiles][H]
  uint32_t* tile_state;     // [tiles][H]: behind a tile, in the order in which they are dealt out
  int tile;                 // rows of one
  int tiles, groups;
};

// The sequence of a tile's first row, and that sequence's rows.
struct TileInfo {
  int s, first, to, pad;
};

__device__ __forceinline__ float sigmoid(float x) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kL2e * x));
}
// 1 - 2 / (1 + e^2x): fewer operations than the quotient of e^-2|x|, off by 2 u
// where tanh is small; e^2x = inf gives 1.
__device__ __forceinline__ float tanh_of(float x) {
  return __builtin_fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(2.0f * kL2e * x)), 1.0f);
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

  __device__ __forceinline__ void load(const Channels<VEC>& c, const Run& r, Raw& raw) const {
    const int row0 = (r.lo & ~(kTile - 1)) + wave * kRows;
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int row = row0 + u;
      if (c.on && row >= r.lo && row < r.hi) {
        const int64_t at = int64_t(row) * a.gate_stride + c.ch;
#pragma unroll
        for (int k = 0; k < 4; ++k) raw.g[k][u] = L::load(a.gates, at + int64_t(k) * a.H);
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
  }

  // The map of the whole run.
  __device__ __forceinline__ void whole_map(float (&A)[VEC], float (&B)[VEC]) const {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      A[v] = 1.0f, B[v] = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float2 m = x.m[buf][w][lane * VEC + v];
        A[v] *= m.x;
        B[v] = __builtin_fmaf(m.x, B[v], m.y);
      }
    }
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
          h[v] = sigmoid(L::get(raw.g[3][u], v)) * tanh_of(cell);
        }
        L::store(a.out, int64_t(row) * a.H + c.ch, h);
      }
    }
  }
};

// By sequence: a block walks over the tiles of one.
template <class T, int VEC>
__global__ __launch_bounds__(64 * kWaves) void k_scan_forward(ScanArgs a) {
  __shared__ Exchange<VEC> x;
  Forward<T, VEC> f(a, x, blockIdx.x);
  typedef typename Forward<T, VEC>::Raw Raw;
  const int s = blockIdx.y;
  const int lo = first_row(a, s), hi = clamp_row(first_row(a, s + 1), lo, a.rows);
  float state[VEC];
  load_state<VEC>(a.c0, s, a, f.c, state);
  if (lo < hi) {
    Run r{lo, min(hi, (lo & ~(kForward - 1)) + kForward)};
    Raw raw;
    f.load(f.c, r, raw);
    for (;;) {
      const Run next{r.hi, min(hi, r.hi + kForward)};
      Raw ahead;
      if (next.lo < hi) f.load(f.c, next, ahead);
      f.maps(r, raw);
      f.fold(r, state);
      f.rows_out(r, raw);
      if (next.lo >= hi) break;
      r = next;
      raw = ahead;
    }
  }
  if (f.wave == 0) store_state<VEC>(a.last, s, a, f.c, state);
}

// ---------------------------------------------------------------------------
// Tiles dealt out one by one.
// ---------------------------------------------------------------------------
constexpr uint32_t kNone = 0xFFFFFFFFu;       // not there yet
constexpr unsigned kPolls = 1u << 20;         // about a second; then the rows are NaN (no wait is without an end)

__device__ __forceinline__ uint32_t word_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return b == kNone ? 0x7FC00000u : b;        // that NaN in another form
}

template <int VEC>
__device__ __forceinline__ void publish_map(const ScanArgs& a, const Channels<VEC>& c, int tile, const float (&A)[VEC],
                                            const float (&B)[VEC]) {
  if (!c.on) return;
#pragma unroll
  for (int v = 0; v < VEC; ++v)
    __hip_atomic_store(a.maps + int64_t(tile) * a.H + c.ch + v, uint64_t(__float_as_uint(B[v])) << 32 | word_of(A[v]),
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int VEC>
__device__ __forceinline__ void publish_state(const ScanArgs& a, const Channels<VEC>& c, int tile, const float (&x)[VEC]) {
  if (!c.on) return;
#pragma unroll
  for (int v = 0; v < VEC; ++v)
    __hip_atomic_store(a.tile_state + int64_t(tile) * a.H + c.ch + v, word_of(x[v]), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}

// One wave: the state that the tiles from `tile` + kDir on bring, by way of their
// maps, four at a time.
template <int VEC, int kDir>
__device__ __forceinline__ void look_back(const ScanArgs& a, const Channels<VEC>& c, int tile, float (&state)[VEC]) {
  float A[VEC], B[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) A[v] = 1.0f, B[v] = 0.0f, state[v] = __builtin_nanf("");
  int q = tile + kDir;
  for (unsigned polls = 0; polls < kPolls;) {
    uint32_t st[4][VEC];
    uint64_t mp[4][VEC];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t at = int64_t(min(max(q + kDir * k, 0), a.tiles - 1)) * a.H + c.ch;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        st[k][v] = c.on ? __hip_atomic_load(a.tile_state + at + v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
        mp[k][v] = c.on ? __hip_atomic_load(a.maps + at + v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
      }
    }
    int used = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (used < k) break;                    // one before was not there
      const int at = q + kDir * k;
      if (at < 0 || at >= a.tiles) break;
      bool has_state = true, has_map = true;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        has_state = has_state && st[k][v] != kNone;
        has_map = has_map && static_cast<uint32_t>(mp[k][v]) != kNone;
      }
      if (__all(has_state)) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) state[v] = __builtin_fmaf(A[v], __uint_as_float(st[k][v]), B[v]);
        return;
      }
      if (!__all(has_map)) break;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        B[v] = __builtin_fmaf(A[v], __uint_as_float(static_cast<uint32_t>(mp[k][v] >> 32)), B[v]);
        A[v] *= __uint_as_float(static_cast<uint32_t>(mp[k][v]));
      }
      used = k + 1;
    }
    q += kDir * used;
    if (used == 0) {
      ++polls;
      __builtin_amdgcn_s_sleep(1);
    }
  }
}

// Clears the words and the counter, finds every tile's sequence, and copies the
// states of sequences without a row (from -> last).
__global__ __launch_bounds__(256) void k_scan_begin(ScanArgs a, const float* from) {
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x, n = int64_t(gridDim.x) * 256;
  const int64_t words = int64_t(a.tiles) * a.H;
  for (int64_t k = i; k < words; k += n) {
    a.maps[k] = ~uint64_t(0);
    a.tile_state[k] = kNone;
  }
  if (i == 0) *a.ticket = 0u;
  for (int64_t k = i; k < a.tiles; k += n) {
    const int s = sequence_of(a, static_cast<int>(k) * a.tile);
    a.info[k] = TileInfo{s, first_row(a, s), first_row(a, s + 1), 0};
  }
  if (a.last)
    for (int64_t k = i; k < int64_t(a.S) * a.H; k += n) {
      const int s = static_cast<int>(k / a.H);
      if (first_row(a, s + 1) <= first_row(a, s)) a.last[k] = from ? from[k] : 0.0f;
    }
}

// The tickets of a block: the tile that it works on, and the one after, whose
// rows are already on their way.
template <int kDir>
struct Tickets {
  const ScanArgs& a;
  unsigned* shared;           // [2]
  int items, par = 0;
  __device__ __forceinline__ Tickets(const ScanArgs& a_, unsigned* shared_)
      : a(a_), shared(shared_), items(a_.tiles * a_.groups) {}
  __device__ __forceinline__ void ask() {
    if (threadIdx.x == 0)
      shared[par] = __hip_atomic_fetch_add(a.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  // Behind a barrier.
  __device__ __forceinline__ int answer() {
    const unsigned t = __builtin_amdgcn_readfirstlane(shared[par]);
    par ^= 1;
    return t < static_cast<unsigned>(items) ? static_cast<int>(t) : items;
  }
  __device__ __forceinline__ int tile(int t) const {
    const int p = t / a.groups;
    return kDir < 0 ? p : a.tiles - 1 - p;
  }
  __device__ __forceinline__ int group(int t) const { return t % a.groups; }
};

template <class T, int VEC>
__global__ __launch_bounds__(64 * kWaves) void k_scan_forward_tiles(ScanArgs a) {
  __shared__ Exchange<VEC> x;
  __shared__ float carry[64 * VEC];
  __shared__ unsigned next[2];
  Forward<T, VEC> f(a, x, 0);
  typedef typename Forward<T, VEC>::Raw Raw;
  const int begin = first_row(a, 0), end = clamp_row(first_row(a, a.S), begin, a.rows);
  Tickets<-1> tickets(a, next);
  auto rows_of = [&](int t) {
    const int lo = tickets.tile(t) * kForward;
    return Run{max(lo, begin), min(lo + kForward, end)};
  };
  tickets.ask();
  __syncthreads();
  int t = tickets.answer();
  tickets.ask();
  __syncthreads();
  int after = tickets.answer();
  Raw raw;
  if (t < tickets.items) f.load(Channels<VEC>(a, tickets.group(t)), rows_of(t), raw);
  while (t < tickets.items) {
    Raw ahead;
    if (after < tickets.items) f.load(Channels<VEC>(a, tickets.group(after)), rows_of(after), ahead);
    tickets.ask();
    const int p = tickets.tile(t);
    const Run tile = rows_of(t);
    f.c = Channels<VEC>(a, tickets.group(t));
    if (tile.lo < tile.hi) {
      const TileInfo info = a.info[p];
      // The first run began in a tile before.  Every tile with rows publishes the
      // state behind its last, wanted or not: no offsets can make a tile wait for
      // one that has nothing to say.
      const bool continued = info.first < tile.lo && tile.lo > begin;
      // The runs that begin here, then the one that goes on from a tile before.
      int lo = continued ? min(info.to, tile.hi) : tile.lo;
      for (bool last = !continued && lo >= tile.hi; !last;) {
        const bool goes_on = lo >= tile.hi;
        const int s = goes_on || lo == tile.lo ? info.s : sequence_of(a, lo);
        const int to = goes_on ? info.to : max(first_row(a, s + 1), lo + 1);
        const Run r{goes_on ? tile.lo : lo, min(to, tile.hi)};
        last = goes_on || (!continued && r.hi >= tile.hi);
        lo = goes_on ? lo : r.hi;
        float state[VEC];
        // In front of maps' barrier: behind it a faster wave may write cT, which
        // may be c0.
        load_state<VEC>(goes_on ? nullptr : a.c0, s, a, f.c, state);
        f.maps(r, raw);
        if (goes_on) {
          if (f.wave == 0) {
            if (r.hi == tile.hi) {
              float A[VEC], B[VEC];
              f.whole_map(A, B);
              publish_map<VEC>(a, f.c, p, A, B);
            }
            look_back<VEC, -1>(a, f.c, p, state);
#pragma unroll
            for (int v = 0; v < VEC; ++v) carry[f.lane * VEC + v] = state[v];
          }
          __syncthreads();
#pragma unroll
          for (int v = 0; v < VEC; ++v) state[v] = carry[f.lane * VEC + v];
        }
        f.fold(r, state);
        if (f.wave == 0 && r.hi == tile.hi) publish_state<VEC>(a, f.c, p, state);
        f.rows_out(r, raw);
        if (f.wave == 0 && to == r.hi) store_state<VEC>(a.last, s, a, f.c, state);
      }
    }
    __syncthreads();
    raw = ahead;
    t = after;
    after = tickets.answer();
  }
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

  __device__ __forceinline__ void load(const Channels<VEC>& c, const Run& r, Raw& raw) const {
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
  __device__ __forceinline__ void entry_state(const Channels<VEC>& c, int lo, int s, int first, float (&x)[VEC]) const {
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
          g[u][v] = tanh_of(L::get(raw.g[2][u], v));
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
          const float t = tanh_of(s), o = sigmoid(L::get(raw.g[3][u], v)), dho = L::get(raw.g[4][u], v) * o;
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

  __device__ __forceinline__ void whole_map(float (&A)[VEC], float (&B)[VEC]) const {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      A[v] = 1.0f, B[v] = 0.0f;
#pragma unroll
      for (int w = kWaves - 1; w >= 0; --w) {
        const float2 m = y.m[buf][w][lane * VEC + v];
        A[v] *= m.x;
        B[v] = __builtin_fmaf(m.x, B[v], m.y);
      }
    }
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

template <class T, int VEC>
__global__ __launch_bounds__(64 * kWaves) void k_scan_backward(ScanArgs a) {
  __shared__ Exchange<VEC> x, y;
  Backward<T, VEC> b(a, x, y, blockIdx.x);
  typedef typename Backward<T, VEC>::Raw Raw;
  const int s = blockIdx.y;
  const int lo = first_row(a, s), hi = clamp_row(first_row(a, s + 1), lo, a.rows);
  float q[VEC];
  load_state<VEC>(a.dcT, s, a, b.c, q);
  if (lo < hi) {
    Run r{max(lo, (hi - 1) & ~(kBackward - 1)), hi};
    Raw raw;
    float entry[VEC];
    b.load(b.c, r, raw);
    b.entry_state(b.c, r.lo, s, lo, entry);
    for (;;) {
      const Run next{max(lo, r.lo - kBackward), r.lo};
      Raw ahead;
      float entry_ahead[VEC];
      if (next.hi > lo) {
        b.load(b.c, next, ahead);
        b.entry_state(b.c, next.lo, s, lo, entry_ahead);
      }
      b.maps(r, raw, entry);
      b.fold(q);
      b.rows_out(r);
      if (next.hi <= lo) break;
      r = next;
      raw = ahead;
#pragma unroll
      for (int v = 0; v < VEC; ++v) entry[v] = entry_ahead[v];
    }
  }
  if (b.wave == 0) store_state<VEC>(a.last, s, a, b.c, q);
}

template <class T, int VEC>
__global__ __launch_bounds__(64 * kWaves) void k_scan_backward_tiles(ScanArgs a) {
  __shared__ Exchange<VEC> x, y;
  __shared__ float carry[64 * VEC];
  __shared__ unsigned next[2];
  Backward<T, VEC> b(a, x, y, 0);
  typedef typename Backward<T, VEC>::Raw Raw;
  const int begin = first_row(a, 0), end = clamp_row(first_row(a, a.S), begin, a.rows);
  Tickets<1> tickets(a, next);
  auto rows_of = [&](int t) {
    const int lo = tickets.tile(t) * kBackward;
    return Run{max(lo, begin), min(lo + kBackward, end)};
  };
  tickets.ask();
  __syncthreads();
  int t = tickets.answer();
  tickets.ask();
  __syncthreads();
  int after = tickets.answer();
  Raw raw;
  if (t < tickets.items) b.load(Channels<VEC>(a, tickets.group(t)), rows_of(t), raw);
  while (t < tickets.items) {
    Raw ahead;
    if (after < tickets.items) b.load(Channels<VEC>(a, tickets.group(after)), rows_of(after), ahead);
    tickets.ask();
    const int p = tickets.tile(t);
    const Run tile = rows_of(t);
    b.c = Channels<VEC>(a, tickets.group(t));
    if (tile.lo < tile.hi) {
      const TileInfo info = a.info[p];
      // The runs from the first on; the last one may go on behind the tile.
      for (int lo = tile.lo; lo < tile.hi;) {
        const int s = lo == tile.lo ? info.s : sequence_of(a, lo);
        const int first = lo == tile.lo ? info.first : lo;
        const int to = max(first_row(a, s + 1), lo + 1);
        const Run r{lo, min(to, tile.hi)};
        const bool front = lo == tile.lo;                       // the tile before may wait for what this passes on
        float entry[VEC], q[VEC];
        const bool goes_on = to > r.hi && r.hi < end;           // the tile behind has rows, and publishes
        b.entry_state(b.c, lo, s, first, entry);
        // In front of maps' barriers: behind them a faster wave may write dc0,
        // which may be dcT.
        load_state<VEC>(goes_on ? nullptr : a.dcT, s, a, b.c, q);
        b.maps(r, raw, entry);
        if (goes_on) {
          if (b.wave == 0) {
            if (front) {
              float A[VEC], B[VEC];
              b.whole_map(A, B);
              publish_map<VEC>(a, b.c, p, A, B);
            }
            look_back<VEC, 1>(a, b.c, p, q);
#pragma unroll
            for (int v = 0; v < VEC; ++v) carry[b.lane * VEC + v] = q[v];
          }
          __syncthreads();
#pragma unroll
          for (int v = 0; v < VEC; ++v) q[v] = carry[b.lane * VEC + v];
        }
        b.fold(q);
        if (b.wave == 0 && front) publish_state<VEC>(a, b.c, p, q);
        b.rows_out(r);
        if (b.wave == 0 && first == lo) store_state<VEC>(a.last, s, a, b.c, q);
        lo = r.hi;
      }
    }
    __syncthreads();
    raw = ahead;
    t = after;
    after = tickets.answer();
  }
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
constexpr int64_t kTileBlocks = 512;      // blocks that work through the tiles: two a compute unit

int64_t tiles_of(const soma_scan_config& c, int tile) { return (int64_t(c.rows) + tile - 1) / tile; }

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

int vec_of(const soma_scan_config& c) { return c.type == SOMA_BFLOAT && c.width % 2 == 0 && c.gate_stride % 2 == 0 ? 2 : 1; }

int groups_of(const soma_scan_config& c, int vec) { return (c.width + 64 * vec - 1) / (64 * vec); }

// Whether tiles are dealt out one by one.  A block for every sequence and group of
// channels needs no words and no other launch, and is the better way where those
// blocks fill the card's 256 compute units, or where a sequence has a few hundred rows.
bool by_tiles(const soma_scan_config& c, int vec) {
  return int64_t(c.sequences) * groups_of(c, vec) < 256 && int64_t(c.rows) > 256 * int64_t(c.sequences);
}

size_t scan_workspace(const soma_scan_config& c) {
  const size_t tiles = size_t(tiles_of(c, kBackward)), words = tiles * c.width;
  return 256 + up256(tiles * sizeof(TileInfo)) + up256(words * 8) + up256(words * 4);
}

// The workspace's parts, cleared.  `from`: the states that empty sequences keep.
int begin_tiles(const soma_scan_config& c, int vec, int tile, void* ws, const float* from, ScanArgs* a, hipStream_t st) {
  char* at = static_cast<char*>(ws);
  const size_t tiles = size_t(tiles_of(c, tile)), words = tiles * c.width;
  a->tile = tile;
  a->tiles = int(tiles);
  a->groups = groups_of(c, vec);
  a->ticket = reinterpret_cast<unsigned*>(at);
  a->info = reinterpret_cast<TileInfo*>(at + 256);
  a->maps = reinterpret_cast<uint64_t*>(at + 256 + up256(tiles * sizeof(TileInfo)));
  a->tile_state = reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(a->maps) + up256(words * 8));
  const size_t blocks = std::min<size_t>((std::max(words, size_t(c.sequences) * c.width) + 255) / 256, 2048);
  hipLaunchKernelGGL(k_scan_begin, dim3(unsigned(blocks)), dim3(256), 0, st, *a, from);
  return launched("k_scan_begin");
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
  const dim3 block(64 * kWaves);
  const hipStream_t st = stream_of(stream);
  if (by_tiles(c, vec)) {
    if (int rc = begin_tiles(c, vec, kForward, workspace, c0, &a, st)) return rc;
    const dim3 grid(unsigned(std::min<int64_t>(int64_t(a.tiles) * a.groups, kTileBlocks)));
    if (c.type == SOMA_FLOAT)
      hipLaunchKernelGGL((k_scan_forward_tiles<float, 1>), grid, block, 0, st, a);
    else if (vec == 2)
      hipLaunchKernelGGL((k_scan_forward_tiles<bf16, 2>), grid, block, 0, st, a);
    else
      hipLaunchKernelGGL((k_scan_forward_tiles<bf16, 1>), grid, block, 0, st, a);
    if (int rc = launched("k_scan_forward_tiles")) return rc;
    return set_ok();
  }
  const dim3 grid(groups_of(c, vec), c.sequences);
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
  const dim3 block(64 * kWaves);
  const hipStream_t st = stream_of(stream);
  if (by_tiles(c, vec)) {
    if (int rc = begin_tiles(c, vec, kBackward, workspace, dcT, &a, st)) return rc;
    const dim3 grid(unsigned(std::min<int64_t>(int64_t(a.tiles) * a.groups, kTileBlocks)));
    if (c.type == SOMA_FLOAT)
      hipLaunchKernelGGL((k_scan_backward_tiles<float, 1>), grid, block, 0, st, a);
    else if (vec == 2)
      hipLaunchKernelGGL((k_scan_backward_tiles<bf16, 2>), grid, block, 0, st, a);
    else
      hipLaunchKernelGGL((k_scan_backward_tiles<bf16, 1>), grid, block, 0, st, a);
    if (int rc = launched("k_scan_backward_tiles")) return rc;
    return set_ok();
  }
  const dim3 grid(groups_of(c, vec), c.sequences);
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
