// soma_adamw.hip -- one AdamW step over many tensors in one launch.
//
//   g = scale * grad;  m <- beta1 m + (1 - beta1) g;  v <- beta2 v + (1 - beta2) g^2
//   p <- (1 - lr decay) p - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + delta)
//
// in fp32 whatever the tensors' types, one rounding for every operation (no
// contraction), p rounded once to its own type.
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
// The step is bound by memory: every element is read and written once.  A
// block takes 4096 consecutive elements of one tensor (a table of blocks, made
// once with the plan, names the tensor), a wave 256 of them at a time, four a
// lane: 16-byte accesses to fp32, and the 256 elements that share a scale are
// one wave's, whose two maxima never leave its registers.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "soma.h"
#include "soma_host.hpp"
#include "soma_types.hpp"

namespace soma {
namespace {

constexpr int kStateBlock = 256;      // elements that share the scales of 8-bit moments
constexpr int kChunk = 4096;          // elements of one block
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
  double lr;
};

// A block's scale from its largest magnitude, and the factor that brings its
// values onto the code's range (0 for a block of zeros, or one whose largest
// has no finite factor).
__device__ __forceinline__ float code_factor(float top, float largest) { return top > 1e-35f ? largest / top : 0.0f; }

__device__ __forceinline__ uint32_t root_code(float y) {
  const uint32_t b = __float_as_uint(y);
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

template <class P, class G, bool kBytes>
__device__ __forceinline__ void adamw_chunk(const Tensor& t, int64_t first, const Rates& r, float scale) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool wide = t.wide != 0;
  const float keep = static_cast<float>(1.0 - r.lr * t.decay);
  P* const param = static_cast<P*>(t.param);
#pragma unroll 2
  for (int k = 0; k < kRounds; ++k) {
    const int64_t block = first + (k * 4 + wave) * kStateBlock;   // the wave's 256 elements
    if (block >= t.count) break;                                  // wave-uniform
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
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[i] = m[i] * fm;
        vw |= root_code(root[i] * fr) << (8 * i);
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
}

__global__ __launch_bounds__(kThreadsAdamw) void k_adamw(const Tensor* tensors, const Block* blocks, Rates r,
                                                         const float* grad_scale) {
  const Block b = blocks[blockIdx.x];
  const Tensor t = tensors[b.tensor];
  const float scale = grad_scale ? *grad_scale : 1.0f;
  const int64_t first = int64_t(b.chunk) * kChunk;
  switch (t.kind) {
    case 0: adamw_chunk<float, float, false>(t, first, r, scale); break;
    case 1: adamw_chunk<float, float, true>(t, first, r, scale); break;
    case 2: adamw_chunk<float, bf16, false>(t, first, r, scale); break;
    case 3: adamw_chunk<float, bf16, true>(t, first, r, scale); break;
    case 4: adamw_chunk<bf16, float, false>(t, first, r, scale); break;
    case 5: adamw_chunk<bf16, float, true>(t, first, r, scale); break;
    case 6: adamw_chunk<bf16, bf16, false>(t, first, r, scale); break;
    default: adamw_chunk<bf16, bf16, true>(t, first, r, scale); break;
  }
}

// The moments' values, in fp32.  The outputs' addresses travel with the
// launch, kOutputs tensors at a time.
constexpr int kOutputs = 200;
struct Outputs {
  float *m[kOutputs], *v[kOutputs];
};

__global__ __launch_bounds__(kThreadsAdamw) void k_adamw_moments(const Tensor* tensors, const Block* blocks, int first_tensor,
                                                                 Outputs out) {
  const Block b = blocks[blockIdx.x];
  const Tensor t = tensors[b.tensor];
  float* const mo = out.m[b.tensor - first_tensor];
  float* const vo = out.v[b.tensor - first_tensor];
  const bool wide = t.wide && reinterpret_cast<uintptr_t>(mo) % 16 == 0 && reinterpret_cast<uintptr_t>(vo) % 16 == 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 2
  for (int k = 0; k < kRounds; ++k) {
    const int64_t block = int64_t(b.chunk) * kChunk + (k * 4 + wave) * kStateBlock;
    if (block >= t.count) break;
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

int64_t chunks_of(int64_t count) { return (count + kChunk - 1) / kChunk; }

int check_tensors(const soma_adamw_tensor* x, int32_t n, int64_t* chunks) {
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
    *chunks += chunks_of(t.count);
  }
  if (*chunks > (int64_t(1) << 30)) return set_error(SOMA_ESHAPE, "more than 2^42 elements");
  return SOMA_OK;
}

size_t table_bytes(int32_t n) { return up256(size_t(n) * sizeof(Tensor)); }

}  // namespace
}  // namespace soma

struct soma_adamw {
  int32_t n;
  int64_t chunks;
  const soma::Tensor* tensors;       // device
  const soma::Block* blocks;         // device
  int64_t* first_chunk;              // host, [n + 1]
};

using namespace soma;

extern "C" {

int soma_adamw_workspace_size(const soma_adamw_tensor* tensors, int32_t n, size_t* bytes) {
  int64_t chunks = 0;
  if (int rc = check_tensors(tensors, n, &chunks)) return rc;
  if (!bytes) return set_error(SOMA_EINVAL, "bytes is NULL");
  *bytes = table_bytes(n) + up256(size_t(chunks) * sizeof(Block));
  return set_ok();
}

int soma_adamw_create(const soma_adamw_tensor* tensors, int32_t n, void* workspace, size_t ws_bytes, void* stream,
                      soma_adamw** out) {
  int64_t chunks = 0;
  if (int rc = check_tensors(tensors, n, &chunks)) return rc;
  if (!out) return set_error(SOMA_EINVAL, "out is NULL");
  const size_t need = table_bytes(n) + up256(size_t(chunks) * sizeof(Block));
  if (int rc = check_workspace(workspace, ws_bytes, need)) return rc;
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
    for (int64_t c = 0; c < chunks_of(x.count); ++c) bb[at++] = Block{i, int32_t(c)};
  }
  first[n] = at;
  const hipStream_t st = stream_of(stream);
  hipError_t e = hipMemcpyAsync(workspace, host, need, hipMemcpyHostToDevice, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  delete[] host;
  if (e != hipSuccess) {
    delete[] first;
    delete plan;
    return set_error(SOMA_EDEVICE, "copying the tensors' table: %s", hipGetErrorString(e));
  }
  *plan = soma_adamw{n, chunks, static_cast<const Tensor*>(workspace),
                     reinterpret_cast<const Block*>(static_cast<char*>(workspace) + table_bytes(n)), first};
  *out = plan;
  return set_ok();
}

void soma_adamw_destroy(soma_adamw* plan) {
  if (!plan) return;
  delete[] plan->first_chunk;
  delete plan;
}

int soma_adamw_step(soma_adamw* plan, int64_t t, double lr, double beta1, double beta2, double delta,
                    const float* grad_scale, void* stream) {
  if (!plan) return set_error(SOMA_EINVAL, "plan is NULL");
  if (t < 1) return set_error(SOMA_EINVAL, "the update number t must be >= 1");
  if (!std::isfinite(lr)) return set_error(SOMA_EINVAL, "lr must be finite");
  if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0))
    return set_error(SOMA_EINVAL, "beta1 and beta2 must be in [0, 1)");
  if (!(std::isfinite(delta) && delta > 0.0)) return set_error(SOMA_EINVAL, "delta must be finite and > 0");
  if (!is_aligned(grad_scale, 4)) return set_error(SOMA_EINVAL, "grad_scale must be 4-byte aligned");
  if (plan->chunks == 0) return set_ok();
  const double bc1 = 1.0 - std::pow(beta1, double(t)), bc2 = 1.0 - std::pow(beta2, double(t));
  const Rates r{float(beta1), float(1.0 - beta1), float(beta2), float(1.0 - beta2), float(lr / bc1),
                float(1.0 / std::sqrt(bc2)), float(delta), lr};
  hipLaunchKernelGGL(k_adamw, dim3(unsigned(plan->chunks)), dim3(kThreadsAdamw), 0, stream_of(stream), plan->tensors,
                     plan->blocks, r, grad_scale);
  if (int rc = launched("k_adamw")) return rc;
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
    hipLaunchKernelGGL(k_adamw_moments, dim3(unsigned(chunks)), dim3(kThreadsAdamw), 0, stream_of(stream),
                       plan->tensors, plan->blocks + plan->first_chunk[i], i, o);
    if (int rc = launched("k_adamw_moments")) return rc;
  }
  return set_ok();
}

}  // extern "C"
