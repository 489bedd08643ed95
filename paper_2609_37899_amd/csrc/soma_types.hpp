// soma_types.hpp -- fp32 and bf16 values in memory, and reductions over a wave.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace soma {

// bf16 is the upper half of an fp32 value.
struct bf16 {
  uint16_t bits;
};

__device__ __forceinline__ float from_bf16(uint32_t bits) { return __uint_as_float(bits << 16); }

// Two fp32 values to bf16, to nearest even (NaN stays NaN): (lo, hi) halves.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  typedef float f2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{lo, hi}, b2));
}

__device__ __forceinline__ float load_value(const float* p) { return *p; }
__device__ __forceinline__ float load_value(const bf16* p) { return from_bf16(p->bits); }
__device__ __forceinline__ void store_value(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_value(bf16* p, float x) { p->bits = static_cast<uint16_t>(bf16_pair(x, 0.0f)); }

// Four consecutive values, aligned to their size.
__device__ __forceinline__ float4 load_four(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load_four(const bf16* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                     __uint_as_float(u.y & 0xFFFF0000u));
}
__device__ __forceinline__ void store_four(float* p, const float4& v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store_four(bf16* p, const float4& v) {
  *reinterpret_cast<uint2*>(p) = make_uint2(bf16_pair(v.x, v.y), bf16_pair(v.z, v.w));
}

// Largest value over the wave's 64 lanes, in every lane.  Within 16 lanes by
// data-parallel moves (each lane's neighbour, the pair's neighbour, then the
// mirrored half row and row), then across the four rows by row swaps.
__device__ __forceinline__ float wave_max(float v) {
#define SOMA_DPP_MAX(ctrl) \
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), ctrl, 0xF, 0xF, true)))
  SOMA_DPP_MAX(0xB1);    // quad_perm [1, 0, 3, 2]
  SOMA_DPP_MAX(0x4E);    // quad_perm [2, 3, 0, 1]
  SOMA_DPP_MAX(0x141);   // row_half_mirror
  SOMA_DPP_MAX(0x140);   // row_mirror
#undef SOMA_DPP_MAX
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

}  // namespace soma
