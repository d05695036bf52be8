// token_values.h -- loads and stores of the token operators' values (bf16 as
// uint16_t bit patterns, fp32) as fp32, one at a time or eight neighbours at
// a time (16-byte aligned), and int8 codes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "activation.h"

namespace pd {

__device__ __forceinline__ float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = (uint16_t)bf16_bits(v); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

__device__ __forceinline__ void load8(const uint16_t* p, float* v) {
  const uint4 w = *(const uint4*)p;
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = __uint_as_float(u[k] << 16);
    v[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
  }
}

__device__ __forceinline__ void load8(const float* p, float* v) {
  const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

// A result is "passing" if it is too large for the 256 MB behind the L2s to keep for its reader together with
// anything else: it is stored past the caches, which leaves them, and the memory's time, to what is still read.
constexpr long long PASSING_BYTES = 128ll << 20;

template <bool PASSING>
__device__ __forceinline__ void store16(void* p, const uint4 w) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
  if constexpr (PASSING)
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, w), (u32x4*)p);
  else
    *(uint4*)p = w;
}

template <bool PASSING = false>
__device__ __forceinline__ void store8(uint16_t* p, const float* v) {
  uint4 w;
  w.x = bf16_pack(v[0], v[1]), w.y = bf16_pack(v[2], v[3]);
  w.z = bf16_pack(v[4], v[5]), w.w = bf16_pack(v[6], v[7]);
  store16<PASSING>(p, w);
}

// (Never past the caches: each of the two stores covers half of every line, which the L2 has to put together.)
template <bool PASSING = false>
__device__ __forceinline__ void store8(float* p, const float* v) {
  *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
  *(float4*)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// Four values rounded to the nearest integers (ties to even) within +-127, v0 in bits 0-7.
__device__ __forceinline__ uint32_t int8_code(float v) {
  return (uint32_t)(int)__builtin_rintf(__builtin_fminf(__builtin_fmaxf(v, -127.0f), 127.0f)) & 0xffu;
}
__device__ __forceinline__ uint32_t int8_pack4(float v0, float v1, float v2, float v3) {
  return int8_code(v0) | int8_code(v1) << 8 | int8_code(v2) << 16 | int8_code(v3) << 24;
}

}  // namespace pd
