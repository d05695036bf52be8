// token_values.h -- loads and stores of the token operators' values (bf16 as
// uint16_t bit patterns, fp32) as fp32, one at a time or eight neighbours at
// a time (16-byte aligned), and int8 codes; on the host, the check of an
// output's strides.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>

#include "activation.h"

namespace pd {

// One axis of a tensor above its rows: its entries, and the values from one to the next.
struct Axis {
  long long size, stride;
};

// Whether rows of `width` values lie clear of each other, as an output's must: from the narrowest axis up, an axis steps
// over all that lies within it.
inline bool rows_apart(long long width, std::initializer_list<Axis> axes) {
  Axis a[4];
  int n = 0;
  for (const Axis& x : axes)
    if (x.size > 1) a[n++] = x;
  auto step = [](const Axis& x) { return x.stride < 0 ? -(__int128)x.stride : (__int128)x.stride; };
  std::sort(a, a + n, [&](const Axis& x, const Axis& y) { return step(x) < step(y); });
  __int128 extent = width;
  for (int k = 0; k < n; ++k) {
    if (step(a[k]) < extent) return false;
    extent += (a[k].size - 1) * step(a[k]);
  }
  return true;
}

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
  store16<PASSING>((void*)p, w);
}

__device__ __forceinline__ void store8(float* p, const float* v) {
  *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
  *(float4*)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// 16 bytes of values: eight bf16 or four fp32.
__device__ __forceinline__ void load16(const uint16_t* p, float* v) { load8(p, v); }
__device__ __forceinline__ void load16(const float* p, float* v) {
  const float4 a = *(const float4*)p;
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
}
template <bool PASSING>
__device__ __forceinline__ void store16(uint16_t* p, const float* v) {
  store8<PASSING>(p, v);
}
template <bool PASSING>
__device__ __forceinline__ void store16(float* p, const float* v) {
  store16<PASSING>((void*)p, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                                        __float_as_uint(v[3])));
}

// Four values within +-127.4 rounded to the nearest integers (ties to even), v0 in bits 0-7: added to 3 2^22, a value's
// integer is in the low bits of the sum.
__device__ __forceinline__ uint32_t int8_pack4(float v0, float v1, float v2, float v3) {
  constexpr float SHIFT = 12582912.0f;
  const uint32_t a = __builtin_amdgcn_perm(__float_as_uint(v1 + SHIFT), __float_as_uint(v0 + SHIFT), 0x0c0c0400u);
  const uint32_t b = __builtin_amdgcn_perm(__float_as_uint(v3 + SHIFT), __float_as_uint(v2 + SHIFT), 0x04000c0cu);
  return a | b;
}

// Four values as E4M3 codes, within the format's range (+-464 rounds to +-448).
__device__ __forceinline__ uint32_t e4m3_pack4_within(float v0, float v1, float v2, float v3) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v0, v1, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v2, v3, lo, true);
}

}  // namespace pd
