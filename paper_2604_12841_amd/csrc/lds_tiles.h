// lds_tiles.h -- tiles of tokens' rows in LDS: loads from memory straight into
// them, where a row's granules lie, reads of transposed operands; and values in
// two bf16 parts.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "activation.h"

namespace pd {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

// Send 16 (4) bytes a lane from memory to LDS at `to` (the same in all lanes) + 16 (4) times the lane; lanes that do
// not take part leave their place as it is.  Complete after sent().  Written out rather than with the builtin, for
// which the compiler waits before any later LDS read, of the other buffer too; no register is an output.  (The wait
// states are those that the load needs after writes of m0 and, by vector instructions, of its scalar base.)
__device__ __forceinline__ uint32_t lds_byte(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
__device__ __forceinline__ void send16(const void* from, const void* to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_byte(to)), "v"(from));
}
__device__ __forceinline__ void send16(const void* base, uint32_t at, const void* to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_byte(to)), "v"(at), "s"(base));
}
__device__ __forceinline__ void send4(const void* base, uint32_t at, const void* to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, %2" ::"s"(lds_byte(to)), "v"(at), "s"(base));
}
__device__ __forceinline__ void send4at(const void* from, const void* to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, off" ::"s"(lds_byte(to)), "v"(from));
}
__device__ __forceinline__ void sent() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
  asm volatile("" ::: "memory");
}

// LDS byte of granule g (8 values) of a key's row (DP values).  Rows are not padded; which
// granule lies where is turned by the key, so that the 16 lanes that are
// served together fall on different banks: K is read 32 keys at a
// time, one granule each, V four keys at a time, two granules each.
template <int DP>
__device__ __forceinline__ int k_place(int key, int g) {
  const int turn = DP == 128 ? key & 15 : DP == 64 ? (key >> 1) & 7 : (key >> 2) & 3;
  return key * (DP * 2) + ((g ^ turn) << 4);
}
template <int DP>
__device__ __forceinline__ int v_place(int key, int g) {
  const int turn = DP == 128 ? (key & 3) << 2 : DP == 64 ? ((key >> 1) & 1) << 2 : 0;
  return key * (DP * 2) + ((g ^ turn) << 4);
}

// Two values in two bf16 parts, to 16 bits: hi + lo.
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = bf16_pack(a, b);
  lo = bf16_pack(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u));
}

// Four rows of 16 columns, 8 bytes a lane of each 16 lanes (row (lane & 15) >> 2, columns 4 (lane & 3) on): a lane gets its column's four rows.
__device__ __forceinline__ s16x4 read_columns(const uint8_t* f) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)f);
}

}  // namespace pd
