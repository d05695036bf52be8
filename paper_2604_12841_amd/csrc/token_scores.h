// token_scores.h -- what the attention kernels' scores are made of: the forms of
// the cap, distances between sites, and a wave's smallest and largest values.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pd {

constexpr float LOG2E = 1.4426950408889634f;
// tanh u for |u| <= 0.35 is u (TANH1 + u^2 (TANH3 + u^2 TANH5)) within 4.9e-7 (fitted for the least largest error)
constexpr float TANH1 = 0.9999902f, TANH3 = -0.33268409f, TANH5 = 0.12248027f;
// ... and u (1 + u^2 (TANH3R + u^2 (TANH5R + u^2 TANH7R))) within 4.2e-8 of itself (fitted for the least relative error)
constexpr float TANH3R = -0.33332664f, TANH5R = 0.13299826f, TANH7R = -0.04914851f;


// Forms of the cap.  CAP_NEAR is off by up to 1e-6 of the cap, however small the score: 6e-5 at the largest cap that
// takes it, below what the probabilities' rounding moves.  CAP_FAR is off by 2^-20 of the score itself, for caps of any
// size, and takes 17 % longer (16 volumes of 2548 tokens, 8 query and 2 key heads of 64: 445 us against 379 in one run).
enum Cap { CAP_NONE, CAP_NEAR, CAP_FAR };
constexpr float MOST_NEAR = 64.0f;

// |a - b| + c in one instruction (the compiler takes three for it in a sum of several)
__device__ __forceinline__ uint32_t far_add(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("v_sad_u32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// Rounds, rows and columns as bytes, for distances between sites that share t >> 8.
__device__ __forceinline__ uint32_t site_bytes(const int4 s) {
  return (uint32_t)(s.x & 255) | (uint32_t)(s.y & 255) << 8 | (uint32_t)(s.z & 255) << 16;
}

// The smallest / largest value of a wave's lanes: inside rows of 16 lanes, then from row to row up to lane 63.
template <int CTRL>
__device__ __forceinline__ int moved(int v) {
  return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false);
}
__device__ __forceinline__ int wave_min(int v) {
  v = min(v, moved<0x111>(v)), v = min(v, moved<0x112>(v)), v = min(v, moved<0x114>(v)), v = min(v, moved<0x118>(v));
  v = min(v, moved<0x142>(v)), v = min(v, moved<0x143>(v));
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int wave_max(int v) {
  v = max(v, moved<0x111>(v)), v = max(v, moved<0x112>(v)), v = max(v, moved<0x114>(v)), v = max(v, moved<0x118>(v));
  v = max(v, moved<0x142>(v)), v = max(v, moved<0x143>(v));
  return __builtin_amdgcn_readlane(v, 63);
}

__device__ __forceinline__ bool in_byte(int v) { return (v & ~255) == 0; }

}  // namespace pd
