// attention8.hip -- attention of new tokens over a cache in 8 bits: scores
// capped by a tanh, a bias by the distance of the sites, masks by volume, round
// and prefix.
//
// As attention over bf16 keys: one pass over tiles of 64 keys with the running maximum
// and sum of the softmax, the heads that share keys as rows of one query matrix (row r is
// token r / group, head r % group), transposed scores K Q^T, whose registers are the right
// operand of out^T += V^T P^T.  The codes go to LDS as they are (64 keys of 64 channels: 8 KB) and become bf16, exactly,
// on their way into the matrix instructions: K a granule of 16 codes of a row at a time, V by the read that
// transposes bytes.  A key's scale multiplies its score, a value's scale its probability.
//
// Few rows: the four waves of a workgroup take the same 32 rows and every fourth tile, each with buffers of its own and
// without a barrier, and join at the end.  Many rows: they take 32 rows each and share the tiles.
//
// What to read: before the keys of 8 (16) tiles a workgroup reads their sites, and skips tiles that none of its rows sees.
//
// The keys are split over workgroups until the card is full; each leaves its maximum, sum and unscaled result (fp32),
// and a last kernel joins them.
#include <float.h>
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>

#include "cache8.h"
#include "lds_tiles.h"
#include "token_scores.h"

namespace {

using namespace pd;

constexpr int TILE = 64;  // keys
constexpr int NW = 4;     // waves of a workgroup
constexpr int RUN = 4;    // neighbouring work items of one XCD
constexpr int MOST_SPLITS = 256;

struct Attn8 {
  int batch, heads, kv_heads, group, head_dim, n_q, capacity, tiles;
  int rows;  // n_q * group
  unsigned items;  // row_tiles * splits * kv_heads * batch
  int row_tiles, splits, tiles_per_split;
  int causal, prefix_last;  // prefix - 1; INT_MIN, below every round: none
  // a score of product x and key scale s, in log2 units: s factor x, or with the cap, for u = s factor x:
  // cap_b + cap_a / (1 + 2^(2 log2(e) u)), and for |u| <= 0.35 a polynomial
  float factor, cap_a, cap_b;
  const uint16_t* q;
  uint16_t* out;
  long long q_b, q_t, q_h, o_b, o_t, o_h;
  const uint8_t* codes;
  const float* scales;
  const int4* sites;
  const int4* q_sites;
  long long q_sites_b;
  const float* slopes;
  float* part_o;    // results of splits, [splits][batch][kv_heads][rows][DP]
  float2* part_ml;  // [splits][batch][kv_heads][rows]: maximum (log2 units), sum
};

// Where granule g (16 codes) of a key's row lies.  Turned by the key, so that the lanes that are served together fall on
// different banks: K is read 16 keys at a time, one granule each, V eight keys, two granules each.
template <int DP>
__device__ __forceinline__ int k8_place(int key, int g) {
  const int turn = DP == 128 ? (key >> 1) & 7 : DP == 64 ? (key >> 2) & 3 : (key >> 3) & 1;
  return key * DP + ((g ^ turn) << 4);
}
template <int DP>
__device__ __forceinline__ int v8_place(int key, int g) {
  const int turn = DP == 128 ? ((key >> 1) & 1) * 2 + ((key >> 3) & 1) * 4 : DP == 64 ? ((key >> 3) & 1) * 2 : 0;
  return key * DP + ((g ^ turn) << 4);
}

// Eight codes as bf16, exactly.
template <bool INT8>
__device__ __forceinline__ bf16x8 decode(uint32_t a, uint32_t b) {
  uint32_t u[4];
  if constexpr (INT8) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const uint32_t w = n ? b : a;
      u[2 * n] = bf16_pack((float)(int8_t)w, (float)(int8_t)(w >> 8));
      u[2 * n + 1] = bf16_pack((float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24));
    }
  } else {
    u[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false));
    u[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true));
    u[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false));
    u[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true));
  }
  return __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3]));
}

// A tile of keys in LDS.
template <int DP>
struct alignas(16) KeyTile {
  uint8_t k[TILE * DP], v[TILE * DP];
  int4 sites[TILE];
  float ks[TILE], vs[TILE];  // scales
};
// What follows from them: ks factor, and site_bytes.
struct alignas(16) KeyNotes {
  float f[TILE];
  uint32_t bytes[TILE];
};

// FEW: the waves share the rows and take tiles in turn.
template <int DP, bool FEW, bool INT8, Cap CAP>
__global__ void __launch_bounds__(NW * 64, 2) attention8_kernel(const Attn8 p) {
  constexpr int NT = FEW ? 64 : NW * 64;  // threads that stage a tile
  constexpr int GR = DP / 16;             // granules of a row
  constexpr int G = TILE * GR / NT > 0 ? TILE * GR / NT : 1;
  constexpr int ROWS = FEW ? 32 : NW * 32;
  constexpr int AHEAD = FEW ? 8 : 16;     // tiles whose sites are looked at together
  __shared__ KeyTile<DP> tiles[FEW ? NW : 1][2];
  __shared__ KeyNotes key_notes[FEW ? NW : 1];
  __shared__ int lq[4][NW];
  __shared__ int visible[FEW ? 1 : AHEAD];
  __shared__ float2 ml[FEW ? NW : 1][32];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  const int part = FEW ? 0 : wave;  // of the tile's staging
  const int stid = FEW ? lane : tid;
  KeyTile<DP>* const mine = tiles[FEW ? wave : 0];
  KeyNotes& notes = key_notes[FEW ? wave : 0];

  // Workgroups are dealt to the eight XCDs in turn.  An XCD takes RUN neighbouring items, which read the same keys, in its L2.
  unsigned item = ((blockIdx.x >> 3) / RUN * 8 + (blockIdx.x & 7)) * RUN + (blockIdx.x >> 3) % RUN;
  if (item >= p.items) return;
  const int row_tile = (int)(item % p.row_tiles);
  item /= p.row_tiles;
  const int split = item % p.splits;
  item /= p.splits;
  const int kvh = item % p.kv_heads, b = item / p.kv_heads;

  const int row = row_tile * ROWS + (FEW ? 0 : wave * 32) + (lane & 31);
  const int r = row < p.rows ? row : p.rows - 1;  // rows past the end repeat the last: not stored
  const int token = r / p.group, head = kvh * p.group + r % p.group;
  const uint16_t* q = p.q + b * p.q_b + token * p.q_t + head * p.q_h;
  const long long k_row = ((long long)(b * 2) * p.kv_heads + kvh) * p.capacity, v_row = k_row + (long long)p.kv_heads * p.capacity;
  const uint8_t* kb = p.codes + k_row * p.head_dim;
  const uint8_t* vb = p.codes + v_row * p.head_dim;
  const int4* sites = p.sites + (long long)b * p.capacity;
  // step 2 s + c of a product takes channels 32 s + 16 half + 8 c on: a lane's granule of K in two
  bf16x8 fq[DP / 16];
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    const int d = 32 * (s >> 1) + 16 * half + 8 * (s & 1);
    const uint4 w = d < p.head_dim ? *(const uint4*)(q + d) : make_uint4(0, 0, 0, 0);
    fq[s] = __builtin_bit_cast(bf16x8, w);
  }
  const int4 at = p.q_sites[b * p.q_sites_b + token];
  const bool there = at.w >= 0;
  const int own_volume = there ? at.w : -2;  // -2: no key's volume
  const int last = p.causal ? max(at.x, p.prefix_last) : INT_MAX;  // the last round that the row sees
  const uint32_t at_bytes = site_bytes(at);
  // Finite slopes past 2^94 leave a row its nearest tokens alone (negative ones its farthest), as 2^94 does, whose products
  // with 2^24 (below) and with any distance stay finite.
  const bool bias = p.slopes != nullptr;
  float slope = bias ? p.slopes[head] : 0.0f;
  if (fabsf(slope) < INFINITY) slope = fminf(fmaxf(slope * -LOG2E, -0x1p94f), 0x1p94f);

  // what this wave's rows see, and the workgroup's
  const int wv_min = wave_min(there ? at.w : INT_MAX), wv_max = wave_max(there ? at.w : -1);
  const int wt_min = wave_min(there ? at.x : INT_MAX), wt_max = wave_max(there ? at.x : INT_MIN);
  const bool w_plain = __all(there) && wv_min == wv_max;
  const bool w_bytes = (wt_min >> 8) == (wt_max >> 8) && __all(!there || (in_byte(at.y) && in_byte(at.z)));
  const int w_whole_last = p.causal ? max(wt_min, p.prefix_last) : INT_MAX, w_last = p.causal ? max(wt_max, p.prefix_last) : INT_MAX;
  int gv_min = wv_min, gv_max = wv_max, g_last = w_last;
  if constexpr (!FEW) {
    if (lane == 0) lq[0][wave] = wv_min, lq[1][wave] = wv_max, lq[2][wave] = w_last;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      gv_min = min(gv_min, lq[0][w]);
      gv_max = max(gv_max, lq[1][w]);
      g_last = max(g_last, lq[2][w]);
    }
    gv_min = __builtin_amdgcn_readfirstlane(gv_min);
    gv_max = __builtin_amdgcn_readfirstlane(gv_max);
    g_last = __builtin_amdgcn_readfirstlane(g_last);
  }

  // The tiles to visit, as a mask over the next AHEAD of this wave's (workgroup's) tiles.
  const int begin = split * p.tiles_per_split + (FEW ? wave : 0), end = min(p.tiles, (split + 1) * p.tiles_per_split);
  constexpr int STRIDE = FEW ? NW : 1;
  int base = begin - AHEAD * STRIDE;
  uint32_t mask = 0;
  auto site_at = [&](int key) { return key < p.capacity ? sites[key] : make_int4(0, 0, 0, -1); };
  auto sees = [&](const int4 s) { return s.w >= 0 && s.w >= gv_min && s.w <= gv_max && s.x <= g_last; };
  auto next_tile = [&]() -> int {  // -1: no more
    while (mask == 0) {
      base += AHEAD * STRIDE;
      if (base >= end) return -1;
      if constexpr (FEW) {
        int4 s[AHEAD];
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) s[n] = base + n * STRIDE < end ? site_at((base + n * STRIDE) * TILE + lane) : make_int4(0, 0, 0, -1);
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) mask |= __any(sees(s[n])) ? 1u << n : 0u;
      } else {
        int4 s[AHEAD / NW];
#pragma unroll
        for (int n = 0; n < AHEAD / NW; ++n) {
          const int tile = base + wave + n * NW;
          s[n] = tile < end ? site_at(tile * TILE + lane) : make_int4(0, 0, 0, -1);
        }
        __syncthreads();  // the last mask is read
#pragma unroll
        for (int n = 0; n < AHEAD / NW; ++n) {
          const bool any = __any(sees(s[n]));
          if (lane == 0) visible[wave + n * NW] = any;
        }
        __syncthreads();
        mask = (uint32_t)__ballot(lane < AHEAD && visible[lane & (AHEAD - 1)]);
      }
    }
    const int bit = __builtin_ctz(mask);
    mask &= mask - 1;
    return base + bit * STRIDE;
  };

  // columns past head_dim stay the zeros that they are set to here
  if (p.head_dim < DP) {
    for (int c = stid; c < TILE * GR; c += NT)
#pragma unroll
      for (int n = 0; n < 2; ++n) *(uint4*)(mine[n].k + c * 16) = *(uint4*)(mine[n].v + c * 16) = make_uint4(0, 0, 0, 0);
    if constexpr (!FEW) __syncthreads();
  }
  // Staging, straight into LDS: granule slots stid + n NT.  Keys past the end repeat the last.
  auto load_tile = [&](KeyTile<DP>& t, int tile) {
    const int k0 = tile * TILE, most_key = p.capacity - 1 - k0;
#pragma unroll
    for (int n = 0; n < G; ++n) {
      const int slot = stid + n * NT, first = (n * NT + part * 64) * 16;
      if (TILE * GR < NT && part * 64 >= TILE * GR) break;  // (32 channels in four waves: two of them)
      const int key = slot / GR, pos = slot % GR;
      const int kg = pos ^ (k8_place<DP>(key, 0) >> 4) % GR, vg = pos ^ (v8_place<DP>(key, 0) >> 4) % GR;
      const long long from = (long long)(k0 + min(key, most_key)) * p.head_dim;
      if (16 * kg < p.head_dim) send16(kb + from + 16 * kg, t.k + first);
      if (16 * vg < p.head_dim) send16(vb + from + 16 * vg, t.v + first);
    }
    const int key = k0 + min(lane, most_key);
    if (FEW || wave == 0) send16(sites + key, t.sites);
    if (FEW || wave == 1) send4at(p.scales + k_row + key, t.ks);
    if (FEW || wave == 2) send4at(p.scales + v_row + key, t.vs);
  };

  f32x16 o[DP / 32];
#pragma unroll
  for (int n = 0; n < DP / 32; ++n)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[n][e] = 0.0f;
  // scores are taken relative to `top`, the row's reference: set by the first tile that it sees, raised when a score
  // exceeds it by 8 (the sums then stay below 2^8 times their number)
  float top = 0.0f, total = 0.0f;
  bool unset = true;

  // LDS places of this lane's operands
  int k_off[DP / 32], v_off[DP / 32];
  const int v_key = 4 * half + ((lane >> 1) & 3) + 8 * ((lane >> 3) & 1);
#pragma unroll
  for (int s = 0; s < DP / 32; ++s) {
    k_off[s] = k8_place<DP>(lane & 31, 2 * s + half);
    v_off[s] = v8_place<DP>(v_key, 2 * s + ((lane >> 4) & 1)) + (lane & 1) * 8;
  }

  auto work = [&](KeyTile<DP>& t, int tile) {
    // what the tile's keys are to this wave's rows: a lane a key
    const int4 s = t.sites[lane];
    const bool held = tile * TILE + lane < p.capacity && s.w >= 0;
    const uint64_t tokens = __ballot(held);
    if (!__any(held && s.w >= wv_min && s.w <= wv_max && s.x <= w_last)) return;
    // every row sees every key, and the bytes give the distances
    const bool whole = w_plain && __all(held && s.w == wv_min && s.x <= w_whole_last &&
                                        (!bias || ((s.x >> 8) == (wt_min >> 8) && in_byte(s.y) && in_byte(s.z)))) &&
                       (!bias || w_bytes);
    // (the waves that share a tile write the same)
    notes.f[lane] = t.ks[lane] * p.factor;
    notes.bytes[lane] = site_bytes(s);
    __builtin_amdgcn_wave_barrier();

    f32x16 z[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
#pragma unroll
      for (int e = 0; e < 16; ++e) z[n][e] = 0.0f;
#pragma unroll
      for (int c = 0; c < DP / 32; ++c) {
        const uint4 w = *(const uint4*)(t.k + k_off[c] + 32 * n * DP);
        z[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode<INT8>(w.x, w.y), fq[2 * c], z[n], 0, 0, 0);
        z[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode<INT8>(w.z, w.w), fq[2 * c + 1], z[n], 0, 0, 0);
      }
    }
    // times the key's scale; whether one of the wave's exceeds 0.35 of the cap
    float size = 0.0f;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 f4 = *(const float4*)&notes.f[32 * n + 8 * g + 4 * half];
        const float f[4] = {f4.x, f4.y, f4.z, f4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          z[n][4 * g + e] *= f[e];
          if constexpr (CAP != CAP_NONE) size = fmaxf(size, fabsf(z[n][4 * g + e]));
        }
      }
    if constexpr (CAP != CAP_NONE) {
      const bool large = __any(!(size <= 0.35f));
      auto capped = [&](auto some_large) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float u = z[n][e], w = u * u;
            if constexpr (CAP == CAP_NEAR) {
              if constexpr (some_large.value)
                z[n][e] = fmaf(p.cap_a, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * (2.0f * LOG2E))), p.cap_b);
              else
                z[n][e] = u * p.cap_b * fmaf(w, fmaf(w, TANH5, TANH3), TANH1);
            } else {
              float x = u * p.cap_b * fmaf(w, fmaf(w, fmaf(w, TANH7R, TANH5R), TANH3R), 1.0f);
              if constexpr (some_large.value)
                x = fabsf(u) <= 0.35f ? x : fmaf(p.cap_a, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * (2.0f * LOG2E))), p.cap_b);
              z[n][e] = x;
            }
          }
      };
      if (large)
        capped(std::true_type());
      else
        capped(std::false_type());
    }
    float most = -INFINITY;
    if (whole) {
      if (bias) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const uint4 w = *(const uint4*)&notes.bytes[32 * n + 8 * g + 4 * half];
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              // dist < 2^10 as an fp16 number below the normal range is dist 2^-24: the mixed multiply-add takes it as it is
              const uint32_t dist = __builtin_amdgcn_sad_u8(u[e], at_bytes, 0);
              z[n][4 * g + e] += fmaf((float)__builtin_bit_cast(_Float16, (uint16_t)dist), slope * 0x1p24f, -top);
              most = fmaxf(most, z[n][4 * g + e]);
            }
          }
      } else {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            z[n][e] -= top;
            most = fmaxf(most, z[n][e]);
          }
      }
    } else {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = 32 * n + 8 * (e >> 2) + 4 * half + (e & 3);
          const int4 k = t.sites[key];
          const uint32_t sign = 0x80000000u;
          const uint32_t dist = far_add((uint32_t)at.x ^ sign, (uint32_t)k.x ^ sign,
                                        far_add((uint32_t)at.y ^ sign, (uint32_t)k.y ^ sign, far_add((uint32_t)at.z ^ sign, (uint32_t)k.z ^ sign, 0)));
          const bool seen = tokens >> key & 1 && k.w == own_volume && k.x <= last;
          z[n][e] = seen ? z[n][e] + (bias ? fmaf((float)dist, slope, -top) : -top) : -INFINITY;
          most = fmaxf(most, z[n][e]);
          if ((e & 3) == 3) __builtin_amdgcn_sched_barrier(0);  // four keys' sites in registers at a time
        }
    }
    if (__any(most > 8.0f || (unset && most > -INFINITY))) {
      most = fmaxf(most, __shfl_xor(most, 32));
      const bool raise = most > 8.0f || (unset && most > -INFINITY);
      const float up = raise ? most : 0.0f;
      const float alpha = raise && !unset ? __builtin_amdgcn_exp2f(-up) : 1.0f;
      if (raise) unset = false;
      top += up;
      total *= alpha;
#pragma unroll
      for (int m = 0; m < DP / 32; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[m][e] *= alpha;
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) z[n][e] -= up;
    }
    // probabilities; times the value's scale, in bf16: keys 16 s + 4 half + {0 .. 3, 8 .. 11} of block n
    uint4 pr[2][2];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        uint32_t u[4];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const float4 f4 = *(const float4*)&t.vs[32 * n + 16 * s2 + 8 * g + 4 * half];
          const float f[4] = {f4.x, f4.y, f4.z, f4.w};
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = z[n][8 * s2 + 4 * g + e], e2 = __builtin_amdgcn_exp2f(y);
            total += e2;
            x[e] = e2 * f[e];
            if (!whole) x[e] = y == -INFINITY ? 0.0f : x[e];  // (an invisible row's scale may be anything)
          }
          u[2 * g] = bf16_pack(x[0], x[1]), u[2 * g + 1] = bf16_pack(x[2], x[3]);
        }
        pr[n][s2] = make_uint4(u[0], u[1], u[2], u[3]);
      }
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        typedef __attribute__((ext_vector_type(2))) int i32x2;
        typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
        uint32_t keep[2] = {~0u, ~0u};
        if (!whole) {  // codes at places without a token may be E4M3's NaN
          const uint32_t bits = (uint32_t)(tokens >> (32 * n + 16 * s2 + 4 * half));
          keep[0] = ((bits & 15) * 0x00204081u & 0x01010101u) * 255u;
          keep[1] = ((bits >> 8 & 15) * 0x00204081u & 0x01010101u) * 255u;
        }
#pragma unroll
        for (int m = 0; m < DP / 32; ++m) {
          const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(t.v + v_off[m] + (32 * n + 16 * s2) * DP));
          o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode<INT8>((uint32_t)w[0] & keep[0], (uint32_t)w[1] & keep[1]),
                                                         __builtin_bit_cast(bf16x8, pr[n][s2]), o[m], 0, 0, 0);
        }
      }
  };

  int tile = next_tile(), buf = 0;
  if (tile >= 0) load_tile(mine[0], tile);
  sent();
  if constexpr (!FEW) __syncthreads();
  while (tile >= 0) {
    const int after = next_tile();
    if (after >= 0) load_tile(mine[buf ^ 1], after);
    __builtin_amdgcn_sched_barrier(0);
    work(mine[buf], tile);
    sent();
    if constexpr (!FEW) __syncthreads();
    tile = after, buf ^= 1;
  }

  total += __shfl_xor(total, 32);
  bool none = unset && total == 0.0f;  // saw nothing (without a reference, but NaN scores: not nothing)
  const long long rows_at = (((long long)split * p.batch + b) * p.kv_heads + kvh) * p.rows;
  if constexpr (FEW) {
    // join the four waves: their results through the tiles' memory, 16 columns of every wave's at a time
    if (half == 0) ml[wave][lane & 31] = make_float2(none ? -INFINITY : top, total);
    float* const lo = (float*)mine;  // [row][DP]
    static_assert(sizeof(KeyTile<DP>) * 2 >= 32 * DP * 4, "a wave's result fits its tiles");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int m = 0; m < DP / 32; ++m)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(float4*)(lo + (lane & 31) * DP + 32 * m + 8 * g + 4 * half) = make_float4(o[m][4 * g], o[m][4 * g + 1], o[m][4 * g + 2], o[m][4 * g + 3]);
    __syncthreads();
    const int rows_here = min(32, p.rows - row_tile * 32);
    for (int c = tid; c < rows_here * (DP / 4); c += NW * 64) {
      const int i = c / (DP / 4), d = c % (DP / 4) * 4;
      float best = -INFINITY;
#pragma unroll
      for (int w = 0; w < NW; ++w) best = fmaxf(best, ml[w][i].x);
      float4 acc = make_float4(0, 0, 0, 0);
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float2 of = ml[w][i];
        if (of.x == -INFINITY) continue;  // the row saw nothing there
        const float weight = __builtin_amdgcn_exp2f(of.x - best);
        const float4 v = *(const float4*)((const float*)tiles[FEW ? w : 0] + i * DP + d);
        acc.x = fmaf(v.x, weight, acc.x), acc.y = fmaf(v.y, weight, acc.y), acc.z = fmaf(v.z, weight, acc.z), acc.w = fmaf(v.w, weight, acc.w);
        sum = fmaf(of.y, weight, sum);
      }
      const int rr = row_tile * 32 + i;
      if (p.splits > 1) {
        *(float4*)(p.part_o + (rows_at + rr) * DP + d) = acc;
        if (d == 0) p.part_ml[rows_at + rr] = make_float2(best, sum);
      } else if (d < p.head_dim) {
        const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : NAN;
        uint2 w;
        w.x = bf16_pack(acc.x * inv, acc.y * inv), w.y = bf16_pack(acc.z * inv, acc.w * inv);
        *(uint2*)(p.out + b * p.o_b + rr / p.group * p.o_t + (kvh * p.group + rr % p.group) * p.o_h + d) = w;
      }
    }
    return;
  }
  if (row >= p.rows) return;
  if (p.splits > 1) {
#pragma unroll
    for (int m = 0; m < DP / 32; ++m)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(float4*)(p.part_o + (rows_at + row) * DP + 32 * m + 8 * g + 4 * half) = make_float4(o[m][4 * g], o[m][4 * g + 1], o[m][4 * g + 2], o[m][4 * g + 3]);
    if (half == 0) p.part_ml[rows_at + row] = make_float2(none ? -INFINITY : top, total);
    return;
  }
  const float inv = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : NAN;
  uint16_t* out = p.out + b * p.o_b + token * p.o_t + head * p.o_h;
#pragma unroll
  for (int m = 0; m < DP / 32; ++m)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = 32 * m + 8 * g + 4 * half;
      if (d < p.head_dim) {
        uint2 w;
        w.x = bf16_pack(o[m][4 * g] * inv, o[m][4 * g + 1] * inv);
        w.y = bf16_pack(o[m][4 * g + 2] * inv, o[m][4 * g + 3] * inv);
        *(uint2*)(out + d) = w;
      }
    }
}

// Joins the splits of one row: out = sum 2^(m_s - m) o_s / sum 2^(m_s - m) l_s.  The weights first, one split a thread; then
// DP / 4 lanes read a split's row, and the workgroup's groups of them take splits in turn.
template <int DP>
__global__ void __launch_bounds__(256) attention8_join_kernel(const Attn8 p) {
  constexpr int L = DP / 4, GROUPS = 256 / L;
  __shared__ float4 so[GROUPS][L];
  __shared__ float weight[MOST_SPLITS];
  __shared__ float2 sm[4];
  const int tid = threadIdx.x, lane = tid % L, g = tid / L;
  const long long item = blockIdx.x;  // (batch, kv_heads, rows)
  const int row = (int)(item % p.rows), kvh = (int)(item / p.rows % p.kv_heads), b = (int)(item / p.rows / p.kv_heads);
  const long long step = (long long)p.batch * p.kv_heads * p.rows;
  const float2 ml = tid < p.splits ? p.part_ml[tid * step + item] : make_float2(-INFINITY, 0.0f);
  float top = ml.x;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
  if ((tid & 63) == 0) sm[tid >> 6].x = top;
  __syncthreads();
  top = fmaxf(fmaxf(sm[0].x, sm[1].x), fmaxf(sm[2].x, sm[3].x));
  const float w = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - top);  // 0: the row saw nothing there
  float total = ml.x == -INFINITY ? 0.0f : ml.y * w;
  weight[tid] = w;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m);
  if ((tid & 63) == 0) sm[tid >> 6].y = total;
  __syncthreads();
  total = (sm[0].y + sm[1].y) + (sm[2].y + sm[3].y);
  float4 acc = make_float4(0, 0, 0, 0);
#pragma unroll 4
  for (int s = g; s < p.splits; s += GROUPS) {
    const float a = weight[s];
    const float4 o = *(const float4*)(p.part_o + (s * step + item) * DP + 4 * lane);
    acc.x = fmaf(o.x, a, acc.x), acc.y = fmaf(o.y, a, acc.y), acc.z = fmaf(o.z, a, acc.z), acc.w = fmaf(o.w, a, acc.w);
  }
  so[g][lane] = acc;
  __syncthreads();
  if (g != 0 || 4 * lane >= p.head_dim) return;
  for (int n = 1; n < GROUPS; ++n) {
    const float4 o = so[n][lane];
    acc.x += o.x, acc.y += o.y, acc.z += o.z, acc.w += o.w;
  }
  const float inv = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : NAN;
  uint2 v;
  v.x = bf16_pack(acc.x * inv, acc.y * inv), v.y = bf16_pack(acc.z * inv, acc.w * inv);
  *(uint2*)(p.out + b * p.o_b + row / p.group * p.o_t + (kvh * p.group + row % p.group) * p.o_h + 4 * lane) = v;
}

// How a call runs.
struct Plan {
  bool few;
  int row_tiles, tiles, splits, tiles_per_split;
  size_t o_bytes, ml_bytes;
  long long items;
};

Plan plan_for(const pd_attention8_args* a) {
  const pd_cache& c = a->cache;
  Plan n = {};
  const long long rows = (long long)a->n_q * (a->heads / c.kv_heads), heads = (long long)c.kv_heads * c.batch;
  n.few = rows <= 64;
  n.row_tiles = (int)((rows + (n.few ? 31 : 127)) / (n.few ? 32 : 128));
  n.tiles = (int)(((long long)c.capacity + TILE - 1) / TILE);
  const int dp = c.head_dim <= 32 ? 32 : c.head_dim <= 64 ? 64 : 128;
  // Splits: to fill the card, down to 8 tiles each
  const long long whole = n.row_tiles * heads, fill = n.few ? (dp == 128 ? 256 : 512) : 512;
  long long splits = (fill + whole - 1) / whole;
  if (splits > n.tiles / 8) splits = n.tiles / 8;
  if (splits > MOST_SPLITS) splits = MOST_SPLITS;
  const long long most = (1ll << 30) / (dp * 4) / heads / rows;  // 1 GB of workspace (the product could pass 64 bits)
  if (splits > most) splits = most;
  if (splits < 1) splits = 1;
  n.tiles_per_split = (int)((n.tiles + splits - 1) / splits);
  if (n.tiles_per_split < 1) n.tiles_per_split = 1;
  n.splits = n.tiles ? (n.tiles + n.tiles_per_split - 1) / n.tiles_per_split : 1;
  n.o_bytes = n.splits > 1 ? (size_t)n.splits * heads * rows * dp * 4 : 0;
  n.ml_bytes = n.splits > 1 ? (size_t)n.splits * heads * rows * 8 : 0;
  n.items = whole * n.splits;
  return n;
}

bool rows16(const void* p, long long b, long long t, long long h) {
  return (uintptr_t)p % 16 == 0 && b % 8 == 0 && t % 8 == 0 && h % 8 == 0;
}

pd_status check(const pd_attention8_args* a, bool pointers) {
  if (!a) return PD_ERR_INVALID_ARG;
  const pd_cache& c = a->cache;
  const pd_status ok = check_cache(c, false);
  if (ok != PD_OK) return ok;
  if (a->heads < 0 || a->n_q < 0 || !(fabsf(a->scale) < INFINITY) || !(a->cap >= 0.0f) || !(a->cap < INFINITY)) return PD_ERR_INVALID_ARG;
  if (a->causal < 0 || a->causal > 1) return PD_ERR_INVALID_ARG;
  if (a->prefix != PD_PREFIX_NONE && (a->prefix < 0 || (a->prefix && !a->causal))) return PD_ERR_INVALID_ARG;
  if (a->heads && (!c.kv_heads || a->heads % c.kv_heads)) return PD_ERR_INVALID_ARG;
  if (a->heads && a->heads / c.kv_heads > 64) return PD_ERR_UNSUPPORTED;
  if (a->heads && c.batch && a->n_q) {
    // rows are counted in 32 bits, work items and rows of all heads by the launches (threads below 2^32)
    if ((long long)a->n_q * (a->heads / c.kv_heads) >= 1ll << 30) return PD_ERR_UNSUPPORTED;
    const Plan n = plan_for(a);
    if (n.items > (1ll << 24) - 8 * RUN || (n.splits > 1 && (__int128)a->n_q * a->heads * c.batch >= 1ll << 24)) return PD_ERR_UNSUPPORTED;
  }
  if (!pointers || !c.batch || !a->heads || !a->n_q) return PD_OK;
  if (!a->q || !a->out || !a->q_sites || a->out == a->q) return PD_ERR_INVALID_ARG;
  if (c.capacity && check_cache(c, true) != PD_OK) return PD_ERR_INVALID_ARG;
  if ((uintptr_t)a->q_sites % 16 || (uintptr_t)a->slopes % 4) return PD_ERR_INVALID_ARG;
  if (!rows16(a->q, a->q_batch_stride, a->q_token_stride, a->q_head_stride) ||
      !rows16(a->out, a->out_batch_stride, a->out_token_stride, a->out_head_stride))
    return PD_ERR_UNSUPPORTED;
  if (!rows_apart(c.head_dim, {{c.batch, a->out_batch_stride}, {a->n_q, a->out_token_stride}, {a->heads, a->out_head_stride}}))
    return PD_ERR_INVALID_ARG;
  const size_t need = predecoder_attention8_workspace(a);
  if (need && (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < need)) return PD_ERR_INVALID_ARG;
  return PD_OK;
}

template <int DP, bool FEW, bool INT8>
void launch(const Attn8& p, Cap cap, hipStream_t st) {
  const dim3 blocks((p.items + 8 * RUN - 1) / (8 * RUN) * (8 * RUN)), threads(NW * 64);
  if (cap == CAP_NONE)
    hipLaunchKernelGGL((attention8_kernel<DP, FEW, INT8, CAP_NONE>), blocks, threads, 0, st, p);
  else if (cap == CAP_NEAR)
    hipLaunchKernelGGL((attention8_kernel<DP, FEW, INT8, CAP_NEAR>), blocks, threads, 0, st, p);
  else
    hipLaunchKernelGGL((attention8_kernel<DP, FEW, INT8, CAP_FAR>), blocks, threads, 0, st, p);
}

template <int DP>
void launch_width(const Attn8& p, const Plan& n, bool int8, Cap cap, hipStream_t st) {
  if (n.few && int8)
    launch<DP, true, true>(p, cap, st);
  else if (n.few)
    launch<DP, true, false>(p, cap, st);
  else if (int8)
    launch<DP, false, true>(p, cap, st);
  else
    launch<DP, false, false>(p, cap, st);
  if (p.splits > 1)
    hipLaunchKernelGGL(attention8_join_kernel<DP>, dim3((unsigned)(p.kv_heads * p.batch) * p.rows), dim3(256), 0, st, p);
}

}  // namespace

extern "C" size_t predecoder_attention8_workspace(const pd_attention8_args* a) {
  if (check(a, false) != PD_OK || !a->cache.batch || !a->heads || !a->n_q) return 0;
  const Plan n = plan_for(a);
  return n.o_bytes + n.ml_bytes;
}

extern "C" pd_status predecoder_attention8(void* hip_stream, const pd_attention8_args* a) {
  const pd_status ok = check(a, true);
  if (ok != PD_OK) return ok;
  const pd_cache& c = a->cache;
  if (!c.batch || !a->heads || !a->n_q) return PD_OK;
  Attn8 p;
  p.batch = c.batch, p.heads = a->heads, p.kv_heads = c.kv_heads, p.group = a->heads / c.kv_heads, p.head_dim = c.head_dim;
  p.n_q = a->n_q, p.capacity = c.capacity, p.causal = a->causal;
  p.prefix_last = a->prefix == PD_PREFIX_NONE ? INT_MIN : a->prefix - 1;
  const Plan n = plan_for(a);
  p.rows = a->n_q * p.group, p.tiles = n.tiles, p.row_tiles = n.row_tiles, p.splits = n.splits, p.tiles_per_split = n.tiles_per_split;
  p.items = (unsigned)n.items;
  const Cap cap = !(a->cap > 0.0f) ? CAP_NONE : a->cap <= MOST_NEAR ? CAP_NEAR : CAP_FAR;
  // (caps past 2^126, whose double would leave the range, differ from it for scores that are themselves of such size alone)
  const float most_cap = fminf(a->cap, 0x1p126f);
  // kept finite, so that scores of zero stay zero
  const float factor = cap == CAP_NONE ? a->scale * LOG2E : a->scale / most_cap;
  p.factor = fminf(fmaxf(factor, -FLT_MAX), FLT_MAX);
  p.cap_a = -2.0f * most_cap * LOG2E, p.cap_b = most_cap * LOG2E;
  p.q = (const uint16_t*)a->q, p.out = (uint16_t*)a->out;
  p.q_b = a->q_batch_stride, p.q_t = a->q_token_stride, p.q_h = a->q_head_stride;
  p.o_b = a->out_batch_stride, p.o_t = a->out_token_stride, p.o_h = a->out_head_stride;
  p.codes = (const uint8_t*)c.codes, p.scales = c.scales, p.sites = (const int4*)c.sites;
  p.q_sites = (const int4*)a->q_sites, p.q_sites_b = a->q_sites_batch_stride, p.slopes = a->slopes;
  p.part_o = (float*)a->workspace;
  p.part_ml = (float2*)((char*)a->workspace + n.o_bytes);
  const bool int8 = c.codes_type == PD_CODES_INT8;
  const hipStream_t st = (hipStream_t)hip_stream;
  if (c.head_dim <= 32)
    launch_width<32>(p, n, int8, cap, st);
  else if (c.head_dim <= 64)
    launch_width<64>(p, n, int8, cap, st);
  else
    launch_width<128>(p, n, int8, cap, st);
  return hipGetLastError() == hipSuccess ? PD_OK : PD_ERR_DEVICE;
}
