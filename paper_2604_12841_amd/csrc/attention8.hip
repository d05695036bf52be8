// attention8.hip -- attention of new tokens over a cache in 8 bits: scores
// capped by a tanh, a bias by the distance of the sites, masks by volume, round
// and prefix.
//
// As attention over bf16 keys: one pass over tiles of 64 keys with the running
// maximum and sum of the softmax, the heads that share keys as rows of one query
// matrix (row r is token r / group, head r % group), transposed scores K Q^T,
// whose registers are the right operand of out^T += V^T P^T.  The codes stay
// codes on their way from memory and become bf16, exactly, as operands: K a
// granule of 16 codes of a row at a time, V by the LDS read that transposes
// bytes.  A key's scale multiplies its score, a value's its probability.
//
// Few rows (up to 64): the eight waves of a workgroup take the same 16 rows and
// every eighth tile, without a barrier; K comes straight into registers, V to
// LDS, a tile ahead; at the end they join.  Sixteen streams of up to 65536
// places, 8 query and 2 key heads of 128, int8: 88 us, 4.9 TB/s (the same loads
// without any work on them: 84 us).  One token against four caches of up to 200
// rounds of d = 13, 8 (2) heads of 64, E4M3: 14.2 us and 4 us of the join.
//
// Many rows: 128 a workgroup, 32 a wave, which share tiles in LDS.  Bound by
// vector instructions, about 20 a score with cap and bias, and by latencies that 1.5
// waves a SIMD leave open: 196 tokens against the same four caches 221 us and 8 us of
// the join (230 TFLOP/s; vector units 0.54 busy without what the exponentials take
// longer, matrix units 0.15, waves wait 0.37 of their cycles).
//
// With a bias, distances come from the last byte of rounds, rows and columns where a
// tile's keys and the queries are of one block of 256 rounds (t >> 8).  Tiles of
// other blocks take the general form, score by score: the same call with rounds 156
// to 355, 100 of them in another block than the queries, takes 448 us against 228, one
// token 22.5 against 18.6.
//
// What to read: before the keys of 8 (16) tiles the sites are read, and tiles
// that no row sees are skipped.
//
// The keys are split over workgroups until the card is full; each leaves its
// maximum, sum and unscaled result (fp32), and a last kernel joins them.
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
constexpr int FW = 8;     // and of one with few rows
constexpr int RUN = 4;    // neighbouring work items of one XCD
constexpr int MOST_SPLITS = 256;

struct Attn8 {
  int batch, heads, kv_heads, group, head_dim, n_q, capacity, tiles;
  int rows;  // n_q * group
  unsigned items;  // row_tiles * splits * kv_heads * batch
  int row_tiles, splits, tiles_per_split;
  int causal, prefix_last;  // prefix - 1; INT_MIN, below every round: none
  // a score of product x and key scale s, in log2 units: s factor x, or with the cap, for u = s factor x:
  // cap_b + cap_a / (1 + 2^(2 log2(e) u)), and for small |u| polynomials.  (CAP_FAR: u = unit s factor x, factor as without a cap:
  // scale / cap, times a key's scale, would lose its last bits below fp32's range.)
  float factor, unit, cap_a, cap_b, poly1, poly3, poly5, low[4], mid[5];
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

// V for few rows: 16 keys of 32 lanes, one granule each.
template <int DP>
__device__ __forceinline__ int vf_place(int key, int g) {
  const int turn = DP == 128 ? ((key >> 1) & 3) | (key >> 2 & 4) : DP == 64 ? ((key >> 2) & 1) | (key >> 3 & 2) : (key >> 4) & 1;
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

// A score in log2 units, t added, from u = x f (x the product, f the key's scale times p.factor): u without a cap, with it cap_b tanh u
// (CAP_FAR: u before the cap, cap_b tanh(unit u)).  TIER: |u| (unit |u|) is at most TIERS[TIER], or 3: anything.
constexpr float TIERS[3] = {0.35f, 0.62f, 0.87f};
// tanh u for |u| <= 0.62 is u (N1 + u^2 (N3 + ...)), for |u| <= 0.87 u (M1 + u^2 (M3 + ...)), within 8e-7 (fitted for the least
// largest error): one and two instructions more than for the small ones, against an exponential and a reciprocal at a quarter of the rate.
// The ranges end where the best polynomials of four and five coefficients pass 8e-7, so that a cap is met within 2^-20 of itself.
constexpr float N1 = 0.99998862f, N3 = -0.33292374f, N5 = 0.12931657f, N7 = -0.03883829f;
constexpr float M1 = 0.99999005f, M3 = -0.33305562f, M5 = 0.13114086f, M7 = -0.04667219f, M9 = 0.01031595f;
template <Cap CAP, int TIER>
__device__ __forceinline__ float score8(const Attn8& p, float u, float t) {
  if constexpr (CAP == CAP_NONE) return u + t;
  const float y = CAP == CAP_FAR ? u * p.unit : u, w = y * y;
  if constexpr (CAP == CAP_NEAR) {
    if constexpr (TIER == 0) return fmaf(u, fmaf(w, fmaf(w, p.poly5, p.poly3), p.poly1), t);
    if constexpr (TIER == 1) return fmaf(u, fmaf(w, fmaf(w, fmaf(w, p.low[3], p.low[2]), p.low[1]), p.low[0]), t);
    if constexpr (TIER == 2) return fmaf(u, fmaf(w, fmaf(w, fmaf(w, fmaf(w, p.mid[4], p.mid[3]), p.mid[2]), p.mid[1]), p.mid[0]), t);
    return fmaf(p.cap_a, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * (2.0f * LOG2E))), p.cap_b + t);
  }
  float x = u * fmaf(w, fmaf(w, fmaf(w, TANH7R, TANH5R), TANH3R), 1.0f);
  if constexpr (TIER > 0)
    x = fabsf(y) <= 0.35f ? x : fmaf(p.cap_a, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y * (2.0f * LOG2E))), p.cap_b);
  return x + t;
}
// Calls f with the tier of a wave's largest |u|.
template <Cap CAP, typename F>
__device__ __forceinline__ void with_tier(const Attn8& p, float size, F&& f) {
  if constexpr (CAP == CAP_FAR) size *= p.unit;
  if constexpr (CAP == CAP_NONE) {
    f(std::integral_constant<int, 0>());
  } else {
    if (!__any(!(size <= TIERS[0])))
      f(std::integral_constant<int, 0>());
    else if (CAP == CAP_NEAR && !__any(!(size <= TIERS[1])))
      f(std::integral_constant<int, 1>());
    else if (CAP == CAP_NEAR && !__any(!(size <= TIERS[2])))
      f(std::integral_constant<int, 2>());
    else
      f(std::integral_constant<int, 3>());
  }
}
// The distance's part of a score: dist < 2^10 as an fp16 number below the normal range is dist 2^-24, which the mixed
// multiply-add takes as it is.
__device__ __forceinline__ float near_part(uint32_t bytes, uint32_t at_bytes, float slope24, float t) {
  return fmaf((float)__builtin_bit_cast(_Float16, (uint16_t)__builtin_amdgcn_sad_u8(bytes, at_bytes, 0)), slope24, t);
}
__device__ __forceinline__ uint32_t distance(const int4 a, const int4 k) {
  const uint32_t sign = 0x80000000u;
  return far_add((uint32_t)a.x ^ sign, (uint32_t)k.x ^ sign, far_add((uint32_t)a.y ^ sign, (uint32_t)k.y ^ sign, far_add((uint32_t)a.z ^ sign, (uint32_t)k.z ^ sign, 0)));
}
// A byte mask of four keys from their bits.
__device__ __forceinline__ uint32_t byte_mask(uint32_t bits) { return ((bits & 15) * 0x00204081u & 0x01010101u) * 255u; }

typedef __attribute__((ext_vector_type(2))) int i32x2;
__device__ __forceinline__ i32x2 read_byte_columns(const uint8_t* f) {
  typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
  return __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)f);
}

// A tile of keys in LDS.
template <int DP>
struct alignas(16) KeyTile {
  uint8_t k[TILE * DP], v[TILE * DP];
  int4 sites[TILE];
  float ks[TILE], vs[TILE];  // scales
};
// What follows from the sites and scales: ks factor, vs (0 where there is no token), and site_bytes.
struct alignas(16) KeyNotes {
  float f[TILE], v[TILE];
  uint32_t bytes[TILE];
};

// What rows of a wave (its 64 lanes) see, and how.
struct Seen {
  int vmin, vmax;        // volumes
  int whole_last, last;  // the last round that all see, that some see
  bool plain;            // all rows are there, of one volume
  bool bytes;            // their sites' bytes give distances to keys of rounds round << 8 on
  int round;
  // whether some row sees a key, and whether all do (and the bytes give the distances)
  __device__ __forceinline__ bool some(const int4 s) const { return s.w >= 0 && s.w >= vmin && s.w <= vmax && s.x <= last; }
  __device__ __forceinline__ bool all(const int4 s, bool bias) const {
    return plain && s.w == vmin && s.x <= whole_last && (!bias || (bytes && (s.x >> 8) == round && in_byte(s.y) && in_byte(s.z)));
  }
};
__device__ __forceinline__ Seen seen_by(const Attn8& p, const int4 at) {
  const bool there = at.w >= 0;
  Seen s;
  s.vmin = wave_min(there ? at.w : INT_MAX), s.vmax = wave_max(there ? at.w : -1);
  const int tmin = wave_min(there ? at.x : INT_MAX), tmax = wave_max(there ? at.x : INT_MIN);
  s.plain = __all(there) && s.vmin == s.vmax;
  s.bytes = (tmin >> 8) == (tmax >> 8) && __all(!there || (in_byte(at.y) && in_byte(at.z)));
  s.round = tmin >> 8;
  s.whole_last = p.causal ? max(tmin, p.prefix_last) : INT_MAX, s.last = p.causal ? max(tmax, p.prefix_last) : INT_MAX;
  return s;
}

// Finite slopes past 2^94 leave a row its nearest tokens alone (negative ones its farthest), as 2^94 does, whose products
// with 2^24 and with any distance stay finite.
__device__ __forceinline__ float slope_of(const Attn8& p, int head) {
  float slope = p.slopes ? p.slopes[head] : 0.0f;
  if (fabsf(slope) < INFINITY) slope = fminf(fmaxf(slope * -LOG2E, -0x1p94f), 0x1p94f);
  return slope;
}

// A key's scale times p.factor: finite for finite scales, so that scores of zero stay zero.
__device__ __forceinline__ float factor_of(const Attn8& p, float scale) {
  const float f = scale * p.factor;
  return fabsf(f) == INFINITY && fabsf(scale) < INFINITY ? copysignf(FLT_MAX, f) : f;
}

struct Item {
  int row_tile, split, kvh, b;
};
// Workgroups are dealt to the eight XCDs in turn.  An XCD takes RUN neighbouring items, which read the same keys, in its L2.
__device__ __forceinline__ bool item_of(const Attn8& p, Item& i) {
  unsigned item = ((blockIdx.x >> 3) / RUN * 8 + (blockIdx.x & 7)) * RUN + (blockIdx.x >> 3) % RUN;
  if (item >= p.items) return false;
  i.row_tile = (int)(item % p.row_tiles);
  item /= p.row_tiles;
  i.split = item % p.splits;
  item /= p.splits;
  i.kvh = item % p.kv_heads, i.b = item / p.kv_heads;
  return true;
}

__device__ __forceinline__ float inverse(float total) { return total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : NAN; }

// Few rows: 16 a workgroup, all of them in each of its waves, which take tiles in turn.  A lane of group g of 16 holds
// keys 16 n + 4 g + {0 .. 3} of row lane & 15.  K comes straight into registers, a tile ahead.
template <int DP, bool INT8, Cap CAP>
__global__ void __launch_bounds__(FW * 64, 2) attention8_few_kernel(const Attn8 p) {
  constexpr int GR = DP / 16;                    // granules of a row
  constexpr int KG = DP > 64 ? 2 : 1;            // granules of K that a lane takes of a key (32 channels: half of one)
  constexpr int STEPS = DP / 32;                 // of a product over the channels
  constexpr int AHEAD = 8;                       // tiles whose sites are looked at together
  __shared__ __attribute__((aligned(16))) uint8_t lv[FW][2][TILE * DP];
  __shared__ KeyNotes key_notes[FW];
  __shared__ float2 ml[FW][16];
  static_assert(2 * TILE * DP >= 16 * DP * 4, "a wave's result fits its tiles");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g4 = lane >> 4;
  KeyNotes& notes = key_notes[wave];
  Item item;
  if (!item_of(p, item)) return;
  const int kvh = item.kvh, b = item.b;
  const long long k_row = ((long long)(b * 2) * p.kv_heads + kvh) * p.capacity, v_row = k_row + (long long)p.kv_heads * p.capacity;
  const uint8_t* kb = p.codes + k_row * p.head_dim;
  const uint8_t* vb = p.codes + v_row * p.head_dim;
  const int4* sites = p.sites + (long long)b * p.capacity;

  // A tile's K, V, sites and scales.  Keys past the end repeat the last.
  uint4 key[4][KG];
  int4 site;
  float ks, vs;
  auto load_v = [&](int buf, int tile) {
    const int k0 = tile * TILE, most_key = p.capacity - 1 - k0;
#pragma unroll
    for (int n = 0; n < GR; ++n) {
      const int slot = lane + n * 64, of = slot / GR, vg = slot % GR ^ (vf_place<DP>(of, 0) >> 4) % GR;
      // (past head_dim the row's last granule: its results are not stored)
      send16(vb + (long long)(k0 + min(of, most_key)) * p.head_dim + min(16 * vg, p.head_dim - 16), lv[wave][buf] + n * 1024);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto load_k = [&](int tile) {
    const int k0 = tile * TILE, most_key = p.capacity - 1 - k0;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint8_t* from = kb + (long long)(k0 + min(16 * n + c, most_key)) * p.head_dim;
#pragma unroll
      for (int j = 0; j < KG; ++j) {
        if constexpr (DP == 32) {
          const uint2 w = *(const uint2*)(from + min(8 * g4, p.head_dim - 8));
          key[n][j].x = w.x, key[n][j].y = w.y;
        } else {
          key[n][j] = *(const uint4*)(from + min(16 * (g4 + 4 * j), p.head_dim - 16));  // (past head_dim q is 0)
        }
      }
    }
    const int at = k0 + min(lane, most_key);
    site = sites[at], ks = p.scales[k_row + at], vs = p.scales[v_row + at];
  };
  const int begin = item.split * p.tiles_per_split + wave, end = min(p.tiles, (item.split + 1) * p.tiles_per_split);
  // the first tile is sent for before it is known whether a row sees it
  if (begin < end) {
    load_v(0, begin);
    load_k(begin);
  }

  const int row = item.row_tile * 16 + c;
  const int r = row < p.rows ? row : p.rows - 1;  // rows past the end repeat the last: not stored
  const int token = r / p.group, head = kvh * p.group + r % p.group;
  const uint16_t* q = p.q + b * p.q_b + token * p.q_t + head * p.q_h;
  bf16x8 fq[STEPS];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int d = DP == 32 ? 8 * g4 : 16 * (g4 + 4 * (s >> 1)) + 8 * (s & 1);
    const uint4 w = *(const uint4*)(q + min(d, p.head_dim - 8));
    fq[s] = __builtin_bit_cast(bf16x8, d < p.head_dim ? w : make_uint4(0, 0, 0, 0));
  }
  const int4 at = p.q_sites[b * p.q_sites_b + token];
  const int own_volume = at.w >= 0 ? at.w : -2;  // -2: no key's volume
  const int last = p.causal ? max(at.x, p.prefix_last) : INT_MAX;
  const uint32_t at_bytes = site_bytes(at);
  const bool bias = p.slopes != nullptr;
  const float slope = slope_of(p, head);
  const Seen seen = seen_by(p, at);

  // the tiles to visit, as a mask over the next AHEAD of this wave's
  int base = begin - AHEAD * FW;
  uint32_t mask = 0;
  auto next_tile = [&]() -> int {  // -1: no more
    while (mask == 0) {
      base += AHEAD * FW;
      if (base >= end) return -1;
      int4 s[AHEAD];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) {
        s[n] = sites[min(min(base + n * FW, end - 1) * TILE + lane, p.capacity - 1)];
      }
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) {
        mask |= base + n * FW < end && __any(seen.some(s[n])) ? 1u << n : 0u;
      }
    }
    const int bit = __builtin_ctz(mask);
    mask &= mask - 1;
    return base + bit * FW;
  };

  f32x4 o[DP / 16];
#pragma unroll
  for (int m = 0; m < DP / 16; ++m) o[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  // scores are taken relative to `top`, the row's reference: set by the first tile that it sees, raised when a score
  // exceeds it by 8 (the sums then stay below 2^8 times their number)
  float top = 0.0f, total = 0.0f;
  bool unset = true;
  // keys 32 s + 4 g4 + {0 .. 3} and 16 more of 16 columns
  const int v_key = 4 * g4 + ((lane >> 1) & 3) + 16 * ((lane >> 3) & 1);
  const int v_off = vf_place<DP>(v_key, 0), v_byte = (lane & 1) * 8;

  int tile = next_tile(), buf = 0;
  if (tile >= 0 && tile != begin) {
    buf = 1;
    load_v(buf, tile);
    load_k(tile);
  }
  while (tile >= 0) {
    // what the tile's keys are to the rows: a lane a key
    const bool held = tile * TILE + lane < p.capacity && site.w >= 0;
    const uint64_t tokens = __ballot(held);
    const bool whole = __all(held && seen.all(site, bias));
    const bool careful = !whole && (tokens != ~0ull || __any(held && !(fabsf(vs) < INFINITY)));
    notes.f[lane] = factor_of(p, ks);
    notes.v[lane] = held ? vs : 0.0f;
    notes.bytes[lane] = site_bytes(site);
    const int4 of_lane = site;
    __builtin_amdgcn_wave_barrier();
    f32x4 z[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      z[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        const uint4 w = key[n][s >> 1];
        z[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(s & 1 ? decode<INT8>(w.z, w.w) : decode<INT8>(w.x, w.y), fq[s], z[n], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    // V has landed: it was sent for before this K, which is used.  The next tile's sends come after that wait.
    const int after = next_tile();
    if (after >= 0) {
      load_v(buf ^ 1, after);
      load_k(after);
    }
    __builtin_amdgcn_sched_barrier(0);

    float size = 0.0f;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const float4 f = *(const float4*)&notes.f[16 * n + 4 * g4];
      z[n][0] *= f.x, z[n][1] *= f.y, z[n][2] *= f.z, z[n][3] *= f.w;
      size = fmaxf(fmaxf(fmaxf(size, fabsf(z[n][0])), fmaxf(fabsf(z[n][1]), fabsf(z[n][2]))), fabsf(z[n][3]));
    }
    float most = -INFINITY;
    if (whole) {
      with_tier<CAP>(p, size, [&](auto tier) {
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const uint4 w = *(const uint4*)&notes.bytes[16 * n + 4 * g4];
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            z[n][e] = score8<CAP, decltype(tier)::value>(p, z[n][e], near_part(u[e], at_bytes, slope * 0x1p24f, -top));
            most = fmaxf(most, z[n][e]);
          }
        }
      });
    } else {
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at_key = 16 * n + 4 * g4 + e;
          const int4 k = make_int4(__shfl(of_lane.x, at_key), __shfl(of_lane.y, at_key), __shfl(of_lane.z, at_key), __shfl(of_lane.w, at_key));
          const bool in = tokens >> at_key & 1 && k.w == own_volume && k.x <= last;
          const float x = score8<CAP, 3>(p, z[n][e], bias ? fmaf((float)distance(at, k), slope, -top) : -top);
          z[n][e] = in ? x : -INFINITY;
          most = fmaxf(most, z[n][e]);
        }
    }
    if (__any(most > 8.0f || (unset && most > -INFINITY))) {
      most = fmaxf(most, __shfl_xor(most, 16));
      most = fmaxf(most, __shfl_xor(most, 32));
      const bool raise = most > 8.0f || (unset && most > -INFINITY);
      const float up = raise ? most : 0.0f;
      const float alpha = raise && !unset ? __builtin_amdgcn_exp2f(-up) : 1.0f;
      if (raise) unset = false;
      top += up;
      total *= alpha;
#pragma unroll
      for (int m = 0; m < DP / 16; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[m][e] *= alpha;
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[n][e] -= up;
    }
    // probabilities, times the value's scale, in two bf16 parts (16 bits: as in the kernel for many rows); and their product with the codes
    auto finish = [&](auto carefully) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        uint32_t hi[4], lo[4], keep[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const float4 f4 = *(const float4*)&notes.v[32 * s + 16 * n + 4 * g4];
          const float f[4] = {f4.x, f4.y, f4.z, f4.w};
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = z[2 * s + n][e], e2 = __builtin_amdgcn_exp2f(y);
            total += e2;
            x[e] = e2 * f[e];
            if constexpr (carefully.value) x[e] = y == -INFINITY ? 0.0f : x[e];  // (an invisible row's scale may be anything)
          }
          split2(x[0], x[1], hi[2 * n], lo[2 * n]);
          split2(x[2], x[3], hi[2 * n + 1], lo[2 * n + 1]);
          // codes at places without a token may be E4M3's NaN
          if constexpr (carefully.value) keep[n] = byte_mask((uint32_t)(tokens >> (32 * s + 16 * n + 4 * g4)));
        }
        const bf16x8 ph = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
        const bf16x8 pl = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
#pragma unroll
        for (int m = 0; m < DP / 16; ++m) {
          i32x2 w = read_byte_columns(lv[wave][buf] + (v_off ^ m << 4) + v_byte + 32 * s * DP);
          if constexpr (carefully.value) w[0] &= keep[0], w[1] &= keep[1];
          const bf16x8 v = decode<INT8>((uint32_t)w[0], (uint32_t)w[1]);
          o[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pl, o[m], 0, 0, 0);
          o[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, ph, o[m], 0, 0, 0);
        }
      }
    };
    if (careful)
      finish(std::true_type());
    else
      finish(std::false_type());
    tile = after, buf ^= 1;
  }

  total += __shfl_xor(total, 16);
  total += __shfl_xor(total, 32);
  const bool none = unset && total == 0.0f;  // saw nothing (without a reference, but NaN scores: not nothing)
  // join the eight waves, through the tiles' memory (what was sent for and not used has to be in before)
  sent();
  if (g4 == 0) ml[wave][c] = make_float2(none ? -INFINITY : top, total);
#pragma unroll
  for (int m = 0; m < DP / 16; ++m)
    *(float4*)((float*)lv[wave] + c * DP + 16 * m + 4 * g4) = make_float4(o[m][0], o[m][1], o[m][2], o[m][3]);
  __syncthreads();
  const long long rows_at = (((long long)item.split * p.batch + b) * p.kv_heads + kvh) * p.rows;
  const int rows_here = min(16, p.rows - item.row_tile * 16);
  for (int x = tid; x < rows_here * (DP / 4); x += FW * 64) {
    const int i = x / (DP / 4), d = x % (DP / 4) * 4;
    float best = -INFINITY;
#pragma unroll
    for (int w = 0; w < FW; ++w) best = fmaxf(best, ml[w][i].x);
    float4 acc = make_float4(0, 0, 0, 0);
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < FW; ++w) {
      const float2 of = ml[w][i];
      if (of.x == -INFINITY) continue;  // the row saw nothing there
      const float weight = __builtin_amdgcn_exp2f(of.x - best);
      const float4 v = *(const float4*)((const float*)lv[w] + i * DP + d);
      acc.x = fmaf(v.x, weight, acc.x), acc.y = fmaf(v.y, weight, acc.y), acc.z = fmaf(v.z, weight, acc.z), acc.w = fmaf(v.w, weight, acc.w);
      sum = fmaf(of.y, weight, sum);
    }
    const int rr = item.row_tile * 16 + i;
    if (p.splits > 1) {
      if (best != -INFINITY) *(float4*)(p.part_o + (rows_at + rr) * DP + d) = acc;  // (the join does not read it otherwise)
      if (d == 0) p.part_ml[rows_at + rr] = make_float2(best, sum);
    } else if (d < p.head_dim) {
      const float inv = inverse(sum);
      uint2 w;
      w.x = bf16_pack(acc.x * inv, acc.y * inv), w.y = bf16_pack(acc.z * inv, acc.w * inv);
      *(uint2*)(p.out + b * p.o_b + rr / p.group * p.o_t + (kvh * p.group + rr % p.group) * p.o_h + d) = w;
    }
  }
}

// Many rows: 32 a wave, 128 a workgroup, whose waves share the tiles.
template <int DP, bool INT8, Cap CAP>
__global__ void __launch_bounds__(NW * 64, 2) attention8_kernel(const Attn8 p) {
  constexpr int NT = NW * 64;
  constexpr int GR = DP / 16;  // granules of a row
  constexpr int AHEAD = 16;    // tiles whose sites are looked at together
  // Queries past 64 channels wait in LDS: in registers they made others spill (62 at 128 channels, 22 now; 196 tokens against four
  // caches of up to 100 rounds, 8 (2) x 128: 194 us against 200).  At 64 channels they cost nothing (228 us; from LDS 232).
  constexpr bool LDS_Q = DP > 64;
  __shared__ KeyTile<DP> tiles[2];
  __shared__ KeyNotes notes;
  __shared__ u32x4 lds_q[LDS_Q ? DP / 16 : 1][NT];  // each thread's own
  __shared__ int lq[3][NW];
  __shared__ int visible[AHEAD];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  Item item;
  if (!item_of(p, item)) return;
  const int kvh = item.kvh, b = item.b;
  const int row = item.row_tile * 128 + wave * 32 + (lane & 31);
  const bool idle = item.row_tile * 128 + wave * 32 >= p.rows;  // a wave without rows sees nothing and sends for its part of the tiles
  const int r = row < p.rows ? row : p.rows - 1;  // rows past the end repeat the last: not stored
  const int token = r / p.group, head = kvh * p.group + r % p.group;
  const uint16_t* q = p.q + b * p.q_b + token * p.q_t + head * p.q_h;
  const long long k_row = ((long long)(b * 2) * p.kv_heads + kvh) * p.capacity, v_row = k_row + (long long)p.kv_heads * p.capacity;
  const uint8_t* kb = p.codes + k_row * p.head_dim;
  const uint8_t* vb = p.codes + v_row * p.head_dim;
  const int4* sites = p.sites + (long long)b * p.capacity;
  // step 2 s + c of a product takes channels 32 s + 16 half + 8 c on: a lane's granule of K in two
  bf16x8 fq[LDS_Q ? 1 : DP / 16];
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    const int d = 32 * (s >> 1) + 16 * half + 8 * (s & 1);
    const uint4 w = d < p.head_dim ? *(const uint4*)(q + d) : make_uint4(0, 0, 0, 0);
    if constexpr (LDS_Q)
      lds_q[s][tid] = __builtin_bit_cast(u32x4, w);
    else
      fq[s] = __builtin_bit_cast(bf16x8, w);
  }
  auto query = [&](int s) {
    if constexpr (LDS_Q)
      return __builtin_bit_cast(bf16x8, lds_q[s][tid]);
    else
      return fq[s];
  };
  const int4 at = p.q_sites[b * p.q_sites_b + token];
  const int own_volume = at.w >= 0 ? at.w : -2;                    // -2: no key's volume
  const int last = p.causal ? max(at.x, p.prefix_last) : INT_MAX;  // the last round that the row sees
  const uint32_t at_bytes = site_bytes(at);
  const bool bias = p.slopes != nullptr;
  const float slope = slope_of(p, head);

  // what this wave's rows see, and the workgroup's
  const Seen seen = seen_by(p, make_int4(at.x, at.y, at.z, idle ? -1 : at.w));
  Seen any = seen;
  if (lane == 0) lq[0][wave] = seen.vmin, lq[1][wave] = seen.vmax, lq[2][wave] = seen.last;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) any.vmin = min(any.vmin, lq[0][w]), any.vmax = max(any.vmax, lq[1][w]), any.last = max(any.last, lq[2][w]);

  // The tiles to visit, as a mask over the next AHEAD.
  const int begin = item.split * p.tiles_per_split, end = min(p.tiles, (item.split + 1) * p.tiles_per_split);
  int base = begin - AHEAD;
  uint32_t mask = 0;
  auto next_tile = [&]() -> int {  // -1: no more
    while (mask == 0) {
      base += AHEAD;
      if (base >= end) return -1;
      int4 s[AHEAD / NW];
#pragma unroll
      for (int n = 0; n < AHEAD / NW; ++n) {
        const int key = (base + wave + n * NW) * TILE + lane;
        s[n] = base + wave + n * NW < end && key < p.capacity ? sites[key] : make_int4(0, 0, 0, -1);
      }
      __syncthreads();  // the last mask is read
#pragma unroll
      for (int n = 0; n < AHEAD / NW; ++n) {
        const bool some = __any(any.some(s[n]));
        if (lane == 0) visible[wave + n * NW] = some;
      }
      __syncthreads();
      mask = (uint32_t)__ballot(lane < AHEAD && visible[lane & (AHEAD - 1)]);
    }
    const int bit = __builtin_ctz(mask);
    mask &= mask - 1;
    return base + bit;
  };

  // columns past head_dim stay the zeros that they are set to here
  if (p.head_dim < DP) {
    for (int c = tid; c < TILE * GR; c += NT)
#pragma unroll
      for (int n = 0; n < 2; ++n) *(uint4*)(tiles[n].k + c * 16) = *(uint4*)(tiles[n].v + c * 16) = make_uint4(0, 0, 0, 0);
    __syncthreads();
  }
  // Staging, straight into LDS: granule slots tid + n NT.  Keys past the end repeat the last.
  auto load_tile = [&](KeyTile<DP>& t, int tile) {
    const int k0 = tile * TILE, most_key = p.capacity - 1 - k0;
#pragma unroll
    for (int n = 0; n < (TILE * GR + NT - 1) / NT; ++n) {
      const int slot = tid + n * NT, first = (n * NT + wave * 64) * 16;
      if (n * NT + wave * 64 >= TILE * GR) break;  // (32 channels: two waves' worth)
      const int key = slot / GR, pos = slot % GR;
      const int kg = pos ^ (k8_place<DP>(key, 0) >> 4) % GR, vg = pos ^ (v8_place<DP>(key, 0) >> 4) % GR;
      const long long from = (long long)(k0 + min(key, most_key)) * p.head_dim;
      if (16 * kg < p.head_dim) send16(kb + from + 16 * kg, t.k + first);
      if (16 * vg < p.head_dim) send16(vb + from + 16 * vg, t.v + first);
    }
    const int key = k0 + min(lane, most_key);
    if (wave == 0) send16(sites + key, t.sites);
    if (wave == 1) send4at(p.scales + k_row + key, t.ks);
    if (wave == 2) send4at(p.scales + v_row + key, t.vs);
  };

  f32x16 o[DP / 32];
#pragma unroll
  for (int n = 0; n < DP / 32; ++n)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[n][e] = 0.0f;
  float top = 0.0f, total = 0.0f;  // as in the kernel for few rows
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
    const int4 site = t.sites[lane];
    const bool held = tile * TILE + lane < p.capacity && site.w >= 0;
    const float vs = t.vs[lane];
    const uint64_t tokens = __ballot(held);
    const bool whole = __all(held && seen.all(site, bias));
    if (!__any(held && seen.some(site))) return;
    const bool careful = !whole && (tokens != ~0ull || __any(held && !(fabsf(vs) < INFINITY)));
    // (the waves write the same)
    notes.f[lane] = factor_of(p, t.ks[lane]);
    notes.v[lane] = held ? vs : 0.0f;
    notes.bytes[lane] = site_bytes(site);
    __builtin_amdgcn_wave_barrier();

    f32x16 z[2];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) z[n][e] = 0.0f;
#pragma unroll
    for (int c = 0; c < DP / 32; ++c) {
      const bf16x8 first = query(2 * c), second = query(2 * c + 1);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const uint4 w = *(const uint4*)(t.k + k_off[c] + 32 * n * DP);
        z[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode<INT8>(w.x, w.y), first, z[n], 0, 0, 0);
        z[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode<INT8>(w.z, w.w), second, z[n], 0, 0, 0);
      }
    }
    float size = 0.0f;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 f = *(const float4*)&notes.f[32 * n + 8 * g + 4 * half];
        z[n][4 * g] *= f.x, z[n][4 * g + 1] *= f.y, z[n][4 * g + 2] *= f.z, z[n][4 * g + 3] *= f.w;
        if constexpr (CAP != CAP_NONE) {
          size = fmaxf(fmaxf(size, fabsf(z[n][4 * g])), fabsf(z[n][4 * g + 1]));
          size = fmaxf(fmaxf(size, fabsf(z[n][4 * g + 2])), fabsf(z[n][4 * g + 3]));
        }
      }
    float most = -INFINITY;
    if (whole) {
      with_tier<CAP>(p, size, [&](auto tier) {
        auto scores = [&](auto biased) {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              uint4 w = make_uint4(0, 0, 0, 0);
              if constexpr (biased.value) w = *(const uint4*)&notes.bytes[32 * n + 8 * g + 4 * half];
              const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float part = biased.value ? near_part(u[e], at_bytes, slope * 0x1p24f, -top) : -top;
                z[n][4 * g + e] = score8<CAP, decltype(tier)::value>(p, z[n][4 * g + e], part);
                most = fmaxf(most, z[n][4 * g + e]);
              }
            }
        };
        if (bias)
          scores(std::true_type());
        else
          scores(std::false_type());
      });
    } else {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = 32 * n + 8 * (e >> 2) + 4 * half + (e & 3);
          const int4 k = t.sites[key];
          const bool in = tokens >> key & 1 && k.w == own_volume && k.x <= last;
          const float x = score8<CAP, 3>(p, z[n][e], bias ? fmaf((float)distance(at, k), slope, -top) : -top);
          z[n][e] = in ? x : -INFINITY;
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
    // probabilities, times the value's scale, in two bf16 parts, keys 16 s + 4 half + {0 .. 3, 8 .. 11}; and their product with the codes.  (In one part
    // the result's error against 64 bits was half as large again as its own rounding's, 0.0024 against 0.0016; the second part costs 228 us against 205,
    // 196 tokens against four caches of up to 200 rounds of d = 13, 8 (2) x 64 E4M3.)
    auto finish = [&](auto carefully) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        uint32_t u[4], ul[4], keep[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const float4 f4 = *(const float4*)&notes.v[16 * s + 8 * g + 4 * half];
          const float f[4] = {f4.x, f4.y, f4.z, f4.w};
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = z[s >> 1][8 * (s & 1) + 4 * g + e], e2 = __builtin_amdgcn_exp2f(y);
            total += e2;
            x[e] = e2 * f[e];
            if constexpr (carefully.value) x[e] = y == -INFINITY ? 0.0f : x[e];  // (an invisible row's scale may be anything)
          }
          split2(x[0], x[1], u[2 * g], ul[2 * g]);
          split2(x[2], x[3], u[2 * g + 1], ul[2 * g + 1]);
          // codes at places without a token may be E4M3's NaN
          if constexpr (carefully.value) keep[g] = byte_mask((uint32_t)(tokens >> (16 * s + 8 * g + 4 * half)));
        }
        const bf16x8 ph = __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3]));
        const bf16x8 pl = __builtin_bit_cast(bf16x8, make_uint4(ul[0], ul[1], ul[2], ul[3]));
#pragma unroll
        for (int m = 0; m < DP / 32; ++m) {
          i32x2 w = read_byte_columns(t.v + v_off[m] + 16 * s * DP);
          if constexpr (carefully.value) w[0] &= keep[0], w[1] &= keep[1];
          const bf16x8 v = decode<INT8>((uint32_t)w[0], (uint32_t)w[1]);
          o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pl, o[m], 0, 0, 0);
          o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, ph, o[m], 0, 0, 0);
        }
        if constexpr (LDS_Q) __builtin_amdgcn_sched_barrier(0);  // (reads of the next columns would spill)
      }
    };
    if (careful)
      finish(std::true_type());
    else
      finish(std::false_type());
  };

  int tile = next_tile(), buf = 0;
  if (tile >= 0) load_tile(tiles[0], tile);
  sent();
  __syncthreads();
  while (tile >= 0) {
    const int after = next_tile();
    if (after >= 0) load_tile(tiles[buf ^ 1], after);
    __builtin_amdgcn_sched_barrier(0);
    work(tiles[buf], tile);
    sent();
    __syncthreads();
    tile = after, buf ^= 1;
  }

  total += __shfl_xor(total, 32);
  if (row >= p.rows) return;
  if (p.splits > 1) {
    const bool none = unset && total == 0.0f;  // saw nothing (without a reference, but NaN scores: not nothing)
    const long long rows_at = (((long long)item.split * p.batch + b) * p.kv_heads + kvh) * p.rows;
    if (!none) {  // (the join does not read it otherwise)
#pragma unroll
      for (int m = 0; m < DP / 32; ++m)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(float4*)(p.part_o + (rows_at + row) * DP + 32 * m + 8 * g + 4 * half) = make_float4(o[m][4 * g], o[m][4 * g + 1], o[m][4 * g + 2], o[m][4 * g + 3]);
    }
    if (half == 0) p.part_ml[rows_at + row] = make_float2(none ? -INFINITY : top, total);
    return;
  }
  const float inv = inverse(total);
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
// DP / 4 lanes read a split's row, and the workgroup's groups of them take splits in turn.  A split in which the row saw
// nothing (m_s = -infinity) left no result, and is not read.  Any other one is, also where its weight is 0 in fp32: what it
// saw may be NaN, and so is the row then.
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
  const bool none = ml.x == -INFINITY;
  const float w = none ? 0.0f : __builtin_amdgcn_exp2f(ml.x - top);
  float total = none ? 0.0f : ml.y * w;
  weight[tid] = none ? -1.0f : w;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m);
  if ((tid & 63) == 0) sm[tid >> 6].y = total;
  __syncthreads();
  total = (sm[0].y + sm[1].y) + (sm[2].y + sm[3].y);
  float4 acc = make_float4(0, 0, 0, 0);
#pragma unroll 4
  for (int s = g; s < p.splits; s += GROUPS) {
    const float a = weight[s];
    const float4 o = a == -1.0f ? make_float4(0, 0, 0, 0) : *(const float4*)(p.part_o + (s * step + item) * DP + 4 * lane);
    acc.x = fmaf(o.x, a, acc.x), acc.y = fmaf(o.y, a, acc.y), acc.z = fmaf(o.z, a, acc.z), acc.w = fmaf(o.w, a, acc.w);
  }
  so[g][lane] = acc;
  __syncthreads();
  if (g != 0 || 4 * lane >= p.head_dim) return;
  for (int n = 1; n < GROUPS; ++n) {
    const float4 o = so[n][lane];
    acc.x += o.x, acc.y += o.y, acc.z += o.z, acc.w += o.w;
  }
  const float inv = inverse(total);
  uint2 v;
  v.x = bf16_pack(acc.x * inv, acc.y * inv), v.y = bf16_pack(acc.z * inv, acc.w * inv);
  *(uint2*)(p.out + b * p.o_b + row / p.group * p.o_t + (kvh * p.group + row % p.group) * p.o_h + 4 * lane) = v;
}

// The same for up to FEW_SPLITS splits of MANY_ROWS rows or more: a thread joins four columns of a row (6272 rows of 10 splits: 7.6 us, above 11;
// 32 rows of 31: 15 us, above 4).
constexpr int FEW_SPLITS = 32, MANY_ROWS = 2048;
template <int DP>
__global__ void __launch_bounds__(256) attention8_join_few_kernel(const Attn8 p) {
  constexpr int L = DP / 4;
  const long long step = (long long)p.batch * p.kv_heads * p.rows;
  const long long item = (long long)blockIdx.x * (256 / L) + threadIdx.x / L;  // (batch, kv_heads, rows)
  const int lane = threadIdx.x % L;
  if (item >= step || 4 * lane >= p.head_dim) return;
  float top = -INFINITY;
#pragma unroll 8
  for (int s = 0; s < p.splits; ++s) top = fmaxf(top, p.part_ml[s * step + item].x);
  float4 acc = make_float4(0, 0, 0, 0);
  float total = 0.0f;
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s) {
    const float2 ml = p.part_ml[s * step + item];
    const bool none = ml.x == -INFINITY;
    const float w = none ? 0.0f : __builtin_amdgcn_exp2f(ml.x - top);
    const float4 o = none ? make_float4(0, 0, 0, 0) : *(const float4*)(p.part_o + (s * step + item) * DP + 4 * lane);
    acc.x = fmaf(o.x, w, acc.x), acc.y = fmaf(o.y, w, acc.y), acc.z = fmaf(o.z, w, acc.z), acc.w = fmaf(o.w, w, acc.w);
    total = none ? total : fmaf(ml.y, w, total);
  }
  const int row = (int)(item % p.rows), kvh = (int)(item / p.rows % p.kv_heads), b = (int)(item / p.rows / p.kv_heads);
  const float inv = inverse(total);
  uint2 v;
  v.x = bf16_pack(acc.x * inv, acc.y * inv), v.y = bf16_pack(acc.z * inv, acc.w * inv);
  *(uint2*)(p.out + b * p.o_b + row / p.group * p.o_t + (kvh * p.group + row % p.group) * p.o_h + 4 * lane) = v;
}

// Threads of a workgroup.
constexpr int threads_of(bool few) { return (few ? FW : NW) * 64; }

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
  // (8 (2) heads of 64 against four caches of up to 200 rounds: 36 rows 46 us for few, 45 for many; 64 rows 34 and 47; 132 rows 81 and 80)
  n.few = rows <= 64;
  n.row_tiles = (int)((rows + (n.few ? 15 : 127)) / (n.few ? 16 : 128));
  n.tiles = (int)(((long long)c.capacity + TILE - 1) / TILE);
  const int dp = c.head_dim <= 32 ? 32 : c.head_dim <= 64 ? 64 : 128;
  // Splits: to fill the card (256 workgroups of eight waves, 512 of four), down to 8 tiles each.  (Two or three times as many cost more than
  // they even out: the token above 25 and 28 us against 19, the round 232 and 235 against 228.)
  const long long whole = n.row_tiles * heads, fill = n.few ? 256 : 512;
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
    // rows are counted in 32 bits, work items and rows of all heads by the launches (threads below 2^32, a join's 256 a row)
    if ((long long)a->n_q * (a->heads / c.kv_heads) >= 1ll << 30) return PD_ERR_UNSUPPORTED;
    const Plan n = plan_for(a);
    if (n.items > (1ll << 32) / threads_of(n.few) - 8 * RUN || (n.splits > 1 && (__int128)a->n_q * a->heads * c.batch >= 1ll << 24)) return PD_ERR_UNSUPPORTED;
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

template <int DP, bool INT8, Cap CAP>
void launch(const Attn8& p, bool few, hipStream_t st) {
  const dim3 blocks((p.items + 8 * RUN - 1) / (8 * RUN) * (8 * RUN)), threads(threads_of(few));
  if (few)
    hipLaunchKernelGGL((attention8_few_kernel<DP, INT8, CAP>), blocks, threads, 0, st, p);
  else
    hipLaunchKernelGGL((attention8_kernel<DP, INT8, CAP>), blocks, threads, 0, st, p);
}

template <int DP, bool INT8>
void launch_cap(const Attn8& p, bool few, Cap cap, hipStream_t st) {
  if (cap == CAP_NONE)
    launch<DP, INT8, CAP_NONE>(p, few, st);
  else if (cap == CAP_NEAR)
    launch<DP, INT8, CAP_NEAR>(p, few, st);
  else
    launch<DP, INT8, CAP_FAR>(p, few, st);
}

template <int DP>
void launch_width(const Attn8& p, const Plan& n, bool int8, Cap cap, hipStream_t st) {
  if (int8)
    launch_cap<DP, true>(p, n.few, cap, st);
  else
    launch_cap<DP, false>(p, n.few, cap, st);
  const unsigned rows = (unsigned)(p.kv_heads * p.batch) * p.rows;
  if (p.splits > 1 && p.splits <= FEW_SPLITS && rows >= MANY_ROWS)
    hipLaunchKernelGGL(attention8_join_few_kernel<DP>, dim3((rows + 1024 / DP - 1) / (1024 / DP)), dim3(256), 0, st, p);
  else if (p.splits > 1)
    hipLaunchKernelGGL(attention8_join_kernel<DP>, dim3(rows), dim3(256), 0, st, p);
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
  const float factor = cap == CAP_NEAR ? a->scale / most_cap : a->scale * LOG2E;
  p.factor = fminf(fmaxf(factor, -FLT_MAX), FLT_MAX);
  p.cap_a = -2.0f * most_cap * LOG2E, p.cap_b = most_cap * LOG2E, p.unit = cap == CAP_FAR ? 1.0f / p.cap_b : 0.0f;
  p.low[0] = p.cap_b * N1, p.low[1] = p.cap_b * N3, p.low[2] = p.cap_b * N5, p.low[3] = p.cap_b * N7;
  p.mid[0] = p.cap_b * M1, p.mid[1] = p.cap_b * M3, p.mid[2] = p.cap_b * M5, p.mid[3] = p.cap_b * M7, p.mid[4] = p.cap_b * M9;
  p.poly1 = p.cap_b * TANH1, p.poly3 = p.cap_b * TANH3, p.poly5 = p.cap_b * TANH5;
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
