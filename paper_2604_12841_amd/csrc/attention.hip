// attention.hip -- grouped-head attention over the tokens of detector volumes:
// scores capped by a tanh, a bias by the distance of the sites, masks by
// volume, round and prefix.
//
// One pass over the keys with the running maximum and sum of the softmax.  The
// heads that share keys are rows of one query matrix: row r is token
// r / group, head r % group of the key head's group.  A wave takes 32 rows, a
// workgroup 32, 64 or 128 (one, two or four waves), and tiles of keys come
// through LDS, two in turn: the next one is on its way there from memory while
// this one is worked on.  A wave computes the transposed scores K Q^T, so a lane holds
// half of the scores of one row (the other half of the wave the rest): maximum
// and sum need one exchange.  The same registers, rounded to bf16, are the
// right operand of out^T += V^T P^T, whose sum over keys may run in any order
// as long as V follows it; V is read transposed from LDS.
//
// What to read: a short kernel notes for every tile of 64 keys which volumes
// and rounds it holds (up to 256 keys are all read).  A workgroup skips tiles that none of its rows sees, and
// tiles that all rows of a wave see whole need no mask.
//
// Few rows against many keys: the keys are split over workgroups, each
// leaves its maximum, sum and unscaled result (fp32), and a last kernel joins them.
//
// Bound by vector instructions, 11.6 a score with cap and bias: 16 volumes of
// 2548 tokens, 8 query and 2 key heads of 64, 389 us (546 TFLOP/s; vector units
// 0.69, matrix units 0.24 busy).  One token against four caches of up to 39200:
// 27.6 us, the keys' part at 3.5 TB/s.
#include <float.h>
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>

#include "../../include/predecoder_ops.h"
#include "lds_tiles.h"
#include "token_scores.h"
#include "token_values.h"

namespace {

using namespace pd;

constexpr int TILE = 64;  // keys of a noted tile
constexpr int SHORT = 4 * TILE;  // up to as many keys: no notes, their sites stay in LDS
constexpr int RUN = 4;    // neighbouring work items of one XCD
constexpr int FEW_SPLITS = 32;  // up to as many: a row's splits that saw nothing leave no result
// What a tile of keys holds: the range of volumes and of rounds over its tokens (vmin > vmax: none).
struct Tile {
  int vmin, vmax, tmin, tmax;
  int flags;  // HOLES, BYTES
  int pad[3];
};
constexpr int HOLES = 1;  // a place holds no token
constexpr int BYTES = 2;  // rows and columns of all tokens are in [0, 255]

struct Attn {
  int batch, heads, kv_heads, group, head_dim;
  int n_q, n_k;
  int rows;  // n_q * group
  unsigned items;  // row_tiles * splits * kv_heads * batch
  int row_tiles, splits, tiles, tiles_per_split;
  int prefix_last;  // prefix - 1; INT_MIN, below every round: none
  int causal;
  bool plain_rows;  // the keys of a tile lie within 32-bit offsets, and head_dim fills the rows in LDS
  float c1;    // log2 units: without a cap z = c1 x; with it z = cap_b + cap_a / (1 + 2^(c1 x))
  float cap_a, cap_b;
  float small, poly1, poly3, poly5;  // |q.k| <= small (0.35 of the cap): CAP_NEAR's z = x (poly1 + x^2 (poly3 + x^2 poly5)) is the cap
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* out;
  long long q_b, q_t, q_h, k_b, k_t, k_h, v_b, v_t, v_h, o_b, o_t, o_h;
  const int4* q_sites;
  const int4* k_sites;
  long long q_sites_b, k_sites_b;
  const float* slopes;
  const Tile* notes;  // [lists][tiles] or null: nothing is skipped, every tile masked
  const uint32_t* bytes;  // with notes: site_bytes and ordered sites of every key, [lists][tiles][TILE]
  const uint4* ordered_sites;
  int notes_b;        // tiles from batch entry to batch entry
  // results of splits, [splits][batch][kv_heads][blocks of 32 rows (of all, if there are fewer)], four values each: few
  // splits: [DP / 4][block_rows], so that a wave writes whole lines; many: [block_rows][DP / 4], so that a row's join
  // reads whole lines
  float4* part_o;
  int blocks, block_rows, part_c, part_r;
  float2* part_ml;    // [splits][batch][kv_heads][rows]: maximum (log2 units), sum
  float unit, c0;  // CAP_FAR: scale / cap, and scale in log2 units
};

// A site as the kernel compares it: coordinates moved to unsigned numbers in the same order, volume -1 for no token.
__device__ __forceinline__ uint4 ordered(const int4 s) {
  const uint32_t sign = 0x80000000u;
  return make_uint4((uint32_t)s.x ^ sign, (uint32_t)s.y ^ sign, (uint32_t)s.z ^ sign, s.w < 0 ? ~0u : (uint32_t)s.w);
}

// Values 4 c .. 4 c + 3 of a row in part_o.
template <int DP>
__device__ __forceinline__ long long part_at(const Attn& p, int split, int b, int kvh, int row, int c) {
  const long long block = (((long long)split * p.batch + b) * p.kv_heads + kvh) * p.blocks + (row >> 5);
  return block * (DP / 4) * p.block_rows + c * p.part_c + (row & 31) * p.part_r;
}

// One wave a tile: what its 64 keys hold, and their sites in the forms that the kernel reads.
__global__ void __launch_bounds__(256) attention_notes_kernel(const int4* __restrict__ sites, long long sites_b, int n_k,
                                                              int tiles, Tile* __restrict__ notes,
                                                              uint32_t* __restrict__ bytes,
                                                              uint4* __restrict__ ordered_sites) {
  const int tile = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (tile >= tiles) return;
  const int key = tile * TILE + lane;
  const int4 s = key < n_k ? sites[blockIdx.y * sites_b + key] : make_int4(0, 0, 0, -1);
  const bool there = s.w >= 0;
  Tile t;
  t.vmin = wave_min(there ? s.w : INT_MAX);
  t.vmax = wave_max(there ? s.w : -1);
  t.tmin = wave_min(there ? s.x : INT_MAX);
  t.tmax = wave_max(there ? s.x : INT_MIN);
  t.flags = (__all(there) ? 0 : HOLES) | (__all(!there || (in_byte(s.y) && in_byte(s.z))) ? BYTES : 0);
  t.pad[0] = t.pad[1] = t.pad[2] = 0;
  const long long at = (long long)blockIdx.y * tiles + tile;
  if (lane == 0) notes[at] = t;
  bytes[at * TILE + lane] = site_bytes(s);
  ordered_sites[at * TILE + lane] = ordered(s);
}

template <int DP, int NW, Cap CAP, bool BIAS>
__global__ void __launch_bounds__(NW * 64, NW == 4 ? (DP == 128 ? 2 : 3) : NW == 2 && DP < 128 ? 2 : 1) attention_kernel(const Attn p) {
  constexpr int TK = NW == 1 ? 32 : 64;       // keys of a step
  constexpr int NT = NW * 64, ROWS = NW * 32;
  constexpr int STEPS = TILE / TK;            // steps of a noted tile
  constexpr int G = TK * (DP / 8) / NT;       // granules of K (and of V) that a thread stages
  constexpr int NB = TK / 32;                 // blocks of 32 keys
  __shared__ __attribute__((aligned(16))) uint8_t lk[2][TK * DP * 2];
  __shared__ __attribute__((aligned(16))) uint8_t lv[2][TK * DP * 2];
  // ordered sites and their bytes: with notes of the step's keys (at buf * TK); without, of all keys, or, if there are
  // no sites, of the last tile's, for its end
  __shared__ uint4 ls[SHORT];
  __shared__ __attribute__((aligned(16))) uint32_t lb[SHORT];
  __shared__ int lq[4][NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;

  // Workgroups are dealt to the eight XCDs in turn.  An XCD takes RUN
  // neighbouring items, which read the same keys, in its L2; longer runs would
  // leave XCDs idle where items see unequal numbers of keys.
  unsigned item = ((blockIdx.x >> 3) / RUN * 8 + (blockIdx.x & 7)) * RUN + (blockIdx.x >> 3) % RUN;
  if (item >= p.items) return;
  // (with rounds seen up to a row's own, later rows see more: they start first)
  const int row_tile = p.causal ? p.row_tiles - 1 - (int)(item % p.row_tiles) : (int)(item % p.row_tiles);
  item /= p.row_tiles;
  const int split = item % p.splits;
  item /= p.splits;
  const int kvh = item % p.kv_heads, b = item / p.kv_heads;

  const int row = row_tile * ROWS + wave * 32 + (lane & 31);
  const int r = row < p.rows ? row : p.rows - 1;  // rows past the end repeat the last: not stored
  const int token = r / p.group, head = kvh * p.group + r % p.group;
  const uint16_t* q = p.q + b * p.q_b + token * p.q_t + head * p.q_h;
  const uint16_t* kb = p.k + b * p.k_b + kvh * p.k_h;
  const uint16_t* vb = p.v + b * p.v_b + kvh * p.v_h;
  const int4* sites = p.k_sites ? p.k_sites + b * p.k_sites_b : nullptr;
  bf16x8 fq[DP / 16];
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    const int d = 16 * s + 8 * half;
    const uint4 w = d < p.head_dim ? *(const uint4*)(q + d) : make_uint4(0, 0, 0, 0);
    fq[s] = __builtin_bit_cast(bf16x8, w);
  }
  const int4 at = p.q_sites ? p.q_sites[b * p.q_sites_b + token] : make_int4(0, 0, 0, 0);
  const bool there = at.w >= 0;
  uint4 own = ordered(at);
  if (!there) own.w = ~1u;  // no key's volume
  // the last round that the row sees
  const uint32_t last = p.causal ? (uint32_t)max(at.x, p.prefix_last) ^ 0x80000000u : ~0u;
  const uint32_t at_bytes = site_bytes(at);
  // Finite slopes past 2^94 leave a row its nearest tokens alone (negative ones its farthest), as 2^94 does, whose products
  // with 2^24 (below) and with any distance stay finite.
  float slope = BIAS ? p.slopes[head] : 0.0f;
  if (fabsf(slope) < INFINITY) slope = fminf(fmaxf(slope * -LOG2E, -0x1p94f), 0x1p94f);

  // what this wave's rows see, and the workgroup's
  const int wv_min = wave_min(there ? at.w : INT_MAX), wv_max = wave_max(there ? at.w : -1);
  const int wt_min = wave_min(there ? at.x : INT_MAX), wt_max = wave_max(there ? at.x : INT_MIN);
  const bool w_plain = __all(there) && wv_min == wv_max;
  const bool w_bytes = (wt_min >> 8) == (wt_max >> 8) && __all(!there || (in_byte(at.y) && in_byte(at.z)));
  int gv_min = wv_min, gv_max = wv_max, gt_max = wt_max;
  if constexpr (NW > 1) {
    if (lane == 0) lq[0][wave] = wv_min, lq[1][wave] = wv_max, lq[2][wave] = wt_max;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      gv_min = min(gv_min, lq[0][w]);
      gv_max = max(gv_max, lq[1][w]);
      gt_max = max(gt_max, lq[2][w]);
    }
    gv_min = __builtin_amdgcn_readfirstlane(gv_min);
    gv_max = __builtin_amdgcn_readfirstlane(gv_max);
    gt_max = __builtin_amdgcn_readfirstlane(gt_max);
  }
  const Tile* notes = p.notes ? p.notes + (long long)b * p.notes_b : nullptr;
  const uint32_t* bytes = p.bytes + (long long)b * p.notes_b * TILE;
  const uint4* ordered_sites = p.ordered_sites + (long long)b * p.notes_b * TILE;
  auto meets = [&](const Tile& t, int vmin, int vmax, int tmax) {
    return t.vmin <= vmax && t.vmax >= vmin && (!p.causal || t.tmin <= tmax || t.tmin <= p.prefix_last);
  };

  // The tiles to visit, 64 at a time as a mask; each lane holds the note of its tile.
  const int end = min(p.tiles, (split + 1) * p.tiles_per_split);
  int base = split * p.tiles_per_split - 64;
  uint64_t mask = 0;
  Tile mine = {};
  auto note_of = [&](int tile) {
    Tile t;
    t.vmin = __builtin_amdgcn_readlane(mine.vmin, tile - base);
    t.vmax = __builtin_amdgcn_readlane(mine.vmax, tile - base);
    t.tmin = __builtin_amdgcn_readlane(mine.tmin, tile - base);
    t.tmax = __builtin_amdgcn_readlane(mine.tmax, tile - base);
    t.flags = __builtin_amdgcn_readlane(mine.flags, tile - base);
    return t;
  };
  auto next_tile = [&]() -> int {  // -1: no more
    while (mask == 0) {
      base += 64;
      if (base >= end) return -1;
      bool visit = base + lane < end;
      if (notes) {
        mine = notes[min(base + lane, end - 1)];
        // (nothing else is on its way here; waiting at once keeps waits for these registers off the loads sent next)
        __builtin_amdgcn_s_waitcnt(0x0f70);
        visit = visit && meets(mine, gv_min, gv_max, gt_max);
      }
      mask = __ballot(visit);
    }
    const int bit = __builtin_ctzll(mask);
    mask &= mask - 1;
    return base + bit;
  };

  // Staging, straight into LDS: granule slots tid + n NT of K and of V.  The
  // thread's keys are KEYS apart, and the column that goes to its slot differs
  // from n to n by an exclusive or alone.  Keys past the end repeat the last
  // (they are masked); columns past head_dim stay the zeros that they are set
  // to here.
  constexpr int KEYS = NT / (DP / 8);
  const int key0 = tid / (DP / 8), slot0 = tid % (DP / 8);
  auto k_column = [&](int n) {
    return (slot0 ^ (k_place<DP>(key0, 0) >> 4) % (DP / 8) ^ (k_place<DP>(KEYS * n, 0) >> 4) % (DP / 8)) * 8;
  };
  const int v_column = (slot0 ^ (v_place<DP>(key0, 0) >> 4) % (DP / 8)) * 8;
  static_assert(KEYS % 4 == 0 && (KEYS & (KEYS - 1)) == 0, "the turns of a thread's keys");
  // bytes from a step's first key to this thread's first one
  const uint32_t k_lane = (uint32_t)(key0 * p.k_t) * 2u, v_lane = (uint32_t)(key0 * p.v_t + v_column) * 2u;
  if (p.head_dim < DP) {
    for (int c = tid; c < TK * (DP / 8); c += NT)
#pragma unroll
      for (int n = 0; n < 2; ++n)
        *(uint4*)(lk[n] + c * 16) = *(uint4*)(lv[n] + c * 16) = make_uint4(0, 0, 0, 0);
    __syncthreads();
  }
  auto load_step = [&](int buf, int k0) {
    const int most_key = p.n_k - 1 - k0;
    const uint16_t* ks = kb + k0 * p.k_t;
    const uint16_t* vs = vb + k0 * p.v_t;
    if (most_key >= TK - 1 && p.plain_rows) {
#pragma unroll
      for (int n = 0; n < G; ++n) {
        const int slot = (n * NT + wave * 64) * 16;
        const int kc = k_column(n);
        const char* const kn = (const char*)(ks + n * KEYS * p.k_t);
        const char* const vn = (const char*)(vs + n * KEYS * p.v_t);
        send16(kn, k_lane + 2u * kc, lk[buf] + slot);
        send16(vn, v_lane, lv[buf] + slot);
      }
    } else {
#pragma unroll
      for (int n = 0; n < G; ++n) {
        const int slot = (n * NT + wave * 64) * 16;
        const int kc = k_column(n);
        const long long key = min(key0 + n * KEYS, most_key);
        if (kc < p.head_dim) send16(ks + key * p.k_t + kc, lk[buf] + slot);
        if (v_column < p.head_dim) send16(vs + key * p.v_t + v_column, lv[buf] + slot);
      }
    }
    if (notes && wave == 0 && lane < TK) send16(ordered_sites + k0, 16u * lane, ls + buf * TK);
    if (BIAS && notes && wave == NW - 1 && lane < TK) send4(bytes + k0, 4u * lane, lb + buf * TK);
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
  const int vkey = (lane & 15) >> 2;  // of four keys
  int v_off[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m)
    v_off[m] = v_place<DP>(vkey, 4 * m + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) + (lane & 1) * 8 + 4 * half * DP * 2;
  int k_off[DP / 16];
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) k_off[s] = k_place<DP>(lane & 31, 2 * s + half);

  if (!notes) {
    const int first = sites ? 0 : max(p.n_k - 1, 0) / TILE * TILE;
    for (int key = tid; key < (sites ? SHORT : TILE); key += NT) {
      int4 s = make_int4(0, 0, 0, first + key < p.n_k ? 0 : -1);
      if (sites && key < p.n_k) s = sites[key];
      ls[key] = ordered(s);
      lb[key] = site_bytes(s);
    }
  }
  int tile = next_tile(), step = 0, buf = 0;
  Tile note = {};
  if (tile >= 0) {
    note = note_of(tile);
    load_step(0, tile * TILE);
  }
  sent();
  __syncthreads();
  while (tile >= 0) {
    int after = tile, after_step = step + 1;
    if (after_step == STEPS || tile * TILE + after_step * TK >= p.n_k) after = next_tile(), after_step = 0;
    Tile after_note = note;
    if (after >= 0) {
      if (after_step == 0) after_note = note_of(after);
      load_step(buf ^ 1, after * TILE + after_step * TK);
    }
    __builtin_amdgcn_sched_barrier(0);

    const int at_step = notes ? buf * TK : (sites ? tile * TILE : 0) + step * TK;  // where the step's sites are
    if (!notes || meets(note, wv_min, wv_max, wt_max)) {
      f32x16 z[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
#pragma unroll
        for (int e = 0; e < 16; ++e) z[n][e] = 0.0f;
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
          const uint4 w = *(const uint4*)(lk[buf] + k_off[s] + 32 * n * DP * 2);
          z[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), fq[s], z[n], 0, 0, 0);
        }
      }
      const float off = (CAP == CAP_NEAR ? p.cap_b : 0.0f) - top, off_small = -top;
      // whether a score of the wave's tile exceeds 0.35 of the cap
      auto large = [&] {
        float size = 0.0f;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 16; e += 2) size = fmaxf(fmaxf(size, fabsf(z[n][e])), fabsf(z[n][e + 1]));
        return __any(size > p.small);
      };
      if constexpr (CAP == CAP_FAR) {
        auto far_capped = [&](auto some_large) {
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float x = z[n][e], u = x * p.unit, w = u * u;
              z[n][e] = x * p.c0 * fmaf(w, fmaf(w, fmaf(w, TANH7R, TANH5R), TANH3R), 1.0f);
              if constexpr (some_large.value) {
                const float part = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * p.c1));
                z[n][e] = fabsf(x) <= p.small ? z[n][e] : fmaf(p.cap_a, part, p.cap_b);
              }
              if ((e & 3) == 3) __builtin_amdgcn_sched_barrier(0);  // four scores' parts in registers at a time
            }
        };
        if (large())
          far_capped(std::true_type());
        else
          far_capped(std::false_type());
      }
      auto capped = [&](float x, float t) {
        if constexpr (CAP == CAP_NEAR)
          return fmaf(p.cap_a, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * p.c1)), t);
        else if constexpr (CAP == CAP_FAR)
          return x + t;
        else
          return fmaf(x, p.c1, t);
      };
      // the score in log2 units, relative to the reference; dist: the sites' distance
      auto score = [&](float x, uint32_t dist) {
        const float t = BIAS ? fmaf((float)dist, slope, off) : off;
        return capped(x, t);
      };
      // dist < 2^10 as an fp16 number below the normal range is dist 2^-24: the mixed multiply-add takes it as it is
      auto score_near = [&](float x, uint32_t dist) {
        const float t = BIAS ? fmaf((float)__builtin_bit_cast(_Float16, (uint16_t)dist), slope * 0x1p24f, off) : off;
        return capped(x, t);
      };
      // the same where no score of the wave's tile exceeds 0.35 of the cap: four instructions instead of five, of which
      // two run at half rate
      auto score_small = [&](float x, uint32_t dist) {
        const float t = BIAS ? fmaf((float)__builtin_bit_cast(_Float16, (uint16_t)dist), slope * 0x1p24f, off_small) : off_small;
        const float w = x * x;
        return fmaf(x, fmaf(w, fmaf(w, p.poly5, p.poly3), p.poly1), t);
      };
      float most = -INFINITY;
      bool whole;  // every row sees every key, and the bytes give the distances
      if (notes) {
        whole = !(note.flags & HOLES) && w_plain && note.vmin == note.vmax && note.vmin == wv_min &&
                (!p.causal || note.tmax <= wt_min || note.tmax <= p.prefix_last) &&
                (!BIAS || (w_bytes && (note.flags & BYTES) && (note.tmin >> 8) == (wt_min >> 8) &&
                           (note.tmax >> 8) == (wt_min >> 8)));
      } else if (!sites) {
        whole = p.n_k - tile * TILE >= TILE;
      } else {
        const uint4 s = ls[at_step + (lane & (TK - 1))];
        const uint32_t t0 = (uint32_t)wt_min ^ 0x80000000u, seen_by_all = p.causal ? (uint32_t)max(wt_min, p.prefix_last) ^ 0x80000000u : ~0u;
        whole = w_plain && __all(s.w == (uint32_t)wv_min && s.x <= seen_by_all &&
                                 (!BIAS || ((s.x ^ t0) < 256u && (s.y ^ 0x80000000u) < 256u && (s.z ^ 0x80000000u) < 256u)));
        if (BIAS && !w_bytes) whole = false;
      }
      auto scores = [&](auto&& score_of) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            uint4 w = make_uint4(0, 0, 0, 0);
            if constexpr (BIAS) w = *(const uint4*)&lb[at_step + 32 * n + 8 * g + 4 * half];
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = score_of(z[n][4 * g + e], BIAS ? __builtin_amdgcn_sad_u8(u[e], at_bytes, 0) : 0);
              z[n][4 * g + e] = x;
              most = fmaxf(most, x);
            }
          }
      };
      if (whole) {
        if constexpr (CAP == CAP_NEAR) {
          if (large())
            scores(score_near);
          else
            scores(score_small);
        } else {
          scores(score_near);
        }
      } else {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint4 key = ls[at_step + 32 * n + 8 * (e >> 2) + 4 * half + (e & 3)];
            uint32_t dist = 0;
            if constexpr (BIAS) dist = far_add(own.x, key.x, far_add(own.y, key.y, far_add(own.z, key.z, 0)));
            const float x = score(z[n][e], dist);
            const bool seen = key.w == own.w && key.x <= last;
            z[n][e] = seen ? x : -INFINITY;
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
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) z[n][e] -= up;
      }
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) z[n][e] = __builtin_amdgcn_exp2f(z[n][e]);
      bool odd = false;  // an infinity or a NaN in V where rows see some keys only
      if (!whole) {
        uint32_t carry = 0;
#pragma unroll
        for (int n = 0; n < TK * (DP / 8) / 64; ++n) {
          const uint4 w = *(const uint4*)(lv[buf] + (lane + 64 * n) * 16);
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) carry |= (u[e] & 0x7f807f80u) + 0x00800080u;  // an exponent of ones carries
        }
        odd = __any((carry & 0x80008000u) != 0);
      }
      // the probabilities in bf16, which the matrix instruction takes, keys 16 s + 4 half + {0 .. 3, 8 .. 11} of block n;
      // and the sum of the rounded ones, with which equal values come out as they are
      uint4 pr[NB][2];
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          uint32_t u[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            u[e] = bf16_pack(z[n][8 * s + 2 * e], z[n][8 * s + 2 * e + 1]);
            total = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, u[e]),
                                                    __builtin_bit_cast(bf16x2, 0x3f803f80u), total, false);
          }
          pr[n][s] = make_uint4(u[0], u[1], u[2], u[3]);
        }
      // V^T of those keys: four keys of 16 columns from each 16 lanes' reads, of which a lane gets its column's
      auto values = [&](int n, int s, int m) {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const uint8_t* f = lv[buf] + v_off[m] + (32 * n + 16 * s) * DP * 2;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)f);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(f + 8 * DP * 2));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      };
      // what a bf16 value is: 0 finite, 1 / 2 positive / negative infinity, 3 NaN
      auto kind_of = [](int bits) { return (bits & 0x7f80) != 0x7f80 ? 0 : bits & 0x7f ? 3 : bits >> 15 ? 2 : 1; };
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          s16x8 a[DP / 32];
#pragma unroll
          for (int m = 0; m < DP / 32; ++m) a[m] = values(n, s, m);
          if (odd) {
#pragma unroll
            for (int m = 0; m < DP / 32; ++m)
#pragma unroll
              for (int e = 0; e < 8; ++e) a[m][e] = kind_of((uint16_t)a[m][e]) ? 0 : a[m][e];
          }
#pragma unroll
          for (int m = 0; m < DP / 32; ++m)
            o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[m]),
                                                           __builtin_bit_cast(bf16x8, pr[n][s]), o[m], 0, 0, 0);
        }
      if (odd) {
        // 0 x infinity: the finite values are in; now, for each kind of others, whether a row sees one in a column
#pragma unroll 1
        for (int kind = 1; kind < 4; ++kind) {
          const float other = kind == 1 ? INFINITY : kind == 2 ? -INFINITY : NAN;
#pragma unroll
          for (int m = 0; m < DP / 32; ++m) {
            f32x16 there;
#pragma unroll
            for (int e = 0; e < 16; ++e) there[e] = 0.0f;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
              for (int s = 0; s < 2; ++s) {
                s16x8 a = values(n, s, m);
#pragma unroll
                for (int e = 0; e < 8; ++e) a[e] = kind_of((uint16_t)a[e]) == kind ? 0x3f80 : 0;  // 1 or 0
                there = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                                __builtin_bit_cast(bf16x8, pr[n][s]), there, 0, 0, 0);
              }
#pragma unroll
            for (int e = 0; e < 16; ++e) o[m][e] += there[e] != 0.0f ? other : 0.0f;
          }
        }
      }
    }
    sent();
    __syncthreads();
    tile = after, step = after_step, buf ^= 1, note = after_note;
  }

  total += __shfl_xor(total, 32);
  if (row >= p.rows) return;
  if (p.splits > 1) {
    const long long at_row = (((long long)split * p.batch + b) * p.kv_heads + kvh) * p.rows + row;
    const bool none = unset && total == 0.0f;  // saw nothing (without a reference, but NaN scores: not nothing)
    if (!none || p.splits > FEW_SPLITS) {      // (the join of many reads them all at once)
      float4* part = p.part_o + part_at<DP>(p, split, b, kvh, row, half);
#pragma unroll
      for (int m = 0; m < DP / 32; ++m)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          part[(8 * m + 2 * g) * p.part_c] =
              make_float4(o[m][4 * g], o[m][4 * g + 1], o[m][4 * g + 2], o[m][4 * g + 3]);
    }
    if (half == 0) p.part_ml[at_row] = make_float2(none ? -INFINITY : top, total);
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

// Values 4 lane .. 4 lane + 3 of a row.
__device__ __forceinline__ void store_joined(const Attn& p, int b, int kvh, int row, int lane, float4 acc, float total) {
  const float inv = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : NAN;
  const int token = row / p.group, head = kvh * p.group + row % p.group;
  uint2 v;
  v.x = bf16_pack(acc.x * inv, acc.y * inv), v.y = bf16_pack(acc.z * inv, acc.w * inv);
  *(uint2*)(p.out + b * p.o_b + token * p.o_t + head * p.o_h + 4 * lane) = v;
}

// Joins the splits of one row: out = sum 2^(m_s - m) o_s / sum 2^(m_s - m) l_s.
// The weights first, one split a thread; then DP / 4 lanes read a split's row, and the workgroup's groups of them take
// splits in turn.
constexpr int MOST_SPLITS = 256;

template <int DP>
__global__ void __launch_bounds__(256) attention_join_kernel(const Attn p) {
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
    const float4 o = p.part_o[part_at<DP>(p, s, b, kvh, row, lane)];
    acc.x = fmaf(o.x, a, acc.x), acc.y = fmaf(o.y, a, acc.y), acc.z = fmaf(o.z, a, acc.z), acc.w = fmaf(o.w, a, acc.w);
  }
  so[g][lane] = acc;
  __syncthreads();
  if (g != 0 || 4 * lane >= p.head_dim) return;
  for (int n = 1; n < GROUPS; ++n) {
    const float4 o = so[n][lane];
    acc.x += o.x, acc.y += o.y, acc.z += o.z, acc.w += o.w;
  }
  store_joined(p, b, kvh, row, lane, acc, total);
}

// The same for up to FEW_SPLITS splits: a workgroup joins a block of 32 rows, one split after the other.
template <int DP>
__global__ void __launch_bounds__(256) attention_join_few_kernel(const Attn p) {
  const int r = threadIdx.x & 31, c0 = threadIdx.x >> 5;
  const unsigned group = blockIdx.x / p.blocks;  // (batch, kv_heads)
  const int kvh = group % p.kv_heads, b = group / p.kv_heads, row = (int)(blockIdx.x % p.blocks) * 32 + r;
  if (row >= p.rows) return;
  const long long step = (long long)p.batch * p.kv_heads * p.rows, item = (long long)group * p.rows + row;
  float top = -INFINITY;
  for (int s = 0; s < p.splits; ++s) top = fmaxf(top, p.part_ml[s * step + item].x);
  float4 acc[DP / 32];
#pragma unroll
  for (int n = 0; n < DP / 32; ++n) acc[n] = make_float4(0, 0, 0, 0);
  float total = 0.0f;
  for (int s = 0; s < p.splits; ++s) {
    const float2 ml = p.part_ml[s * step + item];
    if (ml.x == -INFINITY) continue;  // the row saw nothing there
    const float w = __builtin_amdgcn_exp2f(ml.x - top);
    const float4* part = p.part_o + part_at<DP>(p, s, b, kvh, row, c0);
#pragma unroll
    for (int n = 0; n < DP / 32; ++n) {
      const float4 o = part[8 * n * p.part_c];
      acc[n].x = fmaf(o.x, w, acc[n].x), acc[n].y = fmaf(o.y, w, acc[n].y);
      acc[n].z = fmaf(o.z, w, acc[n].z), acc[n].w = fmaf(o.w, w, acc[n].w);
    }
    total = fmaf(ml.y, w, total);
  }
#pragma unroll
  for (int n = 0; n < DP / 32; ++n)
    if (4 * (c0 + 8 * n) < p.head_dim) store_joined(p, b, kvh, row, c0 + 8 * n, acc[n], total);
}

// How a call runs.
struct Plan {
  int waves;  // of a workgroup: 1, 2 or 4
  int row_tiles, tiles, splits, tiles_per_split;
  bool notes;
  size_t notes_bytes, bytes_bytes, sites_bytes, o_bytes, ml_bytes;
  long long items;
};

Plan plan_for(const pd_attention_args* a) {
  Plan n = {};
  const long long group = a->heads / a->kv_heads, rows = a->n_q * group;
  // workgroups of 64 rows where those of 128 would leave over a tenth of their rows empty
  const long long full4 = (rows + 127) / 128 * 128, full2 = (rows + 63) / 64 * 64;
  n.waves = rows <= 32 ? 1 : 10 * (full4 - full2) > full4 ? 2 : 4;
  n.row_tiles = (int)((rows + 32 * n.waves - 1) / (32 * n.waves));
  n.tiles = (int)(((long long)a->n_k + TILE - 1) / TILE);
  // a few tiles are read whole: the notes' launch would cost more than it saves
  n.notes = a->k_sites && a->n_k > SHORT;
  const long long heads = (long long)a->kv_heads * a->batch, whole = n.row_tiles * heads;
  // Splits: to fill the card once (512 workgroups of four waves, or 2048 waves of few rows), down to 8 (2) tiles each;
  // and, while they keep 32 tiles, until there are eight times as many, which evens out rows that see unequal numbers of tiles.  A
  // split's result costs about as much as 5 tiles of its rows.
  const long long fill = 2048 / n.waves, even = 8 * 512 * 4 / n.waves;
  const long long least = n.waves == 1 ? 2 : 8;
  long long splits = (fill + whole - 1) / whole;
  if (splits > n.tiles / least) splits = n.tiles / least;
  long long more = (even + whole - 1) / whole;
  if (more > n.tiles / 32) more = n.tiles / 32;
  if (splits < more) splits = more;
  if (splits > MOST_SPLITS) splits = MOST_SPLITS;
  const int dp = a->head_dim <= 32 ? 32 : a->head_dim <= 64 ? 64 : 128;
  const long long most = (1ll << 30) / (dp * 4) / heads / rows;  // 1 GB of workspace (the product could pass 64 bits)
  if (splits > most) splits = most;
  if (splits < 1) splits = 1;
  n.tiles_per_split = (int)((n.tiles + splits - 1) / splits);
  if (n.tiles_per_split < 1) n.tiles_per_split = 1;
  n.splits = n.tiles ? (n.tiles + n.tiles_per_split - 1) / n.tiles_per_split : 1;
  const long long lists = a->k_sites_batch_stride ? a->batch : 1;
  n.notes_bytes = n.notes ? (size_t)lists * n.tiles * sizeof(Tile) : 0;
  n.bytes_bytes = n.notes ? (size_t)lists * n.tiles * TILE * 4 : 0;
  n.sites_bytes = 4 * n.bytes_bytes;
  const long long part_rows = rows < 32 ? rows : (rows + 31) / 32 * 32;
  n.o_bytes = n.splits > 1 ? (size_t)n.splits * heads * part_rows * dp * 4 : 0;
  n.ml_bytes = n.splits > 1 ? (size_t)n.splits * heads * rows * 8 : 0;
  n.items = whole * n.splits;
  return n;
}

bool rows16(const void* p, long long b, long long t, long long h) {
  return (uintptr_t)p % 16 == 0 && b % 8 == 0 && t % 8 == 0 && h % 8 == 0;
}

// The argument checks: sizes alone, or with the pointers.
pd_status check(const pd_attention_args* a, bool pointers) {
  if (!a || a->batch < 0 || a->heads < 0 || a->kv_heads < 0 || a->n_q < 0 || a->n_k < 0) return PD_ERR_INVALID_ARG;
  if (a->head_dim < 1 || !(fabsf(a->scale) < INFINITY) || !(a->cap >= 0.0f) || !(a->cap < INFINITY))
    return PD_ERR_INVALID_ARG;
  if (a->causal < 0 || a->causal > 1) return PD_ERR_INVALID_ARG;
  if (a->prefix != PD_PREFIX_NONE && (a->prefix < 0 || (a->prefix && !a->causal))) return PD_ERR_INVALID_ARG;
  if (a->heads && (!a->kv_heads || a->heads % a->kv_heads)) return PD_ERR_INVALID_ARG;
  if (a->head_dim % 8 || a->head_dim > 128) return PD_ERR_UNSUPPORTED;
  if (a->heads && a->heads / a->kv_heads > 64) return PD_ERR_UNSUPPORTED;
  if (a->kv_heads > 65535 || a->batch > 65535) return PD_ERR_UNSUPPORTED;  // the grid's axes
  if (a->heads && a->batch && a->n_q) {
    // rows are counted in 32 bits, work items and rows of all heads by the launches (threads below 2^32)
    if ((long long)a->n_q * (a->heads / a->kv_heads) >= 1ll << 30) return PD_ERR_UNSUPPORTED;
    const Plan n = plan_for(a);
    if (n.items > (1ll << 24) - 8 * RUN || (n.splits > 1 && (long long)a->n_q * a->heads * a->batch >= 1ll << 24))
      return PD_ERR_UNSUPPORTED;
  }
  if (!pointers || !a->batch || !a->heads || !a->n_q) return PD_OK;
  if (!a->q || !a->out || (a->n_k && (!a->k || !a->v))) return PD_ERR_INVALID_ARG;
  // (the sites of no keys may have no address)
  if (a->n_k && !a->q_sites != !a->k_sites) return PD_ERR_INVALID_ARG;
  if (!a->q_sites && (a->slopes || a->causal || a->k_sites)) return PD_ERR_INVALID_ARG;
  if ((uintptr_t)a->q_sites % 16 || (uintptr_t)a->k_sites % 16 || (uintptr_t)a->slopes % 4) return PD_ERR_INVALID_ARG;
  if (!rows16(a->q, a->q_batch_stride, a->q_token_stride, a->q_head_stride) ||
      !rows16(a->k, a->k_batch_stride, a->k_token_stride, a->k_head_stride) ||
      !rows16(a->v, a->v_batch_stride, a->v_token_stride, a->v_head_stride) ||
      !rows16(a->out, a->out_batch_stride, a->out_token_stride, a->out_head_stride))
    return PD_ERR_UNSUPPORTED;
  // rows of out may not overlap
  if (!rows_apart(a->head_dim, {{a->batch, a->out_batch_stride}, {a->n_q, a->out_token_stride}, {a->heads, a->out_head_stride}}))
    return PD_ERR_INVALID_ARG;
  const size_t need = predecoder_attention_workspace(a);
  if (need && (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < need)) return PD_ERR_INVALID_ARG;
  return PD_OK;
}

}  // namespace

extern "C" size_t predecoder_attention_workspace(const pd_attention_args* a) {
  if (check(a, false) != PD_OK || !a->batch || !a->heads || !a->n_q) return 0;
  const Plan n = plan_for(a);
  return n.o_bytes + n.notes_bytes + n.bytes_bytes + n.sites_bytes + n.ml_bytes;
}

namespace {

template <int DP, int NW, Cap CAP>
void launch_cap(const Attn& p, bool bias, unsigned items, hipStream_t st) {
  if (bias)
    hipLaunchKernelGGL((attention_kernel<DP, NW, CAP, true>), dim3(items), dim3(NW * 64), 0, st, p);
  else
    hipLaunchKernelGGL((attention_kernel<DP, NW, CAP, false>), dim3(items), dim3(NW * 64), 0, st, p);
}

template <int DP, int NW>
void launch(const Attn& p, Cap cap, bool bias, unsigned items, hipStream_t st) {
  if (cap == CAP_NONE)
    launch_cap<DP, NW, CAP_NONE>(p, bias, items, st);
  else if (cap == CAP_NEAR)
    launch_cap<DP, NW, CAP_NEAR>(p, bias, items, st);
  else
    launch_cap<DP, NW, CAP_FAR>(p, bias, items, st);
}

template <int DP>
void launch_width(const Attn& p, const Plan& n, Cap cap, bool bias, hipStream_t st) {
  const unsigned blocks = (p.items + 8 * RUN - 1) / (8 * RUN) * (8 * RUN);
  if (n.waves == 1)
    launch<DP, 1>(p, cap, bias, blocks, st);
  else if (n.waves == 2)
    launch<DP, 2>(p, cap, bias, blocks, st);
  else
    launch<DP, 4>(p, cap, bias, blocks, st);
  if (p.splits > 1)
  {
    const unsigned groups = (unsigned)(p.kv_heads * p.batch);
    if (p.splits <= FEW_SPLITS)
      hipLaunchKernelGGL(attention_join_few_kernel<DP>, dim3(groups * p.blocks), dim3(256), 0, st, p);
    else
      hipLaunchKernelGGL(attention_join_kernel<DP>, dim3(groups * p.rows), dim3(256), 0, st, p);
  }
}

}  // namespace

extern "C" pd_status predecoder_attention(void* hip_stream, const pd_attention_args* a) {
  const pd_status ok = check(a, true);
  if (ok != PD_OK) return ok;
  if (!a->batch || !a->heads || !a->n_q) return PD_OK;
  const Plan n = plan_for(a);
  Attn p;
  p.batch = a->batch, p.heads = a->heads, p.kv_heads = a->kv_heads, p.group = a->heads / a->kv_heads;
  p.head_dim = a->head_dim;
  p.n_q = a->n_q, p.n_k = a->n_k, p.rows = a->n_q * p.group;
  p.items = (unsigned)n.items, p.row_tiles = n.row_tiles, p.splits = n.splits, p.tiles = n.tiles, p.tiles_per_split = n.tiles_per_split;
  p.prefix_last = a->prefix == PD_PREFIX_NONE ? INT_MIN : a->prefix - 1, p.causal = a->causal;
  const Cap cap = !(a->cap > 0.0f) ? CAP_NONE : a->cap <= MOST_NEAR ? CAP_NEAR : CAP_FAR;
  // (caps past 2^126, whose double would leave the range, differ from it for scores that are themselves of such size alone)
  const float most_cap = fminf(a->cap, 0x1p126f);
  // kept finite, so that scores of zero stay zero; at the bounds any other score is past the cap, or past all of its row
  auto finite = [](float c) { return fminf(fmaxf(c, -FLT_MAX), FLT_MAX); };
  p.c1 = finite(a->cap > 0.0f ? a->scale * 2.0f * LOG2E / most_cap : a->scale * LOG2E);
  if (a->cap > 0.0f) {
    const float u = a->scale / most_cap, c = most_cap * LOG2E;
    p.small = 0.35f / fabsf(u);
    if (cap == CAP_NEAR) p.small = fminf(p.small, 0x1p60f);  // its polynomial takes the square
    p.poly1 = c * u * TANH1, p.poly3 = c * u * u * u * TANH3, p.poly5 = c * u * u * u * u * u * TANH5;
    if (cap == CAP_NEAR && !(fabsf(p.poly1) + fabsf(p.poly3) + fabsf(p.poly5) < INFINITY))
      p.small = -1.0f;  // 0 x infinity
  } else {
    p.small = p.poly1 = p.poly3 = p.poly5 = 0.0f;
  }
  p.cap_a = -2.0f * most_cap * LOG2E, p.cap_b = most_cap * LOG2E;
  p.unit = a->cap > 0.0f ? finite(a->scale / most_cap) : 0.0f, p.c0 = finite(a->scale * LOG2E);
  p.q = (const uint16_t*)a->q, p.k = (const uint16_t*)a->k, p.v = (const uint16_t*)a->v, p.out = (uint16_t*)a->out;
  p.q_b = a->q_batch_stride, p.q_t = a->q_token_stride, p.q_h = a->q_head_stride;
  p.k_b = a->k_batch_stride, p.k_t = a->k_token_stride, p.k_h = a->k_head_stride;
  p.v_b = a->v_batch_stride, p.v_t = a->v_token_stride, p.v_h = a->v_head_stride;
  p.o_b = a->out_batch_stride, p.o_t = a->out_token_stride, p.o_h = a->out_head_stride;
  p.q_sites = (const int4*)a->q_sites, p.k_sites = (const int4*)a->k_sites;
  p.q_sites_b = a->q_sites_batch_stride, p.k_sites_b = a->k_sites_batch_stride;
  p.slopes = a->slopes;
  auto near = [](long long t) { return t >= 0 && t < (1ll << 24); };
  p.plain_rows = near(p.k_t) && near(p.v_t) && (p.head_dim == 32 || p.head_dim == 64 || p.head_dim == 128);
  p.part_o = (float4*)a->workspace;
  p.blocks = (p.rows + 31) / 32, p.block_rows = p.rows < 32 ? p.rows : 32;
  const bool few = n.splits <= FEW_SPLITS;
  p.part_c = few ? p.block_rows : 1;
  p.part_r = few ? 1 : (a->head_dim <= 32 ? 32 : a->head_dim <= 64 ? 64 : 128) / 4;
  Tile* notes = (Tile*)((char*)a->workspace + n.o_bytes);
  uint32_t* bytes = (uint32_t*)((char*)notes + n.notes_bytes);
  uint4* ordered_sites = (uint4*)((char*)bytes + n.bytes_bytes);
  p.part_ml = (float2*)((char*)ordered_sites + n.sites_bytes);
  p.notes = n.notes ? notes : nullptr;
  p.bytes = bytes, p.ordered_sites = ordered_sites;
  p.notes_b = a->k_sites_batch_stride ? n.tiles : 0;
  const hipStream_t st = (hipStream_t)hip_stream;
  if (n.notes) {
    const unsigned lists = a->k_sites_batch_stride ? (unsigned)a->batch : 1u;
    hipLaunchKernelGGL(attention_notes_kernel, dim3((unsigned)(n.tiles + 3) / 4, lists), dim3(256), 0, st, p.k_sites,
                       p.k_sites_b, p.n_k, p.tiles, notes, bytes, ordered_sites);
  }
  const bool bias = a->slopes != nullptr;
  if (a->head_dim <= 32)
    launch_width<32>(p, n, cap, bias, st);
  else if (a->head_dim <= 64)
    launch_width<64>(p, n, cap, bias, st);
  else
    launch_width<128>(p, n, cap, bias, st);
  return hipGetLastError() == hipSuccess ? PD_OK : PD_ERR_DEVICE;
}
