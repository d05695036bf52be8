// linear_attention.hip -- linear attention with a decay for each head, over
// rounds of tokens:
//   S_t = exp(-slope) S_(t-1) + sum over the tokens m of round t of k_m v_m^T
//   out_n = scale q_n S_t(n)
//
// Chunked form.  S stays in registers, in blocks over the waves of a workgroup;
// tiles of 64 (48) tokens of K and V come through LDS, two in turn, and S += K^T V with
// both operands read transposed.  As the left operand of out^T = S^T q^T a copy
// of S goes to LDS, in two bf16 parts (16 bits).  Heads of more than 64 channels: a workgroup holds
// 64 of the value's, so that two fit a CU.
//   Wide rounds (more than 32 tokens): S takes a whole round in, then the round's
//   queries read it, beside the next round's tiles: no token sees a part of a
//   round, so there are no pairs.  One stream of 1000 rounds of 196 tokens, 8 query
//   and 2 key heads of 128: 216 to 235 us (1.0 GB, 4.5 TB/s; matrix units 0.25, LDS 0.5 busy); 64 volumes
//   of 13 such rounds, 8 heads of 64, in one pass: 165 us, 4.0 TB/s.
//   Narrow rounds: a tile holds as many whole rounds as fit.  Its queries read S from
//   before the tile, decayed, and the tile's keys in pairs:
//   out_i = w^(t_i + 1) q_i S + sum over t_j <= t_i of w^(t_i - t_j) (q_i.k_j) v_j;
//   then S = w^R S + sum of w^(R - 1 - t_j) k_j v_j^T.  The weighted keys are split
//   into three bf16 parts (24 bits: two would leave the state off by 2^-18 of itself), weighted pairs into
//   two.  8 rows of up to 4097 single-token rounds, 6 heads of 64: 33 us, a chain of latencies
//   for each tile (vector units 0.33, LDS 0.34 busy).
//
// Few entries and heads against many rounds: the rounds are cut into segments.
// A first pass leaves each segment's own S (64 and 14 us above), a scan turns them into the S that
// each segment starts from (13 and 6 us), and the last pass runs the segments side by side.
//
// Recurrent form (one token an entry): S is read, updated, multiplied by q and
// written by threads that hold four columns of some rows.  256 entries, 8 heads of 128:
// 51 us, 5.3 TB/s, the rate of a large copy.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>

#include "../../include/predecoder_ops.h"
#include "lds_tiles.h"
#include "token_values.h"

namespace {

using namespace pd;

constexpr float LOG2E = 1.4426950408889634f;
constexpr int NARROW = 32;  // a round of up to as many tokens shares its tile with others

struct Linear {
  int batch, heads, kv_heads, group, head_dim, n, per_round;
  int tile_rounds;  // narrow rounds: of a tile
  int tile_tokens;  // narrow rounds: tile_rounds per_round; else a tile's
  int segments;
  int segment_rounds;  // narrow rounds: a multiple of tile_rounds
  float scale;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* out;
  long long q_b, q_t, q_h, k_b, k_t, k_h, v_b, v_t, v_h, o_b, o_t, o_h;
  const float* slopes;
  const int* lengths;
  const float* state;
  float* state_out;
  float* starts;  // [batch][kv_heads][segments][head_dim][head_dim]
};

__device__ __forceinline__ int length_of(const Linear& p, int b) { return p.lengths ? min(max(p.lengths[b], 0), p.n) : p.n; }

// exp(-slope rounds) as a sum of two numbers: a decay is applied once a round, and what its rounding loses would add up.
struct Fade {
  float hi, lo;
};
__device__ __forceinline__ Fade fade_of(const Linear& p, int kvh, int rounds) {
  const double f = p.slopes && rounds ? exp(-(double)p.slopes[kvh] * rounds) : 1.0;
  Fade r;
  r.hi = (float)f;
  r.lo = fabsf(r.hi) < INFINITY ? (float)(f - (double)r.hi) : 0.0f;
  return r;
}
__device__ __forceinline__ float faded(float s, Fade f, float add) { return fmaf(s, f.hi, fmaf(s, f.lo, add)); }

__device__ __forceinline__ float bf16_of(uint32_t bits16) { return __uint_as_float(bits16 << 16); }

// A workgroup holds all rows of S (the key's channels, padded to DP) and VP of its columns (the value's channels).
template <int DP>
struct Shape {
  static constexpr int VP = DP == 128 ? 64 : DP;
  static constexpr int TILE = DP == 128 ? 48 : 64;      // tokens: two workgroups' tiles and S fit a CU's LDS
  static constexpr int KB = DP / 32, VB = VP / 32;      // blocks of 32 channels
  static constexpr int NW = DP == 32 ? 1 : 4;           // waves
  static constexpr int NBW = KB * VB / NW;              // blocks of S of a wave
  static constexpr int NT = NW * 64;
};

// This workgroup's segment, key head and entry, and its first column of S; false: none.
// (Workgroups are dealt to the eight XCDs in turn: the two that share a segment's queries and keys go to one, for its L2.)
template <int DP>
__device__ __forceinline__ bool item_of(const Linear& p, int& segment, int& kvh, int& b, int& v0) {
  constexpr int VP = Shape<DP>::VP;
  const int item = VP == DP ? blockIdx.x : (blockIdx.x >> 4) * 8 + (blockIdx.x & 7);
  v0 = VP == DP ? 0 : VP * ((blockIdx.x >> 3) & 1);
  segment = item % p.segments, kvh = item / p.segments % p.kv_heads, b = item / p.segments / p.kv_heads;
  return item < p.batch * p.kv_heads * p.segments;
}

// Sends for W columns from `first` on of tokens at .. at + TILE - 1, straight into LDS: granule slots tid + n NT, of which
// place() tells the turn.  Tokens past the tile's end repeat its last; columns past D are left as they are.
template <int TILE, int W, int NT, typename F>
__device__ __forceinline__ void send_rows(const uint16_t* rows, long long stride, uint8_t* to, int first, bool full, int D, long long at, int valid,
                                          int tid, int wave, F&& place) {
  constexpr int GR = W / 8;  // granules of a row
#pragma unroll
  for (int n = 0; n < (TILE * GR + NT - 1) / NT; ++n) {
    if (n * NT + wave * 64 >= TILE * GR) break;
    const int slot = tid + n * NT, key = slot / GR, c = first + (slot % GR ^ (place(key) >> 4) % GR) * 8;
    const uint16_t* const from = rows + (at + min(key, valid - 1)) * stride + c;
    if (full)
      send16(from, to + (n * NT + wave * 64) * 16);
    else if (c < D)
      send16(from, to + (n * NT + wave * 64) * 16);
  }
}

// Wide rounds.  OUT: the results of a segment from the S that it starts from; otherwise its own S.
template <int DP, bool OUT>
__global__ void __launch_bounds__(Shape<DP>::NT, 2) linear_kernel(const Linear p) {
  using Sh = Shape<DP>;
  constexpr int VP = Sh::VP, TILE = Sh::TILE, KB = Sh::KB, VB = Sh::VB, NW = Sh::NW, NBW = Sh::NBW, NT = Sh::NT;
  __shared__ __attribute__((aligned(16))) uint8_t lk[2][TILE * DP * 2];
  __shared__ __attribute__((aligned(16))) uint8_t lv[2][TILE * VP * 2];
  __shared__ __attribute__((aligned(16))) uint8_t ls[OUT ? 2 : 1][OUT ? VP * DP * 2 : 16];  // S^T in two parts, rows placed as K's
  __shared__ __attribute__((aligned(16))) uint8_t lo[OUT ? NW : 1][OUT ? 32 * 64 : 16];  // 32 columns of a unit's results
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  int segment, kvh, b, v0;
  if (!item_of<DP>(p, segment, kvh, b, v0)) return;
  const int D = p.head_dim, len = length_of(p, b);
  const long long first = (long long)segment * p.segment_rounds * p.per_round;  // tokens of this segment
  const long long last = min((long long)len, first + (long long)p.segment_rounds * p.per_round);
  const long long state_at = (long long)(b * p.kv_heads + kvh) * D * D;
  float* const own = p.starts + (state_at * p.segments + (long long)segment * D * D);
  const int dkb = wave % KB, dvb = wave / KB * NBW;

  f32x16 S[NBW];
  {
    const float* from = !OUT ? nullptr : p.segments > 1 ? own : p.state ? p.state + state_at : nullptr;
#pragma unroll
    for (int j = 0; j < NBW; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int dk = 32 * dkb + 8 * (e >> 2) + 4 * half + (e & 3), dv = v0 + 32 * (dvb + j) + (lane & 31);
        S[j][e] = from ? from[min(dk, D - 1) * D + min(dv, D - 1)] : 0.0f;
        if (dk >= D || dv >= D) S[j][e] = 0.0f;
      }
  }
  auto store_state = [&](float* to) {
#pragma unroll
    for (int j = 0; j < NBW; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int dk = 32 * dkb + 8 * (e >> 2) + 4 * half + (e & 3), dv = v0 + 32 * (dvb + j) + (lane & 31);
        if (dk < D && dv < D) to[dk * D + dv] = S[j][e];
      }
  };
  const Fade fade = fade_of(p, kvh, 1);

  const uint16_t* kb = p.k + b * p.k_b + kvh * p.k_h;
  const uint16_t* vb = p.v + b * p.v_b + kvh * p.v_h;
  // columns past head_dim stay the zeros that they are set to here
  if (D < DP) {
    for (int c = tid; c < 2 * TILE * (DP / 8); c += NT) *(uint4*)(lk[0] + c * 16) = make_uint4(0, 0, 0, 0);
    for (int c = tid; c < 2 * TILE * (VP / 8); c += NT) *(uint4*)(lv[0] + c * 16) = make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  auto load_tile = [&](int buf, long long at, int valid) {
    send_rows<TILE, DP, NT>(kb, p.k_t, lk[buf], 0, D == DP, D, at, valid, tid, wave, [](int key) { return k_place<DP>(key, 0); });
    send_rows<TILE, VP, NT>(vb, p.v_t, lv[buf], v0, D == DP, D, at, valid, tid, wave, [](int key) { return v_place<VP>(key, 0); });
  };
  // LDS places of this lane's transposed operands: four tokens from 4 half on, and eight on from there
  const int vkey = (lane & 15) >> 2, vgran = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1), vbyte = (lane & 1) * 8;
  const int k_tr[2] = {k_place<DP>(vkey + 4 * half, 4 * dkb + vgran) + vbyte, k_place<DP>(vkey + 4 * half + 8, 4 * dkb + vgran) + vbyte};
  auto v_tr = [&](int block, int hi) { return v_place<VP>(vkey, 4 * block + vgran) + vbyte + (4 * half + 8 * hi) * VP * 2; };
  auto columns = [&](const uint8_t* f, const uint8_t* g) {
    return __builtin_shufflevector(read_columns(f), read_columns(g), 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // token 16 s + 4 half + {0 .. 3, 8 .. 11} of elements 0 .. 7
  auto token_of = [&](int s, int e) { return 16 * s + 4 * half + (e & 3) + 8 * (e >> 2); };

  // S = fade S + K^T V over the tile's tokens
  auto update = [&](int buf, int valid, bool begins, Fade f) {
    if (begins) {
#pragma unroll
      for (int j = 0; j < NBW; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) S[j][e] = faded(S[j][e], f, 0.0f);
    }
#pragma unroll(OUT ? 1 : 2)
    for (int s = 0; s < TILE / 16; ++s) {
      if (16 * s >= valid) break;
      s16x8 a = columns(lk[buf] + k_tr[0] + 16 * s * DP * 2, lk[buf] + k_tr[1] + 16 * s * DP * 2);
      s16x8 v[NBW];
#pragma unroll
      for (int j = 0; j < NBW; ++j) v[j] = columns(lv[buf] + v_tr(dvb + j, 0) + 16 * s * VP * 2, lv[buf] + v_tr(dvb + j, 1) + 16 * s * VP * 2);
      if (16 * s + 16 > valid) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool in = token_of(s, e) < valid;
          a[e] = in ? a[e] : 0;
#pragma unroll
          for (int j = 0; j < NBW; ++j) v[j][e] = in ? v[j][e] : 0;
        }
      }
#pragma unroll
        for (int j = 0; j < NBW; ++j)
          S[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, v[j]), S[j], 0, 0, 0);
    }
  };
  auto share_state = [&] {
#pragma unroll
    for (int j = 0; j < NBW; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint2 hi, lo;
        split2(S[j][4 * g], S[j][4 * g + 1], hi.x, lo.x);
        split2(S[j][4 * g + 2], S[j][4 * g + 3], hi.y, lo.y);
        const int at = k_place<DP>(32 * (dvb + j) + (lane & 31), 4 * dkb + g) + 8 * half;
        *(uint2*)(ls[0] + at) = hi;
        *(uint2*)(ls[OUT ? 1 : 0] + at) = lo;
      }
  };

  // The results of the queries of tokens at .. at + tokens - 1: rows token * group + head, 32 of them a unit.  The
  // queries of a wave's next unit are on their way while it works on one; fetch() sends for those of the first.
  int unit = 0;  // this wave's next
  u32x4 next_q[DP / 16];
  // (a division by the group: of the unit's first row, the same for all lanes, and of less than 128 by a product)
  const int group_part = 65536 / p.group + 1;
  auto token_at = [&](int unit, int lane_row, int& i, int& head) {
    const int first = unit * 32, from = first / p.group, x = first - from * p.group + lane_row, more = x * group_part >> 16;
    i = from + more, head = kvh * p.group + x - more * p.group;
  };
  // (four lanes read 64 bytes of a row: 16 rows a load; single rows' lanes lie apart in the products' operands)
  auto fetch_unit = [&](long long at, int tokens, int unit) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      int i, head;
      token_at(unit, min(16 * j + lane / 4, tokens * p.group - 1 - unit * 32), i, head);
      const uint16_t* q = p.q + b * p.q_b + (at + i) * p.q_t + head * p.q_h;
#pragma unroll
      for (int s = 0; s < DP / 32; ++s)  // (past head_dim anything of the row will do: S is 0 there)
        next_q[2 * s + j] = *(const u32x4*)(q + min(32 * s + 8 * (lane & 3), D - 8));
    }
  };
  auto granule = [&](int r, int g) { return lo[wave] + (r * 4 + (g ^ (r >> 2 & 3))) * 16; };  // 32 rows of 64 bytes
  auto units_of = [&](int tokens) { return (tokens * p.group + 31) / 32; };
  auto fetch = [&](long long at, int tokens) {
    unit = wave;
    if (wave < units_of(tokens)) fetch_unit(at, tokens, wave);
  };
  // `most` of them.  (The next tile is waited for before the first result is stored: later, the wait would be for the stores too.)
  auto results = [&](long long at, int tokens, int most) {
    const int rows = tokens * p.group, units = units_of(tokens);
#pragma unroll 1
    for (int done = 0; done < most && unit < units; ++done, unit += NW) {
      bf16x8 fq[DP / 16];
#pragma unroll
      for (int s = 0; s < DP / 32; ++s) {
#pragma unroll
        for (int j = 0; j < 2; ++j) *(u32x4*)granule(16 * j + lane / 4, lane & 3) = next_q[2 * s + j];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < 2; ++j) fq[2 * s + j] = __builtin_bit_cast(bf16x8, *(const u32x4*)granule(lane & 31, 2 * j + half));
        __builtin_amdgcn_wave_barrier();
      }
      if (unit + NW < units) fetch_unit(at, tokens, unit + NW);
      __builtin_amdgcn_sched_barrier(0);
      f32x16 o[VB];
#pragma unroll
      for (int m = 0; m < VB; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[m][e] = 0.0f;
      // (the parts of S are read a step ahead of the products that take them)
      uint4 part[2][VB][2];
      auto read_parts = [&](int s) {
#pragma unroll
        for (int m = 0; m < VB; ++m)
#pragma unroll
          for (int n = 0; n < 2; ++n) part[s & 1][m][n] = *(const uint4*)(ls[OUT ? n : 0] + k_place<DP>(32 * m + (lane & 31), 2 * s + half));
      };
      read_parts(0);
#pragma unroll
      for (int s = 0; s < DP / 16; ++s) {
        if (s + 1 < DP / 16) read_parts(s + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 1; n >= 0; --n)
#pragma unroll
          for (int m = 0; m < VB; ++m)
            o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, part[s & 1][m][n]), fq[s], o[m], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (done == 0) sent();
      // Lanes hold 8 bytes of a row here and there: through LDS, 32 columns at a time, they get 16 bytes each of whole pieces.
#pragma unroll
      for (int m = 0; m < VB; ++m) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          uint2 w;
          w.x = bf16_pack(o[m][4 * g] * p.scale, o[m][4 * g + 1] * p.scale);
          w.y = bf16_pack(o[m][4 * g + 2] * p.scale, o[m][4 * g + 3] * p.scale);
          *(uint2*)(granule(lane & 31, g) + 8 * half) = w;
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int r = lane / 4 + 16 * n, rr = unit * 32 + r, d = v0 + 32 * m + 8 * (lane & 3);
          const uint4 w = *(const uint4*)granule(r, lane & 3);
          int ri, rh;
          token_at(unit, r, ri, rh);
          if (rr < rows && d < D) *(uint4*)(p.out + b * p.o_b + (at + ri) * p.o_t + rh * p.o_h + d) = w;
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
  };

  // The tiles: [at, at + valid), which do not cross a round's end.
  auto tile_end = [&](long long at, long long round_end) { return (int)(min(min(at + TILE, round_end), last) - at); };
  long long at = first, round_end = first + p.per_round;
  int buf = 0, valid = 0;
  if (at < last) {
    valid = tile_end(at, round_end);
    load_tile(0, at, valid);
  }
  sent();
  __syncthreads();
  long long round_at = at;
  long long due_at = at;  // the tokens whose results are to come from the S in LDS
  int due = 0;
  while (at < last) {
    const long long next = at + valid;
    const bool ends = next == round_end || next == last;
    const long long next_end = next == round_end ? round_end + p.per_round : round_end;
    int next_valid = 0;
    if (next < last) {
      next_valid = tile_end(next, next_end);
      load_tile(buf ^ 1, next, next_valid);
    }
    __builtin_amdgcn_sched_barrier(0);
    update(buf, valid, at == round_at, fade);
    if constexpr (OUT) {
      // a share of the round before's results with each tile of this one
      const int left = (int)((min(round_end, last) - at + TILE - 1) / TILE), mine = (units_of(due) - unit + NW - 1) / NW;
      if (mine > 0)
        results(due_at, due, (mine + left - 1) / left);
      else
        sent();
      if (ends) {
        __syncthreads();  // S of the round before is read
        share_state();
        due_at = round_at, due = (int)(next - round_at);
        fetch(due_at, due);
      }
    } else {
      sent();
    }
    __syncthreads();
    if (ends) round_at = next;
    at = next, valid = next_valid, round_end = next_end, buf ^= 1;
  }
  if constexpr (OUT) results(due_at, due, INT_MAX);
  if constexpr (!OUT)
    store_state(own);
  else if (p.segments == 1 && p.state_out)
    store_state(p.state_out + state_at);
}

// Narrow rounds: a tile holds whole rounds.  Products of 16 x 16 blocks, so that a tile's few queries keep the waves busy:
// lane (c, g) of a block's result holds column c = lane & 15 and rows 4 g + {0 .. 3}, g = lane >> 4.
// OUT: the results of a segment from the S that it starts from; otherwise its own S.
template <int DP, bool OUT>
__global__ void __launch_bounds__(256, 2) linear_narrow_kernel(const Linear p) {
  constexpr int VP = Shape<DP>::VP, TILE = Shape<DP>::TILE, NT = 256, NW = 4;
  constexpr int NK = DP / 16 > NW ? DP / 16 / NW : 1, NV = DP == 32 ? 1 : VP / 16;  // blocks of S of a wave: NK x NV
  constexpr int STEPS = DP / 32;                                                    // of a product over the key's channels
  constexpr int PARTS = (TILE + 31) / 32;                                           // of a tile: 32 tokens
  __shared__ __attribute__((aligned(16))) uint8_t lk[2][TILE * DP * 2];
  __shared__ __attribute__((aligned(16))) uint8_t lv[2][TILE * VP * 2];
  __shared__ __attribute__((aligned(16))) uint8_t ls[OUT ? 2 : 1][OUT ? VP * DP * 2 : 16];  // S^T in two parts, rows placed as K's
  __shared__ __attribute__((aligned(16))) uint8_t lo[OUT ? NW : 1][OUT ? 16 * 64 : 16];     // 32 columns of a unit's results
  __shared__ __attribute__((aligned(16))) float lt[64];                                     // round of a tile's token, or NEVER
  __shared__ __attribute__((aligned(16))) float lw[64];                                     // what its key counts for after the tile
  __shared__ float lp[65];                                                                  // decay over that many rounds
  __shared__ int odd_flag[2];
  constexpr float NEVER = 1e30f;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g4 = lane >> 4;
  int segment, kvh, b, v0;
  if (!item_of<DP>(p, segment, kvh, b, v0)) return;
  const int D = p.head_dim, len = length_of(p, b);
  const long long first = (long long)segment * p.segment_rounds * p.per_round;  // tokens of this segment
  const long long last = min((long long)len, first + (long long)p.segment_rounds * p.per_round);
  const long long state_at = (long long)(b * p.kv_heads + kvh) * D * D;
  float* const own = p.starts + (state_at * p.segments + (long long)segment * D * D);
  const int dk0 = 16 * (DP == 32 ? wave & 1 : wave * NK), dv0 = DP == 32 ? 16 * (wave >> 1) : 0;  // of this wave's blocks

  f32x4 S[NK][NV];
  {
    const float* from = !OUT ? nullptr : p.segments > 1 ? own : p.state ? p.state + state_at : nullptr;
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int dk = dk0 + 16 * i + 4 * g4 + e, dv = v0 + dv0 + 16 * j + c;
          S[i][j][e] = from ? from[min(dk, D - 1) * D + min(dv, D - 1)] : 0.0f;
          if (dk >= D || dv >= D) S[i][j][e] = 0.0f;
        }
  }
  // Slopes past 2^60 leave a row its own round, as 2^60 does; zero rounds stay 0.
  const float slope = p.slopes ? fminf(fmaxf(p.slopes[kvh] * -LOG2E, -0x1p60f), 0x1p60f) : 0.0f;
  const Fade fade = fade_of(p, kvh, p.tile_rounds);
  const uint16_t* kb = p.k + b * p.k_b + kvh * p.k_h;
  const uint16_t* vb = p.v + b * p.v_b + kvh * p.v_h;
  // columns past head_dim stay the zeros that they are set to here
  if (D < DP) {
    for (int i = tid; i < 2 * TILE * (DP / 8); i += NT) *(uint4*)(lk[0] + i * 16) = make_uint4(0, 0, 0, 0);
    for (int i = tid; i < 2 * TILE * (VP / 8); i += NT) *(uint4*)(lv[0] + i * 16) = make_uint4(0, 0, 0, 0);
  }
  for (int i = tid; i <= 64; i += NT) lp[i] = p.slopes && i ? (float)exp(-(double)p.slopes[kvh] * i) : 1.0f;
  if (tid < 2) odd_flag[tid] = 0;
  __syncthreads();
  auto rounds_of = [&](int tokens) { return (tokens + p.per_round - 1) / p.per_round; };
  // the tokens' rounds and weights in a tile of so many
  auto weigh = [&](int tokens) {
    if (tid < 64) {
      const int t = tid / p.per_round;
      lt[tid] = tid < tokens ? (float)t : NEVER;
      lw[tid] = lp[max(rounds_of(tokens) - 1 - t, 0)];
    }
  };
  auto load_tile = [&](int buf, long long at, int valid) {
    send_rows<TILE, DP, NT>(kb, p.k_t, lk[buf], 0, D == DP, D, at, valid, tid, wave, [](int key) { return k_place<DP>(key, 0); });
    send_rows<TILE, VP, NT>(vb, p.v_t, lv[buf], v0, D == DP, D, at, valid, tid, wave, [](int key) { return v_place<VP>(key, 0); });
  };
  // notes an infinity or a NaN in V, once this thread's granules have landed
  auto note_odd = [&](int buf) {
    uint32_t carry = 0;
#pragma unroll
    for (int n = 0; n < (TILE * (VP / 8) + NT - 1) / NT; ++n) {
      if (n * NT + wave * 64 >= TILE * (VP / 8)) break;
      const uint4 w = *(const uint4*)(lv[buf] + (tid + n * NT) * 16);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) carry |= (u[e] & 0x7f807f80u) + 0x00800080u;  // an exponent of ones carries
    }
    if (carry & 0x80008000u) odd_flag[buf] = 1;
  };
  // Transposed operands: columns 16 block + c of tokens 32 s + 4 g4 + {0 .. 3} and, elements 4 .. 7, 16 on from there.
  const int t_row = 4 * g4 + (c >> 2), t_gran = (c >> 1) & 1, t_byte = (c & 1) * 8;
  auto columns = [&](const uint8_t* f, int half_tile) {
    return __builtin_shufflevector(read_columns(f), read_columns(f + half_tile), 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // (places repeat every 16 rows; where a tile ends with the first 16, they stand for the others too, which count for nothing)
  auto second = [&](int s) { return 32 * s + 16 < TILE ? 16 : 0; };
  auto k_columns = [&](int buf, int channel, int s) {
    return columns(lk[buf] + k_place<DP>(t_row, channel / 8 + t_gran) + t_byte + 32 * s * DP * 2, second(s) * DP * 2);
  };
  auto v_columns = [&](int buf, int channel, int s) {
    return columns(lv[buf] + v_place<VP>(t_row, channel / 8 + t_gran) + t_byte + 32 * s * VP * 2, second(s) * VP * 2);
  };
  auto token_of = [&](int s, int e) { return 32 * s + 4 * g4 + (e & 3) + 16 * (e >> 2); };

  // S = fade S + K^T V over the tile's tokens, the keys weighted
  auto update = [&](int buf, int valid, Fade f) {
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[i][j][e] = faded(S[i][j][e], f, 0.0f);
#pragma unroll
    for (int s = 0; s < PARTS; ++s) {
      s16x8 v[NV];
#pragma unroll
      for (int j = 0; j < NV; ++j) v[j] = v_columns(buf, dv0 + 16 * j, s);
      const float4 w0 = *(const float4*)&lw[32 * s + 4 * g4], w1 = *(const float4*)&lw[32 * s + 4 * g4 + 16];
      const float w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
      const bool cut = 32 * s + 32 > valid;
      if (cut) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int j = 0; j < NV; ++j) v[j][e] = token_of(s, e) < valid ? v[j][e] : 0;
      }
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        s16x8 a = k_columns(buf, dk0 + 16 * i, s);
        if (cut) {
#pragma unroll
          for (int e = 0; e < 8; ++e) a[e] = token_of(s, e) < valid ? a[e] : 0;
        }
        uint32_t part[3][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = bf16_of((uint16_t)a[2 * e]) * w[2 * e], y = bf16_of((uint16_t)a[2 * e + 1]) * w[2 * e + 1];
          part[0][e] = bf16_pack(x, y);
          const float x1 = x - __uint_as_float(part[0][e] << 16), y1 = y - __uint_as_float(part[0][e] & 0xffff0000u);
          split2(x1, y1, part[1][e], part[2][e]);
        }
#pragma unroll
        for (int n = 2; n >= 0; --n)
#pragma unroll
          for (int j = 0; j < NV; ++j)
            S[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, make_uint4(part[n][0], part[n][1], part[n][2], part[n][3])), __builtin_bit_cast(bf16x8, v[j]), S[i][j], 0, 0, 0);
      }
    }
  };
  auto share_state = [&] {
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        uint2 hi, lo;
        split2(S[i][j][0], S[i][j][1], hi.x, lo.x);
        split2(S[i][j][2], S[i][j][3], hi.y, lo.y);
        const int at = k_place<DP>(dv0 + 16 * j + c, (dk0 + 16 * i) / 8 + (g4 >> 1)) + 8 * (g4 & 1);
        *(uint2*)(ls[0] + at) = hi;
        *(uint2*)(ls[OUT ? 1 : 0] + at) = lo;
      }
  };

  // The results of a tile's queries: rows token * group + head, 16 of them a unit, which the waves take in turn.  The queries of a
  // wave's next unit are on their way while it works on one, and those of the next tile's first (fetch()) for a whole tile.
  u32x4 first_q[STEPS], next_q[STEPS];
  const int group_part = 65536 / p.group + 1;
  // (a division by the group: of the unit's first row, the same for all lanes, and of less than 128 by a product)
  auto token_at = [&](int unit, int of_unit, int& i, int& head) {
    const int from = 16 * unit / p.group, x = 16 * unit - from * p.group + of_unit, more = x * group_part >> 16;
    i = from + more, head = kvh * p.group + x - more * p.group;
  };
  auto fetch_unit = [&](u32x4 (&to)[STEPS], long long at, int tokens, int unit) {
    // (four lanes read 64 bytes of a row; a row's lanes lie apart in the products' operands)
    int i, head;
    token_at(unit, min(lane / 4, tokens * p.group - 1 - 16 * unit), i, head);
    const uint16_t* q = p.q + b * p.q_b + (at + i) * p.q_t + head * p.q_h;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) to[s] = *(const u32x4*)(q + min(32 * s + 8 * (lane & 3), D - 8));  // (past head_dim S and the keys are 0)
  };
  auto granule = [&](int r, int g) { return lo[wave] + (r * 4 + (g ^ (r >> 2 & 3))) * 16; };  // 16 rows of 64 bytes
  auto units_of = [&](int tokens) { return (tokens * p.group + 15) / 16; };
  auto fetch = [&](long long at, int tokens) {
    if (wave < units_of(tokens)) fetch_unit(first_q, at, tokens, wave);
  };
  // (the next tile is waited for before the first result is stored: later, the wait would be for the stores too)
  auto results = [&](int buf, long long at, int tokens) {
    const int rows = tokens * p.group, units = units_of(tokens);
    const bool odd = __any(odd_flag[buf] != 0);
#pragma unroll 1
    for (int unit = wave; unit < units; unit += NW) {
      bf16x8 fq[STEPS];
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        *(u32x4*)granule(lane / 4, lane & 3) = next_q[s];
        __builtin_amdgcn_wave_barrier();
        fq[s] = __builtin_bit_cast(bf16x8, *(const u32x4*)granule(c, g4));
        __builtin_amdgcn_wave_barrier();
      }
      if (unit + NW < units) fetch_unit(next_q, at, tokens, unit + NW);
      int i, head, i_end, head_end;
      token_at(unit, min(c, rows - 1 - 16 * unit), i, head);
      token_at(unit, min(15, rows - 1 - 16 * unit), i_end, head_end);
      const float ti = lt[i], before = lp[(int)ti + 1], t_end = lt[i_end];
      f32x4 o[VP / 16];
#pragma unroll
      for (int m = 0; m < VP / 16; ++m) o[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int n = 1; n >= 0; --n)
#pragma unroll
          for (int m = 0; m < VP / 16; ++m) {
            const uint4 w = *(const uint4*)(ls[OUT ? n : 0] + k_place<DP>(16 * m + c, 4 * s + g4));
            o[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), fq[s], o[m], 0, 0, 0);
          }
#pragma unroll
      for (int m = 0; m < VP / 16; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[m][e] *= before;
#pragma unroll 1
      for (int part = 0; part < PARTS; ++part) {
        if (__any(lt[32 * part] > t_end)) break;  // later rounds than the unit's
        f32x4 z[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          z[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int s = 0; s < STEPS; ++s) {
            const uint4 w = *(const uint4*)(lk[buf] + k_place<DP>(min(32 * part + 16 * n, TILE - 16) + c, 4 * s + g4));
            z[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), fq[s], z[n], 0, 0, 0);
          }
        }
        uint32_t hi[4], lo2[4];
        float far[2][4];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const float4 t = *(const float4*)&lt[32 * part + 16 * n + 4 * g4];
          far[n][0] = ti - t.x, far[n][1] = ti - t.y, far[n][2] = ti - t.z, far[n][3] = ti - t.w;
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = far[n][e] >= 0.0f ? z[n][e] * __builtin_amdgcn_exp2f(slope * far[n][e]) : 0.0f;
          split2(x[0], x[1], hi[2 * n], lo2[2 * n]);
          split2(x[2], x[3], hi[2 * n + 1], lo2[2 * n + 1]);
        }
        const bf16x8 ph = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
        const bf16x8 pl = __builtin_bit_cast(bf16x8, make_uint4(lo2[0], lo2[1], lo2[2], lo2[3]));
#pragma unroll
        for (int m = 0; m < VP / 16; ++m) {
          s16x8 v = v_columns(buf, 16 * m, part);
          if (odd) {
            // 0 x infinity: values that are not finite count as 0, and then make the rows that see them NaN
            s16x8 there, ones;
            f32x4 count = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              there[e] = (v[e] & 0x7f80) == 0x7f80 ? 0x3f80 : 0;
              v[e] = there[e] ? 0 : v[e];
              ones[e] = far[e >> 2][e & 3] >= 0.0f ? 0x3f80 : 0;
            }
            count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, there), __builtin_bit_cast(bf16x8, ones), count, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[m][e] = count[e] != 0.0f ? NAN : o[m][e];
          }
          o[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), pl, o[m], 0, 0, 0);
          o[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), ph, o[m], 0, 0, 0);
        }
      }
      if (unit == wave) sent();
      // Lanes hold 8 bytes of a row here and there: through LDS, 32 columns at a time, they get 16 bytes each of whole pieces.
#pragma unroll
      for (int m = 0; m < VP / 32; ++m) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          uint2 w;
          w.x = bf16_pack(o[2 * m + n][0] * p.scale, o[2 * m + n][1] * p.scale);
          w.y = bf16_pack(o[2 * m + n][2] * p.scale, o[2 * m + n][3] * p.scale);
          *(uint2*)(granule(c, 2 * n + (g4 >> 1)) + 8 * (g4 & 1)) = w;
        }
        __builtin_amdgcn_wave_barrier();
        const int r = lane >> 2, d = v0 + 32 * m + 8 * (lane & 3);
        const uint4 w = *(const uint4*)granule(r, lane & 3);
        int ri, rh;
        token_at(unit, r, ri, rh);
        if (16 * unit + r < rows && d < D) *(uint4*)(p.out + b * p.o_b + (at + ri) * p.o_t + rh * p.o_h + d) = w;
        __builtin_amdgcn_wave_barrier();
      }
    }
  };

  long long at = first;
  auto tile_end = [&](long long from) { return (int)(min(from + p.tile_tokens, last) - from); };
  int buf = 0, valid = 0;
  if (at < last) {
    valid = tile_end(at);
    load_tile(0, at, valid);
    if constexpr (OUT) fetch(at, valid);
  }
  weigh(valid);
  if constexpr (OUT) share_state();
  sent();
  if constexpr (OUT) note_odd(0);
  __syncthreads();
  while (at < last) {
    const long long next = at + valid;
    int next_valid = 0;
    if (next < last) {
      next_valid = tile_end(next);
      load_tile(buf ^ 1, next, next_valid);
      if constexpr (OUT) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) next_q[s] = first_q[s];
        fetch(next, next_valid);
      }
    } else if (OUT) {
#pragma unroll
      for (int s = 0; s < STEPS; ++s) next_q[s] = first_q[s];
    }
    __builtin_amdgcn_sched_barrier(0);
    const int rounds = rounds_of(valid);
    update(buf, valid, rounds == p.tile_rounds ? fade : fade_of(p, kvh, rounds));
    if constexpr (OUT) results(buf, at, valid);
    if (!OUT || wave >= units_of(valid)) sent();
    __syncthreads();  // S, the weights and this tile are read
    if (next < last) {
      if (OUT && tid == 0) odd_flag[buf] = 0;
      if constexpr (OUT) {
        note_odd(buf ^ 1);
        share_state();
      }
      if (next_valid != valid) weigh(next_valid);
    }
    __syncthreads();
    at = next, valid = next_valid, buf ^= 1;
  }
  float* const to = !OUT ? own : p.segments == 1 && p.state_out ? p.state_out + state_at : nullptr;
  if (to) {
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int dk = dk0 + 16 * i + 4 * g4 + e, dv = v0 + dv0 + 16 * j + c;
          if (dk < D && dv < D) to[dk * D + dv] = S[i][j][e];
        }
  }
}

// The S that each segment starts from, in the place of its own, and the last one.  A thread an element of S.
__global__ void __launch_bounds__(256) linear_scan_kernel(const Linear p) {
  const long long size = (long long)p.head_dim * p.head_dim;
  const int blocks = (int)((size + 255) / 256);
  const int bh = blockIdx.x / blocks, kvh = bh % p.kv_heads, b = bh / p.kv_heads;
  const long long i = (long long)(blockIdx.x % blocks) * 256 + threadIdx.x;
  if (i >= size) return;
  const int len = length_of(p, b);
  const int rounds = (int)(((long long)len + p.per_round - 1) / p.per_round);
  const int whole = rounds / p.segment_rounds, rest = rounds % p.segment_rounds;
  const Fade fade = fade_of(p, kvh, p.segment_rounds);
  float s = p.state ? p.state[bh * size + i] : 0.0f;
  float* at = p.starts + bh * p.segments * size + i;
  // (loads of several segments together: a store after each would hold the next one back)
  constexpr int BATCH = 16;
  for (int n0 = 0; n0 < whole; n0 += BATCH) {
    float own[BATCH];
#pragma unroll
    for (int n = 0; n < BATCH; ++n) own[n] = n0 + n < whole ? at[(n0 + n) * size] : 0.0f;
#pragma unroll
    for (int n = 0; n < BATCH; ++n)
      if (n0 + n < whole) {
        at[(n0 + n) * size] = s;
        s = faded(s, fade, own[n]);
      }
  }
  if (rest) {
    const float own = at[whole * size];
    at[whole * size] = s;
    s = faded(s, fade_of(p, kvh, rest), own);
  }
  if (p.state_out) p.state_out[bh * size + i] = s;
}

// One token an entry: thread (r, c) holds columns 4 c .. 4 c + 3 of rows r + ROWS n.  States are read and written past the caches, which
// are for what is read again sooner than at the next token: 256 entries, 8 heads of 128, 51 us against 59; 32 entries 9.1 against 10.4.
template <int DP>
__global__ void __launch_bounds__(256) linear_token_kernel(const Linear p) {
  constexpr int COLS = DP / 4, ROWS = 256 / COLS, N = DP / ROWS;
  __shared__ float4 part[ROWS][COLS];
  const int tid = threadIdx.x, c = tid % COLS, r = tid / COLS, D = p.head_dim;
  const int kvh = blockIdx.x % p.kv_heads, b = blockIdx.x / p.kv_heads;
  const long long at = (long long)blockIdx.x * D * D;
  const bool token = length_of(p, b) > 0;
  const bool col = 4 * c < D;
  f32x4 s[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    s[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (p.state && col && r + ROWS * n < D) s[n] = __builtin_nontemporal_load((const f32x4*)(p.state + at + (r + ROWS * n) * D + 4 * c));
  }
  if (token) {
    const Fade fade = fade_of(p, kvh, 1);
    const uint16_t* k = p.k + b * p.k_b + kvh * p.k_h;
    float v[4] = {};
    if (col) {
      const uint2 w = *(const uint2*)(p.v + b * p.v_b + kvh * p.v_h + 4 * c);
      v[0] = bf16_of(w.x & 0xffff), v[1] = bf16_of(w.x >> 16), v[2] = bf16_of(w.y & 0xffff), v[3] = bf16_of(w.y >> 16);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float x = r + ROWS * n < D ? load1(k + r + ROWS * n) : 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = faded(s[n][e], fade, x * v[e]);
    }
  }
#pragma unroll
  for (int n = 0; n < N; ++n)
    if (p.state_out && col && r + ROWS * n < D) __builtin_nontemporal_store(s[n], (f32x4*)(p.state_out + at + (r + ROWS * n) * D + 4 * c));
  if (!token) return;
  for (int g = 0; g < p.group; ++g) {
    const int h = kvh * p.group + g;
    const uint16_t* q = p.q + b * p.q_b + h * p.q_h;
    float4 o = make_float4(0, 0, 0, 0);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float x = r + ROWS * n < D ? load1(q + r + ROWS * n) : 0.0f;
      o.x = fmaf(x, s[n][0], o.x), o.y = fmaf(x, s[n][1], o.y), o.z = fmaf(x, s[n][2], o.z), o.w = fmaf(x, s[n][3], o.w);
    }
    __syncthreads();
    part[r][c] = o;
    __syncthreads();
    if (r == 0 && col) {
      for (int n = 1; n < ROWS; ++n) {
        const float4 w = part[n][c];
        o.x += w.x, o.y += w.y, o.z += w.z, o.w += w.w;
      }
      uint2 w;
      w.x = bf16_pack(o.x * p.scale, o.y * p.scale), w.y = bf16_pack(o.z * p.scale, o.w * p.scale);
      *(uint2*)(p.out + b * p.o_b + h * p.o_h + 4 * c) = w;
    }
  }
}

// How a call runs.
struct Plan {
  bool pairs;
  int tile_rounds, tile_tokens, segments, segment_rounds;
  size_t bytes;
  long long items;
};

Plan plan_for(const pd_linear_attention_args* a) {
  Plan n = {};
  n.pairs = a->per_round <= NARROW;
  const int tile = a->head_dim <= 64 ? 64 : Shape<128>::TILE;
  n.tile_rounds = n.pairs ? tile / a->per_round : 1;
  n.tile_tokens = n.pairs ? n.tile_rounds * a->per_round : tile;
  const long long rounds = ((long long)a->n + a->per_round - 1) / a->per_round, heads = std::max(1ll, (long long)a->batch * a->kv_heads);
  // Segments, to fill the card, while each holds tokens whose reading outweighs its state's (written, read twice and written
  // by the scan).  (Twice as many for 128 channels: the stream above 349 us against 338; half as many again for 64: the rows above 68 against 58.)
  const long long fill = a->head_dim <= 32 ? 2048 : a->head_dim <= 64 ? 512 : 256;
  const long long most = (long long)a->n / (4 * a->head_dim < 256 ? 256 : 4 * a->head_dim);
  long long segments = fill / heads;
  if (segments > most) segments = most;
  if (segments < 1) segments = 1;
  long long each = rounds ? (rounds + segments - 1) / segments : 1;
  each = (each + n.tile_rounds - 1) / n.tile_rounds * n.tile_rounds;
  n.segment_rounds = (int)(each < INT32_MAX - 64 ? each : INT32_MAX - 64);
  n.segments = rounds ? (int)((rounds + n.segment_rounds - 1) / n.segment_rounds) : 1;
  n.bytes = n.segments > 1 ? (size_t)heads * n.segments * a->head_dim * a->head_dim * 4 : 0;
  n.items = heads * n.segments;
  return n;
}

bool rows16(const void* p, long long b, long long t, long long h) {
  return (uintptr_t)p % 16 == 0 && b % 8 == 0 && t % 8 == 0 && h % 8 == 0;
}

pd_status check(const pd_linear_attention_args* a, bool pointers) {
  if (!a || a->batch < 0 || a->heads < 0 || a->kv_heads < 0 || a->n < 0 || a->per_round < 1 || a->head_dim < 1) return PD_ERR_INVALID_ARG;
  if (!(fabsf(a->scale) < INFINITY)) return PD_ERR_INVALID_ARG;
  if (a->heads && (!a->kv_heads || a->heads % a->kv_heads)) return PD_ERR_INVALID_ARG;
  if (a->head_dim % 8 || a->head_dim > 128) return PD_ERR_UNSUPPORTED;
  if (a->heads && a->heads / a->kv_heads > 64) return PD_ERR_UNSUPPORTED;
  // threads of a launch below 2^32: 256 for each work item (twice as many where two workgroups share it) or, of the recurrent form, key head.  (The
  // scan's, up to 64 workgroups a key head, are fewer: segments are made of up to 1024 key heads.)
  if ((__int128)a->kv_heads * a->batch >= 1ll << 24) return PD_ERR_UNSUPPORTED;
  if (a->n != 1 && (plan_for(a).items + 7) * (a->head_dim > 64 ? 2 : 1) >= 1ll << 24) return PD_ERR_UNSUPPORTED;
  if ((__int128)a->n * (a->kv_heads ? a->heads / a->kv_heads : 1) >= 1ll << 30) return PD_ERR_UNSUPPORTED;  // rows, in 32 bits
  if (!pointers || !a->batch) return PD_OK;
  if (!a->heads) return a->kv_heads && a->state_out ? PD_ERR_INVALID_ARG : PD_OK;  // (states without a query: not handed on)
  if ((uintptr_t)a->slopes % 4 || (uintptr_t)a->lengths % 4 || (uintptr_t)a->state % 16 || (uintptr_t)a->state_out % 16) return PD_ERR_INVALID_ARG;
  if (a->state && a->state_out && a->state != a->state_out) {
    const uintptr_t x = (uintptr_t)a->state, y = (uintptr_t)a->state_out;
    if ((x < y ? y - x : x - y) < (size_t)a->batch * a->kv_heads * a->head_dim * a->head_dim * 4) return PD_ERR_INVALID_ARG;
  }
  if (!a->n) return PD_OK;
  if (!a->q || !a->k || !a->v || !a->out || a->out == a->q || a->out == a->k || a->out == a->v) return PD_ERR_INVALID_ARG;
  if (!rows16(a->q, a->q_batch_stride, a->q_token_stride, a->q_head_stride) ||
      !rows16(a->k, a->k_batch_stride, a->k_token_stride, a->k_head_stride) ||
      !rows16(a->v, a->v_batch_stride, a->v_token_stride, a->v_head_stride) ||
      !rows16(a->out, a->out_batch_stride, a->out_token_stride, a->out_head_stride))
    return PD_ERR_UNSUPPORTED;
  if (!rows_apart(a->head_dim, {{a->batch, a->out_batch_stride}, {a->n, a->out_token_stride}, {a->heads, a->out_head_stride}}))
    return PD_ERR_INVALID_ARG;
  const size_t need = plan_for(a).bytes;
  if (need && (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < need)) return PD_ERR_INVALID_ARG;
  return PD_OK;
}

template <int DP>
void launch(const Linear& p, bool pairs, hipStream_t st) {
  const unsigned heads = (unsigned)(p.batch * p.kv_heads);
  if (p.n == 1) {
    hipLaunchKernelGGL(linear_token_kernel<DP>, dim3(heads), dim3(256), 0, st, p);
    return;
  }
  const unsigned items = heads * p.segments;
  const dim3 grid(Shape<DP>::VP == DP ? items : (items + 7) / 8 * 16), threads(Shape<DP>::NT);
  if (p.segments > 1) {
    if (pairs)
      hipLaunchKernelGGL((linear_narrow_kernel<DP, false>), grid, dim3(256), 0, st, p);
    else
      hipLaunchKernelGGL((linear_kernel<DP, false>), grid, threads, 0, st, p);
    hipLaunchKernelGGL(linear_scan_kernel, dim3(heads * ((p.head_dim * p.head_dim + 255) / 256)), dim3(256), 0, st, p);
  }
  if (pairs)
    hipLaunchKernelGGL((linear_narrow_kernel<DP, true>), grid, dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((linear_kernel<DP, true>), grid, threads, 0, st, p);
}

}  // namespace

extern "C" size_t predecoder_linear_attention_workspace(const pd_linear_attention_args* a) {
  if (check(a, false) != PD_OK || !a->batch || !a->heads) return 0;
  return plan_for(a).bytes;
}

extern "C" pd_status predecoder_linear_attention(void* hip_stream, const pd_linear_attention_args* a) {
  const pd_status ok = check(a, true);
  if (ok != PD_OK) return ok;
  if (!a->batch || !a->heads) return PD_OK;
  Linear p;
  p.batch = a->batch, p.heads = a->heads, p.kv_heads = a->kv_heads, p.group = a->heads / a->kv_heads, p.head_dim = a->head_dim;
  p.n = a->n, p.per_round = a->per_round, p.scale = a->scale;
  p.q = (const uint16_t*)a->q, p.k = (const uint16_t*)a->k, p.v = (const uint16_t*)a->v, p.out = (uint16_t*)a->out;
  p.q_b = a->q_batch_stride, p.q_t = a->q_token_stride, p.q_h = a->q_head_stride;
  p.k_b = a->k_batch_stride, p.k_t = a->k_token_stride, p.k_h = a->k_head_stride;
  p.v_b = a->v_batch_stride, p.v_t = a->v_token_stride, p.v_h = a->v_head_stride;
  p.o_b = a->out_batch_stride, p.o_t = a->out_token_stride, p.o_h = a->out_head_stride;
  p.slopes = a->slopes, p.lengths = a->lengths, p.state = a->state, p.state_out = a->state_out;
  const Plan n = plan_for(a);
  p.tile_rounds = n.tile_rounds, p.tile_tokens = n.tile_tokens, p.segments = n.segments, p.segment_rounds = n.segment_rounds;
  p.starts = (float*)a->workspace;
  const hipStream_t st = (hipStream_t)hip_stream;
  if (a->head_dim <= 32)
    launch<32>(p, n.pairs, st);
  else if (a->head_dim <= 64)
    launch<64>(p, n.pairs, st);
  else
    launch<128>(p, n.pairs, st);
  return hipGetLastError() == hipSuccess ? PD_OK : PD_ERR_DEVICE;
}
