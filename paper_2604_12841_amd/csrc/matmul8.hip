// matmul8.hip -- product of 8-bit codes (E4M3 or int8) with scales for each
// token and channel, bias and activation.
//
//   out[m][n] = act(a_scales[m] w_scales[n] sum_k a[m][k] w[n][k] + bias[n])
//
// Both operands run along k, as the matrix instructions read them.  Channels
// are the instruction's rows and tokens its columns, so a lane ends up with
// four neighbouring channels of one token at a time.
//
// int8 sums are exact (int32).  E4M3 sums of a bf16 output use the fp8 matrix
// instruction, which adds eight neighbouring products at a time and drops of
// each what lies below 2^-13 of the largest of the eight (measured; the groups'
// sums are fp32): at most 7 2^-13 of every group's largest, together below
// 2^-10 of the sum of |products| and so below half of the output's rounding,
// but not where the sum cancels.  For an fp32 output it would be the largest
// error by far, so its codes are widened to bf16 (exact) and summed by the bf16
// instruction in fp32.  That takes longer (for bf16 outputs 8192^3 769 us instead
// of 421, 163072 x 2048 x 512 with GELU 38 % more), which callers pay who ask for fp32.
//
// Tiles: the largest of 256 x 256 (eight waves, two by four), 128 x 128 and 64 x 64
// (four waves, two by two) that there are enough of, each wave with MB x NB blocks of
// 32 x 32.  Codes of aligned rows go straight to LDS, 128 of k a step in two buffers,
// one step ahead of their use (64 x 64 tiles: 64 in three buffers, two steps
// ahead); those of other rows pass through registers, one step ahead.
// Few tiles: a workgroup's waves share one 32 x 32 block and split k.
//
// A long sum runs at 2.2 to 2.3 PFLOP/s (8192^3, E4M3 and int8).  At K = 512 the sum
// and the epilogue take turns (one workgroup a CU): 163072 x 2048 x 512 E4M3
// with GELU 284 us, matrix units busy 0.28, vector units 0.43.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/predecoder_ops.h"
#include "token_values.h"

namespace {

using namespace pd;

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(16))) int i32x16;
typedef __attribute__((ext_vector_type(16))) float f32x16;

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

enum Sum { SUM_INT8, SUM_FP8, SUM_WIDE };  // the instruction that sums the products

struct Mm {
  long long M;
  int N, K;
  const uint8_t* a;
  const uint8_t* w;
  long long a_stride, w_stride, out_stride;
  const float* a_scales;
  const float* w_scales;
  const float* bias;
  void* out;
  bool lines;   // rows of out are 16-byte aligned
  bool passing;  // see token_values.h
};

// 16 bytes of a row from column k on, zero past K; nothing outside the row is read.  (Device memory takes unaligned
// 16-byte loads.)
__device__ __forceinline__ uint4 row16(const uint8_t* __restrict__ row, int k, int K) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (k + 16 <= K) {
    __builtin_memcpy(&v, row + k, 16);
  } else if (k < K && K >= 16) {  // the row's last 16 bytes, moved down
    unsigned __int128 w;
    __builtin_memcpy(&w, row + K - 16, 16);
    w >>= 8 * (k + 16 - K);
    v = __builtin_bit_cast(uint4, w);
  } else if (k < K) {
    uint32_t u[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (k + e < K) u[e >> 2] |= (uint32_t)row[k + e] << (8 * (e & 3));
    v = make_uint4(u[0], u[1], u[2], u[3]);
  }
  return v;
}

// Eight E4M3 codes (lo: the first four) as bf16.
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// acc += 32 channels x 32 tokens over 64 codes: a lane holds the row of its
// channel (w) and of its token (a), codes 0-31 or 32-63 by its half.
template <int SUM>
struct Acc {
  using type = f32x16;
};
template <>
struct Acc<SUM_INT8> {
  using type = i32x16;
};

template <int SUM>
__device__ __forceinline__ void mma64(const uint4 w0, const uint4 w1, const uint4 a0, const uint4 a1,
                                      typename Acc<SUM>::type& acc) {
  if constexpr (SUM == SUM_INT8) {
    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, w0), __builtin_bit_cast(i32x4, a0), acc, 0,
                                                0, 0);
    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, w1), __builtin_bit_cast(i32x4, a1), acc, 0,
                                                0, 0);
  } else if constexpr (SUM == SUM_FP8) {
    const i32x8 va = {(int)a0.x, (int)a0.y, (int)a0.z, (int)a0.w, (int)a1.x, (int)a1.y, (int)a1.z, (int)a1.w};
    const i32x8 vw = {(int)w0.x, (int)w0.y, (int)w0.z, (int)w0.w, (int)w1.x, (int)w1.y, (int)w1.z, (int)w1.w};
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vw, va, acc, 0, 0, 0, 0, 0, 0);
  } else {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(w0.x, w0.y), widen8(a0.x, a0.y), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(w0.z, w0.w), widen8(a0.z, a0.w), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(w1.x, w1.y), widen8(a1.x, a1.y), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(w1.z, w1.w), widen8(a1.z, a1.w), acc, 0, 0, 0);
  }
}

// Sends 16 bytes a lane from base + at to LDS byte `to` (the same in all lanes) + 16 times the lane.  Written out
// rather than with the builtin, for which the compiler waits before any later LDS read, of the other buffers too; the
// kernel counts the loads in flight itself.  No register is an output.  (The wait states are those that the load needs
// after writes of m0 and, by vector instructions, of its scalar base.)
__device__ __forceinline__ void send16(const uint8_t* base, uint32_t at, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(at), "s"(base));
}

template <int N>
__device__ __forceinline__ void wait_sent() {  // all but the last N loads are there
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);
  asm volatile("" ::: "memory");
}

// The activation of a result, which keeps NaN: a row that the norm marked by its scale stays marked.  (The conv layers'
// ReLU gives 0 for it.)
template <int ACT>
__device__ __forceinline__ float activated(float y) {
  if constexpr (ACT == PD_ACT_RELU)
    return y <= 0.0f ? 0.0f : y;
  else
    return act_fn<ACT>(y);
}

// The scales, bias, activation and rounding of a wave's blocks, 32 tokens at a time through LDS to whole lines.
// acc[mb][nb]: tokens m0 + 32 mb, channels n0 + 32 nb on; sa: the scales of this lane's tokens; sw: the channels'
// scales and, ws further, biases in LDS; `stage`: 4 KB of LDS of this wave's own.
template <typename T, int SUM, int ACT, int MB, int NB, bool PASSING>
__device__ __forceinline__ void finish(const Mm& p, typename Acc<SUM>::type (&acc)[MB][NB], long long m0, int n0,
                                       const float (&sa)[MB], const float* sw, int ws, uint8_t* stage) {
  const int lane = threadIdx.x & 63, half = lane >> 5;
  constexpr int PER = sizeof(T) == 2 && NB > 1 ? 2 : 1;     // blocks of channels a pass
  constexpr int ROW = PER * 32 * (int)sizeof(T);            // bytes of a token's row: 64 or 128
  constexpr int GR = ROW / 16;                              // granules of a row
  constexpr int E = 16 / (int)sizeof(T);                    // values of a granule
#pragma unroll
  for (int pass = 0; pass < NB / PER; ++pass)
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const int r = lane & 31;
#pragma unroll
      for (int q = 0; q < PER; ++q)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int nb = pass * PER + q;
          const float4 s4 = *(const float4*)(sw + 32 * nb + 8 * g + 4 * half);
          const float4 b4 = *(const float4*)(sw + ws + 32 * nb + 8 * g + 4 * half);
          const float s[4] = {s4.x, s4.y, s4.z, s4.w}, b[4] = {b4.x, b4.y, b4.z, b4.w};
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[e] = activated<ACT>(fmaf((float)acc[mb][nb][4 * g + e] * s[e], sa[mb], b[e]));
          if constexpr (sizeof(T) == 2) {
            const int at = r * ROW + (((4 * q + g) ^ (r >> 1 & (GR - 1))) << 4) + 8 * half;
            *(uint2*)(stage + at) = make_uint2(bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]));
          } else {
            const int at = r * ROW + (((2 * g + half) ^ (r >> 1 & (GR - 1))) << 4);
            *(float4*)(stage + at) = make_float4(v[0], v[1], v[2], v[3]);
          }
        }
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wave's rows are in LDS
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < GR / 2; ++i) {
        const int c = lane + 64 * i, rr = c / GR, g = c % GR;
        const long long m = m0 + 32 * mb + rr;
        const int n = n0 + 32 * PER * pass + g * E;
        const uint4 w = *(const uint4*)(stage + rr * ROW + ((g ^ (rr >> 1 & (GR - 1))) << 4));
        if (m < p.M && n < p.N) {
          T* to = (T*)p.out + m * p.out_stride + n;
          if (p.lines && n + E <= p.N) {
            store16<PASSING>(to, w);
          } else {
            T v[E];
            __builtin_memcpy(v, &w, 16);
#pragma unroll
            for (int e = 0; e < E; ++e)
              if (n + e < p.N) to[e] = v[e];
          }
        }
      }
      __builtin_amdgcn_s_waitcnt(0xc07f);  // the reads are done before the next rows are written
      __builtin_amdgcn_wave_barrier();
    }
}

// The scales and biases of a tile on their way: this lane's tokens', and channel threadIdx.x's.
template <int MB>
struct Scales {
  float a[MB], w, bias;
};
template <int MB>
__device__ __forceinline__ Scales<MB> load_scales(const Mm& p, long long m0, int n0) {
  Scales<MB> s;
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) s.a[mb] = p.a_scales[min(m0 + 32 * mb + (threadIdx.x & 31), p.M - 1)];
  const int n = min(n0 + (int)threadIdx.x, p.N - 1);
  s.w = p.w_scales[n];
  s.bias = p.bias ? p.bias[n] : 0.0f;
  return s;
}
template <int MB, int N>
__device__ __forceinline__ void keep_scales(const Scales<MB>& s, float* sw) {  // complete after a barrier
  if (threadIdx.x < N) {
    sw[threadIdx.x] = s.w;
    sw[N + threadIdx.x] = s.bias;
  }
}

// 2 x WN waves of MB x NB blocks; BK codes of k a step, BUFS steps in LDS.  With wide loads a workgroup takes several
// tiles, and the loads run on into the next one: its first steps arrive while this one's results are written.
template <typename T, int SUM, int ACT, int MB, int NB, int WN, int BK, int BUFS, bool WIDE, bool PASSING>
__global__ void __launch_bounds__(128 * WN, MB * NB >= 4 ? 2 : 3) matmul8_kernel(const Mm p) {
  constexpr int TM = 64 * MB, TN = 32 * NB * WN;
  constexpr int BUF = (TM + TN) * BK;          // bytes of a step: tokens, then channels
  constexpr int SENDS = BUF / 1024 / (2 * WN);  // 1 KB pieces that a wave loads a step
  // results go through a buffer whose codes are used up, or, where it is too small, through LDS of their own
  constexpr int STAGE = 32 * (sizeof(T) == 2 && NB == 1 ? 64 : 128);  // bytes of a wave's
  constexpr bool OWN = 2 * WN * STAGE > BUF;
  constexpr int GR = BK / 16;                  // granules of a row
  __shared__ __attribute__((aligned(1024))) uint8_t lds[BUFS * BUF + (OWN ? 2 * WN * STAGE : 0)];
  __shared__ __attribute__((aligned(16))) float sw[2 * TN];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroups are dealt to the eight XCDs in turn: an XCD takes neighbouring
  // tiles, bands of eight by all channels, whose codes stay in its L2.
  const unsigned tiles_n = (p.N + TN - 1) / TN, tiles_m = (unsigned)((p.M + TM - 1) / TM), items = tiles_m * tiles_n;
  const unsigned xcd = blockIdx.x & 7, per = items >> 3, rest = items & 7;
  const unsigned first = xcd * per + min(xcd, rest), end = first + per + (xcd < rest);
  const unsigned stride = (gridDim.x - xcd + 7) >> 3;  // workgroups of this XCD
  auto place = [&](unsigned item, long long& m0, int& n0) {
    const unsigned band = item / (8 * tiles_n), in_band = item - band * 8 * tiles_n;
    const unsigned high = min(8u, tiles_m - 8 * band);
    m0 = (long long)(8 * band + in_band % high) * TM;
    n0 = (int)(in_band / high) * TN;
  };
  const int wm = wave & 1, wn = wave >> 1;
  const int steps = (p.K + BK - 1) / BK;

  // Granule slot s of a step's buffer: row s / GR (tokens, then channels), and
  // granule (s % GR) ^ turn of its BK bytes: the 16 lanes that read at once
  // then fall on all banks.  A wave loads slots (wave SENDS + n) 64 + lane.
  auto turn_of = [](int row) { return BK == 64 ? row >> 2 & 3 : row >> 1 & 7; };
  // the tile that loads are for
  const uint8_t* a0;
  const uint8_t* w0;
  uint32_t from[SENDS];  // byte offset of the slot's granule from the tile's first row, or in its row
  const uint8_t* rows[WIDE ? 1 : SENDS];
  auto aim = [&](unsigned item) {
    long long m0;
    int n0;
    place(item, m0, n0);
    a0 = p.a + m0 * p.a_stride;
    w0 = p.w + n0 * p.w_stride;
#pragma unroll
    for (int n = 0; n < SENDS; ++n) {
      const int row = ((wave * SENDS + n) * 64 + lane) / GR, g = (lane & (GR - 1)) ^ turn_of(row);
      const bool token = (wave * SENDS + n) * (1024 / BK) < TM;  // whole rows a piece
      const int r = token ? (int)min((long long)row, p.M - 1 - m0) : min(row - TM, p.N - 1 - n0);
      if constexpr (WIDE)
        from[n] = (uint32_t)r * (uint32_t)(token ? p.a_stride : p.w_stride) + g * 16;
      else
        from[n] = g * 16, rows[n] = token ? a0 + r * p.a_stride : w0 + r * p.w_stride;
    }
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)lds;
  auto send_step = [&](int step, int buf) {  // WIDE
    const int k0 = step * BK;
    const uint32_t to = lds0 + buf * BUF + wave * SENDS * 1024;
    const uint8_t* const ak = a0 + k0;
    const uint8_t* const wk = w0 + k0;
    if (k0 + BK <= p.K) {
#pragma unroll
      for (int n = 0; n < SENDS; ++n)
        send16((wave * SENDS + n) * (1024 / BK) < TM ? ak : wk, from[n], to + n * 1024);
    } else {
#pragma unroll
      for (int n = 0; n < SENDS; ++n) {
        const int row = ((wave * SENDS + n) * 64 + lane) / GR, g = (lane & (GR - 1)) ^ turn_of(row);
        if (k0 + g * 16 < p.K)
          send16((wave * SENDS + n) * (1024 / BK) < TM ? ak : wk, from[n], to + n * 1024);
        else
          *(uint4*)(lds + buf * BUF + (wave * SENDS + n) * 1024 + lane * 16) = make_uint4(0, 0, 0, 0);
      }
    }
  };
  uint4 staged[WIDE ? 1 : SENDS];
  auto load_step = [&](int step) {
#pragma unroll
    for (int n = 0; n < (WIDE ? 0 : SENDS); ++n) staged[n] = row16(rows[n], step * BK + from[n], p.K);
  };
  auto store_step = [&](int buf) {
#pragma unroll
    for (int n = 0; n < (WIDE ? 0 : SENDS); ++n)
      *(uint4*)(lds + buf * BUF + (wave * SENDS + n) * 1024 + lane * 16) = staged[n];
  };

  typename Acc<SUM>::type acc[MB][NB];
  // this lane's row of a block, and granules 4 u + 2 half, + 1 of it
  const int turn = turn_of(lane & 31), h2 = lane >> 5 << 1;
  const int arow = (wm * 32 * MB + (lane & 31)) * BK, wrow = (TM + wn * 32 * NB + (lane & 31)) * BK;
  auto compute = [&](int buf) {
    const uint8_t* const s = lds + buf * BUF;
#pragma unroll
    for (int u = 0; u < BK / 64; ++u) {
      const int g0 = ((4 * u + h2) ^ turn) << 4, g1 = ((4 * u + h2 + 1) ^ turn) << 4;
      uint4 fa[MB][2], fw[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        fw[nb][0] = *(const uint4*)(s + wrow + nb * 32 * BK + g0);
        fw[nb][1] = *(const uint4*)(s + wrow + nb * 32 * BK + g1);
      }
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        fa[mb][0] = *(const uint4*)(s + arow + mb * 32 * BK + g0);
        fa[mb][1] = *(const uint4*)(s + arow + mb * 32 * BK + g1);
      }
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) mma64<SUM>(fw[nb][0], fw[nb][1], fa[mb][0], fa[mb][1], acc[mb][nb]);
    }
  };

  auto clear = [&] {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[mb][nb][e] = 0;
  };
  auto results = [&](unsigned item, const Scales<MB>& s, int buf) {  // through LDS buffer `buf`
    long long m0;
    int n0;
    place(item, m0, n0);
    keep_scales<MB, TN>(s, sw);
    __syncthreads();  // ... and all waves are done with the buffer
    finish<T, SUM, ACT, MB, NB, PASSING>(p, acc, m0 + wm * 32 * MB, n0 + wn * 32 * NB, s.a, sw + wn * 32 * NB, TN,
                                lds + (OWN ? BUFS : buf) * BUF + wave * STAGE);
  };
  auto scales = [&](unsigned item) {
    long long m0;
    int n0;
    place(item, m0, n0);
    return load_scales<MB>(p, m0 + wm * 32 * MB, n0);
  };

  unsigned item = first + (blockIdx.x >> 3);
  if (item >= end) return;
  if constexpr (WIDE) {
    static_assert(BUFS == 2 || BUFS == 3, "one or two steps ahead");
    unsigned next = item;  // the tile and the step that loads are for
    int next_step = 0, next_buf = 0;
    auto send_next = [&] {
      if (next >= end) return;
      if (next_step == 0) aim(next);
      send_step(next_step, next_buf);
      next_buf = next_buf == BUFS - 1 ? 0 : next_buf + 1;
      if (++next_step == steps) next_step = 0, next += stride;
    };
    if (steps > 0) {
      send_next();
      if (BUFS == 3) send_next();
    }
    int buf = 0;
    bool there = false;  // the step's loads have been waited for
    for (; item < end; item += stride) {
      const Scales<MB> s = scales(item);
      clear();
      for (int step = 0; step < steps; ++step) {
        // all but the newest loads, those of the step after this one; the last of all has none behind it
        if (!there) {
          if (BUFS == 3 && (step + 1 < steps || item + stride < end))
            wait_sent<SENDS>();
          else
            wait_sent<0>();
        }
        there = false;
        __syncthreads();  // the step's codes are there for all; the buffer before it is read to the end
        send_next();
        compute(buf);
        buf = buf == BUFS - 1 ? 0 : buf + 1;
      }
      if (steps > 0 && item + stride < end) {
        // wait for the next tile's first step before the stores are behind its loads
        if (BUFS == 3 && (steps > 1 || item + 2 * stride < end))
          wait_sent<SENDS>();
        else
          wait_sent<0>();
        there = true;
      }
      results(item, s, buf == 0 ? BUFS - 1 : buf - 1);
      if (steps == 0) __syncthreads();  // the scales' LDS is read to the end
    }
  } else {
    const Scales<MB> s = scales(item);
    clear();
    aim(item);
    if (steps > 0) {
      load_step(0);
      store_step(0);
    }
    int buf = 0;
    for (int step = 0; step < steps; ++step) {
      if (step + 1 < steps) load_step(step + 1);
      __syncthreads();
      compute(buf);
      buf = buf == BUFS - 1 ? 0 : buf + 1;
      if (step + 1 < steps) store_step(buf);
    }
    __syncthreads();
    results(item, s, 0);
  }
}

// 32 tokens x 32 channels a workgroup of eight waves, each with every eighth step of k, straight from memory.
template <typename T, int SUM, int ACT, bool WIDE>
__global__ void __launch_bounds__(512) matmul8_few_kernel(const Mm p) {
  constexpr int W = 8;
  __shared__ __attribute__((aligned(16))) typename Acc<SUM>::type sums[W / 2][64];
  __shared__ __attribute__((aligned(16))) uint8_t stage[4096];
  __shared__ __attribute__((aligned(16))) float sw[2 * 32];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int tiles_n = (p.N + 31) / 32;
  const long long m0 = (long long)(blockIdx.x / tiles_n) * 32;
  const int n0 = (int)(blockIdx.x % tiles_n) * 32;
  const long long ra = min(m0 + (lane & 31), p.M - 1);
  const int rw = min(n0 + (lane & 31), p.N - 1);
  const uint8_t* const pa = p.a + ra * p.a_stride;
  const uint8_t* const pw = p.w + rw * p.w_stride;
  const Scales<1> s = load_scales<1>(p, m0, n0);
  keep_scales<1, 32>(s, sw);
  typename Acc<SUM>::type acc[1][1];
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[0][0][e] = 0;
  auto load = [&](const uint8_t* row, int k) {
    if constexpr (WIDE) return k < p.K ? *(const uint4*)(row + k) : make_uint4(0, 0, 0, 0);
    else return row16(row, k, p.K);
  };
  for (int k0 = wave * 64; k0 < p.K; k0 += W * 64) {
    const int k = k0 + 32 * half;
    const uint4 a0 = load(pa, k), a1 = load(pa, k + 16), w0 = load(pw, k), w1 = load(pw, k + 16);
    mma64<SUM>(w0, w1, a0, a1, acc[0][0]);
  }
  // waves 4 .. 7 to 0 .. 3, then 2 and 3, then 1: one order of sums
#pragma unroll
  for (int n = W / 2; n > 0; n >>= 1) {
    if (wave >= n && wave < 2 * n) sums[wave - n][lane] = acc[0][0];
    __syncthreads();
    if (wave < n) {
      const typename Acc<SUM>::type other = sums[wave][lane];
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[0][0][e] += other[e];
    }
    __syncthreads();
  }
  if (wave == 0) finish<T, SUM, ACT, 1, 1, false>(p, acc, m0, n0, s.a, sw, 32, stage);
}

template <typename T, int SUM, int ACT, int MB, int NB, int WN, int BK, int BUFS>
void launch_tiles(const Mm& p, bool wide, hipStream_t st) {
  constexpr int TM = 64 * MB, TN = 32 * NB * WN;
  const unsigned items = (unsigned)(((p.M + TM - 1) / TM) * ((p.N + TN - 1) / TN));
  const unsigned most = 256 * (MB * NB == 8 ? 1 : MB * NB == 4 ? 2 : 3);  // workgroups that the card holds at once
  constexpr bool MAY_PASS = MB * NB == 8;  // smaller tiles have smaller results
  if (wide && MAY_PASS && p.passing)
    hipLaunchKernelGGL((matmul8_kernel<T, SUM, ACT, MB, NB, WN, BK, BUFS, true, MAY_PASS>),
                       dim3(items < most ? items : most), dim3(128 * WN), 0, st, p);
  else if (wide)
    hipLaunchKernelGGL((matmul8_kernel<T, SUM, ACT, MB, NB, WN, BK, BUFS, true, false>),
                       dim3(items < most ? items : most), dim3(128 * WN), 0, st, p);
  else
    hipLaunchKernelGGL((matmul8_kernel<T, SUM, ACT, MB, NB, WN, BK, BUFS, false, false>), dim3(items), dim3(128 * WN), 0,
                       st, p);
}

template <typename T, int SUM, int ACT>
void launch(const Mm& p, bool wide, hipStream_t st) {
  auto tiles = [&](int m, int n) { return ((p.M + m - 1) / m) * ((p.N + n - 1) / n); };
  if (tiles(256, 256) >= 256) {
    launch_tiles<T, SUM, ACT, 4, 2, 4, 128, 2>(p, wide, st);
  } else if (tiles(128, 128) >= 256) {
    launch_tiles<T, SUM, ACT, 2, 2, 2, 128, 2>(p, wide, st);
  } else if (tiles(64, 64) >= 192) {
    launch_tiles<T, SUM, ACT, 1, 1, 2, 64, 3>(p, wide, st);
  } else {
    const unsigned blocks = (unsigned)tiles(32, 32);
    if (wide)
      hipLaunchKernelGGL((matmul8_few_kernel<T, SUM, ACT, true>), dim3(blocks), dim3(512), 0, st, p);
    else
      hipLaunchKernelGGL((matmul8_few_kernel<T, SUM, ACT, false>), dim3(blocks), dim3(512), 0, st, p);
  }
}

}  // namespace

extern "C" pd_status predecoder_matmul8(void* hip_stream, const pd_matmul8_args* a) {
  if (!a || a->M < 0 || a->N < 0 || a->K < 0) return PD_ERR_INVALID_ARG;
  if (a->codes_type != PD_CODES_E4M3 && a->codes_type != PD_CODES_INT8) return PD_ERR_INVALID_ARG;
  if (a->out_dtype != PD_DTYPE_BF16 && a->out_dtype != PD_DTYPE_FP32) return PD_ERR_INVALID_ARG;
  if (a->act < PD_ACT_NONE || a->act > PD_ACT_RELU) return PD_ERR_INVALID_ARG;
  if (a->M == 0 || a->N == 0) return PD_OK;
  if ((a->K > 0 && (!a->a || !a->w)) || !a->a_scales || !a->w_scales || !a->out) return PD_ERR_INVALID_ARG;
  if (a->M > 1 && a->out_stride < a->N) return PD_ERR_INVALID_ARG;  // rows of out may not overlap
  const int elem = a->out_dtype == PD_DTYPE_BF16 ? 2 : 4;
  if ((uintptr_t)a->out % elem || (uintptr_t)a->a_scales % 4 || (uintptr_t)a->w_scales % 4 || (uintptr_t)a->bias % 4)
    return PD_ERR_INVALID_ARG;
  if (a->codes_type == PD_CODES_INT8 && a->K > 131071) return PD_ERR_UNSUPPORTED;  // |sum| <= 2^31 - 1
  // threads stay below 2^32
  if (a->M > (1ll << 30) || ((a->M + 63) / 64) * (((long long)a->N + 63) / 64) >= (1ll << 24)) return PD_ERR_UNSUPPORTED;
  Mm p;
  p.M = a->M, p.N = a->N, p.K = a->K;
  p.a = (const uint8_t*)a->a, p.w = (const uint8_t*)a->w;
  p.a_stride = a->a_stride, p.w_stride = a->w_stride, p.out_stride = a->out_stride;
  p.a_scales = a->a_scales, p.w_scales = a->w_scales, p.bias = a->bias, p.out = a->out;
  // (163072 x 2048 x 512 E4M3 to bf16, no activation: 228 us past the caches, 250 through them)
  p.passing = a->M * a->N * elem > PASSING_BYTES;
  p.lines = (uintptr_t)a->out % 16 == 0 && (a->out_stride * elem) % 16 == 0;
  // 256 rows of a tile within 32-bit offsets
  const bool wide = a->K % 16 == 0 && (uintptr_t)a->a % 16 == 0 && (uintptr_t)a->w % 16 == 0 &&
                    a->a_stride % 16 == 0 && a->w_stride % 16 == 0 && a->a_stride >= 0 && a->w_stride >= 0 &&
                    a->a_stride < (1 << 23) && a->w_stride < (1 << 23);
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool int8 = a->codes_type == PD_CODES_INT8;
  with_activation(a->act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    if (a->out_dtype == PD_DTYPE_BF16)
      int8 ? launch<uint16_t, SUM_INT8, ACT>(p, wide, st) : launch<uint16_t, SUM_FP8, ACT>(p, wide, st);
    else
      int8 ? launch<float, SUM_INT8, ACT>(p, wide, st) : launch<float, SUM_WIDE, ACT>(p, wide, st);
  });
  return hipGetLastError() == hipSuccess ? PD_OK : PD_ERR_DEVICE;
}
