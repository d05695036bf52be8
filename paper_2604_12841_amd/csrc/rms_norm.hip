// rms_norm.hip -- root-mean-square norm over the rows of a matrix, with the
// residual's addition before it and an 8-bit output with one scale per row.
//
//   s = x + residual;  y = s / sqrt(mean(s^2) + eps) * gain
//   scale = max |y| / Q;  code = round(y / scale) = round(s gain Q / max |s gain|)
//
// One pass: a row is read once into registers (by LPR lanes with NV granules
// of 8 values each), both statistics -- the sum of s^2 and the largest
// |s gain| -- come from there, and every output is written from there.  The
// code needs no division by the norm: it cancels.  Bound by memory: 163072 x
// 512 bf16 with a residual to a sum and E4M3 codes 103 us, 5.7 TB/s.  (Rows of more
// than 8192 columns spill 14 to 71 registers: 4096 x 16384 bf16 173 us.)
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/predecoder_ops.h"
#include "activation.h"
#include "token_values.h"

namespace {

using namespace pd;

struct Norm {
  long long rows;
  int width;
  float inv_width, eps, qmax;
  const void* x;
  const void* residual;
  const float* gain;
  void* sum;
  void* out;
  uint8_t* codes;
  float* scales;
  long long x_stride, residual_stride, sum_stride, out_stride, codes_stride;
  int int8;
  bool passing;  // sum and out, see token_values.h
};

// The column of value e (0 .. 8 NV - 1) of a lane: V neighbours (16 bytes of
// the row's type, so that a wave's load or store covers whole lines), or
// (rows without wide loads) one value in every LPR.
template <int LPR, int V, bool WIDE>
__device__ __forceinline__ int column(int lane, int e) {
  return WIDE ? (e / V * LPR + lane) * V + e % V : e * LPR + lane;
}

template <int V>
__device__ __forceinline__ void load_some(const uint16_t* p, float* v) {
  load16(p, v);
}
template <int V>
__device__ __forceinline__ void load_some(const float* p, float* v) {
  if constexpr (V == 8)
    load8(p, v);
  else
    load16(p, v);
}

template <typename T, int LPR, int NV, int V, bool WIDE>
__device__ __forceinline__ void load_row(const T* __restrict__ p, int lane, int width, float (&v)[8 * NV]) {
  if constexpr (WIDE) {
#pragma unroll
    for (int g = 0; g < 8 * NV / V; ++g) {
      const int c = column<LPR, V, true>(lane, V * g);
      float t[V];
#pragma unroll
      for (int e = 0; e < V; ++e) t[e] = 0.0f;
      if (c < width) load_some<V>(p + c, t);
#pragma unroll
      for (int e = 0; e < V; ++e) v[V * g + e] = t[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8 * NV; ++e) {
      const int c = column<LPR, V, false>(lane, e);
      v[e] = c < width ? load1(p + c) : 0.0f;
    }
  }
}

template <typename T, int LPR, int NV, int V, bool WIDE, bool PASSING>
__device__ __forceinline__ void store_row(T* __restrict__ p, int lane, int width, const float (&v)[8 * NV]) {
  if constexpr (WIDE) {
#pragma unroll
    for (int g = 0; g < 8 * NV / V; ++g) {
      const int c = column<LPR, V, true>(lane, V * g);
      if (c < width) store16<PASSING>(p + c, &v[V * g]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8 * NV; ++e) {
      const int c = column<LPR, V, false>(lane, e);
      if (c < width) store1(p + c, v[e]);
    }
  }
}

// The row's sum of `a` and largest `b` in every lane of the row.
template <int LPR>
__device__ __forceinline__ void reduce_row(float& a, float& b, float* shared) {
#pragma unroll
  for (int m = 1; m < (LPR < 64 ? LPR : 64); m <<= 1) {
    a += __shfl_xor(a, m);
    b = fmaxf(b, __shfl_xor(b, m));
  }
  if constexpr (LPR > 64) {
    constexpr int W = LPR / 64;
    const int wave = threadIdx.x >> 6;
    __syncthreads();  // the row before is done with `shared`
    if ((threadIdx.x & 63) == 0) {
      shared[wave] = a;
      shared[W + wave] = b;
    }
    __syncthreads();
    a = 0.0f, b = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      a += shared[w];
      b = fmaxf(b, shared[W + w]);
    }
  }
}

template <typename T, int LPR, int NV, bool WIDE, bool PASSING, bool TINY>
__global__ void __launch_bounds__(LPR > 256 ? LPR : 256) rms_norm_kernel(const Norm p) {
  constexpr int THREADS = LPR > 256 ? LPR : 256;
  constexpr int ROWS = THREADS / LPR;  // rows of a workgroup
  constexpr int V = 16 / (int)sizeof(T);
  __shared__ float shared[LPR > 64 ? 2 * (LPR / 64) : 1];
  const int lane = threadIdx.x % LPR;
  for (long long row = (long long)blockIdx.x * ROWS + threadIdx.x / LPR; row < p.rows;
       row += (long long)gridDim.x * ROWS) {
    float s[8 * NV];
    load_row<T, LPR, NV, V, WIDE>((const T*)p.x + row * p.x_stride, lane, p.width, s);
    if (p.residual) {
      float r[8 * NV];
      load_row<T, LPR, NV, V, WIDE>((const T*)p.residual + row * p.residual_stride, lane, p.width, r);
#pragma unroll
      for (int e = 0; e < 8 * NV; ++e) s[e] += r[e];
    }
    float g[8 * NV];
    if (p.gain) {
      load_row<float, LPR, NV, V, WIDE>(p.gain, lane, p.width, g);
    } else {
#pragma unroll
      for (int e = 0; e < 8 * NV; ++e) g[e] = 1.0f;
    }
    if (p.sum) store_row<T, LPR, NV, V, WIDE, PASSING>((T*)p.sum + row * p.sum_stride, lane, p.width, s);
    // TINY: rows of values below 2^-45 are taken 2^100 times as large, and eps 2^200 times, which leaves y and the codes as
    // they are
    float eps = p.eps;
    if constexpr (TINY) {
      float none = 0.0f, size = 0.0f;
#pragma unroll
      for (int e = 0; e < 8 * NV; ++e) size = fmaxf(size, fabsf(s[e]));
      reduce_row<LPR>(none, size, shared);
      const float lift = size < 0x1p-45f ? 0x1p100f : 1.0f;
      eps = eps * lift * lift;
#pragma unroll
      for (int e = 0; e < 8 * NV; ++e) s[e] *= lift;
    }
    float square = 0.0f, most = 0.0f, check = 0.0f;
    float low[8 * NV];  // what the rounding of s gain lost
#pragma unroll
    for (int e = 0; e < 8 * NV; ++e) {
      square = fmaf(s[e], s[e], square);
      const float v = s[e] * g[e];
      low[e] = fmaf(s[e], g[e], -v);
      s[e] = v;
      most = fmaxf(most, fabsf(v));  // drops NaN
      check = fmaf(v, 0.0f, check);  // NaN from an infinite or NaN s gain
    }
    if (!(check == 0.0f)) most = INFINITY;
    reduce_row<LPR>(square, most, shared);
    const float mean = fmaf(square, p.inv_width, eps);
    const float inv = TINY && mean == 0.0f ? 0.0f : 1.0f / sqrtf(mean);  // (a row of zeros without an eps is zeros)
    if (p.out) {
      float y[8 * NV];
#pragma unroll
      for (int e = 0; e < 8 * NV; ++e) y[e] = s[e] * inv;
      store_row<T, LPR, NV, V, WIDE, PASSING>((T*)p.out + row * p.out_stride, lane, p.width, y);
    }
    if (p.codes) {
      const bool finite = square < INFINITY && most < INFINITY;  // false for a NaN square
      // s gain and Q / most to twice the precision: a code then has the one rounding that the format makes, but for values
      // within 2^-24 of halfway between two codes
      const bool codes = finite && most > 0.0f;
      float big = most;
      if (big < 0x1p-64f) {  // rows of tiny values are lifted by a power of two, so that Q / most stays finite
        big *= 0x1p64f;
#pragma unroll
        for (int e = 0; e < 8 * NV; ++e) s[e] *= 0x1p64f, low[e] *= 0x1p64f;
      }
      const float q = codes ? p.qmax / big : 0.0f;
      const float q_low = fmaf(-q, big, p.qmax) * (q / p.qmax);
      if (lane == 0) p.scales[row] = finite ? most * inv / p.qmax : NAN;
      uint8_t* c = p.codes + row * p.codes_stride;
      float y[8 * NV];
#pragma unroll
      for (int e = 0; e < 8 * NV; ++e) y[e] = codes ? fmaf(s[e], q, fmaf(s[e], q_low, low[e] * q)) : 0.0f;
      if constexpr (WIDE) {
#pragma unroll
        for (int n = 0; n < 8 * NV / V; ++n) {
          const int at = column<LPR, V, true>(lane, V * n);
          if (at < p.width) {
            uint32_t w[V / 4];
#pragma unroll
            for (int k = 0; k < V / 4; ++k) {
              const float* v = &y[V * n + 4 * k];
              w[k] = p.int8 ? int8_pack4(v[0], v[1], v[2], v[3]) : e4m3_pack4_within(v[0], v[1], v[2], v[3]);
            }
            if constexpr (V == 8)
              *(uint2*)(c + at) = make_uint2(w[0], w[1]);
            else
              *(uint32_t*)(c + at) = w[0];
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8 * NV; ++e) {
          const int at = column<LPR, V, false>(lane, e);
          if (at < p.width) c[at] = (uint8_t)(p.int8 ? int8_pack4(y[e], 0, 0, 0) : e4m3_pack4(y[e], 0, 0, 0));
        }
      }
    }
  }
}

template <typename T, int LPR, int NV, bool WIDE, bool PASSING>
void launch_eps(const Norm& p, unsigned blocks, unsigned threads, hipStream_t st) {
  // Squares of values below 2^-45 lose bits, or all of them, that an eps below 2^-80 does not cover.  Finding the row's
  // largest value first takes up to 3 % longer (bf16 with residual to E4M3: 163072 x 512 2 %, 4096 x 16384 3 %).
  if (p.eps < 0x1p-80f)
    hipLaunchKernelGGL((rms_norm_kernel<T, LPR, NV, WIDE, PASSING, true>), dim3(blocks), dim3(threads), 0, st, p);
  else
    hipLaunchKernelGGL((rms_norm_kernel<T, LPR, NV, WIDE, PASSING, false>), dim3(blocks), dim3(threads), 0, st, p);
}

template <typename T, int LPR, int NV>
void launch(const Norm& p, bool wide, hipStream_t st) {
  constexpr int THREADS = LPR > 256 ? LPR : 256;
  constexpr int ROWS = THREADS / LPR;
  const long long want = (p.rows + ROWS - 1) / ROWS;
  // Waves of narrow rows take several, sixteen workgroups to a CU at most (rows of 128 to 512: 10 % less time than one each);
  // where a workgroup shares a row that only lengthens its chain of barriers (2048 fp32 columns: 7 % more), and the
  // bound keeps threads below 2^32.
  const long long most = LPR <= 64 ? 4096 : 1 << 21;
  const unsigned blocks = (unsigned)(want < most ? want : most);
  constexpr bool MAY_PASS = LPR <= 64;
  if (wide && MAY_PASS && p.passing)
    launch_eps<T, LPR, NV, true, MAY_PASS>(p, blocks, THREADS, st);
  else if (wide)
    launch_eps<T, LPR, NV, true, false>(p, blocks, THREADS, st);
  else
    launch_eps<T, LPR, NV, false, false>(p, blocks, THREADS, st);
}

// As few lanes as hold the row with one granule each up to a wave (a wave
// then reduces several narrow rows at once), then more granules, then a
// workgroup to a row.
template <typename T>
void launch_for_width(const Norm& p, bool wide, hipStream_t st) {
  if (p.width <= 64) return launch<T, 8, 1>(p, wide, st);
  if (p.width <= 128) return launch<T, 16, 1>(p, wide, st);
  if (p.width <= 256) return launch<T, 32, 1>(p, wide, st);
  if (p.width <= 512) return launch<T, 64, 1>(p, wide, st);
  if (p.width <= 1024) return launch<T, 64, 2>(p, wide, st);
  if (p.width <= 2048) return launch<T, 256, 1>(p, wide, st);
  if (p.width <= 4096) return launch<T, 256, 2>(p, wide, st);
  if (p.width <= 8192) return launch<T, 1024, 1>(p, wide, st);
  return launch<T, 1024, 4>(p, wide, st);
}

bool aligned(const void* p, long long stride, int elem, int to) {
  return !p || ((uintptr_t)p % to == 0 && (stride * elem) % to == 0);
}

}  // namespace

extern "C" pd_status predecoder_rms_norm(void* hip_stream, const pd_norm_args* a) {
  if (!a || a->rows < 0 || a->width < 1 || !(a->eps >= 0.0f) || !(a->eps < INFINITY)) return PD_ERR_INVALID_ARG;
  if (a->dtype != PD_DTYPE_BF16 && a->dtype != PD_DTYPE_FP32) return PD_ERR_INVALID_ARG;
  if (a->codes_type < PD_CODES_NONE || a->codes_type > PD_CODES_INT8) return PD_ERR_INVALID_ARG;
  if (a->rows == 0) return PD_OK;
  const bool codes = a->codes_type != PD_CODES_NONE;
  if (codes != (a->codes != nullptr) || codes != (a->scales != nullptr)) return PD_ERR_INVALID_ARG;
  if (!a->x || (!a->sum && !a->out && !codes)) return PD_ERR_INVALID_ARG;
  // an output's rows may not overlap each other; an input's may
  if (a->rows > 1 && ((a->sum && a->sum_stride < a->width) || (a->out && a->out_stride < a->width) ||
                      (codes && a->codes_stride < a->width)))
    return PD_ERR_INVALID_ARG;
  const int elem = a->dtype == PD_DTYPE_BF16 ? 2 : 4;
  if ((uintptr_t)a->x % elem || (uintptr_t)a->residual % elem || (uintptr_t)a->sum % elem ||
      (uintptr_t)a->out % elem || (uintptr_t)a->gain % 4 || (uintptr_t)a->scales % 4)
    return PD_ERR_INVALID_ARG;
  if (a->width > 32768 || a->rows > (1ll << 40)) return PD_ERR_UNSUPPORTED;  // values and work are counted in 64 bits
  // an output at an input's address is that input, row for row; two outputs do not share one
  auto other_rows = [&](const void* out, long long out_stride, const void* in, long long in_stride) {
    return out && out == in && a->rows > 1 && out_stride != in_stride;
  };
  if (other_rows(a->sum, a->sum_stride, a->x, a->x_stride) || other_rows(a->out, a->out_stride, a->x, a->x_stride) ||
      other_rows(a->sum, a->sum_stride, a->residual, a->residual_stride) ||
      other_rows(a->out, a->out_stride, a->residual, a->residual_stride) || (a->sum && a->sum == a->out))
    return PD_ERR_INVALID_ARG;
  Norm p;
  p.rows = a->rows;
  p.width = a->width;
  p.inv_width = 1.0f / (float)a->width;
  p.eps = a->eps;
  p.int8 = a->codes_type == PD_CODES_INT8;
  p.qmax = p.int8 ? 127.0f : 448.0f;
  p.x = a->x, p.residual = a->residual, p.gain = a->gain, p.sum = a->sum, p.out = a->out;
  p.codes = (uint8_t*)a->codes, p.scales = a->scales;
  p.passing = a->rows * a->width * elem > PASSING_BYTES;
  p.x_stride = a->x_stride, p.residual_stride = a->residual_stride, p.sum_stride = a->sum_stride;
  p.out_stride = a->out_stride, p.codes_stride = a->codes_stride;
  const bool wide = a->width % 8 == 0 && aligned(a->x, a->x_stride, elem, 16) &&
                    aligned(a->residual, a->residual_stride, elem, 16) && aligned(a->gain, 0, 4, 16) &&
                    aligned(a->sum, a->sum_stride, elem, 16) && aligned(a->out, a->out_stride, elem, 16) &&
                    aligned(a->codes, a->codes_stride, 1, 8);
  if (a->dtype == PD_DTYPE_BF16)
    launch_for_width<uint16_t>(p, wide, (hipStream_t)hip_stream);
  else
    launch_for_width<float>(p, wide, (hipStream_t)hip_stream);
  return hipGetLastError() == hipSuccess ? PD_OK : PD_ERR_DEVICE;
}
