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
// instruction, which keeps 2^-16 of a step's sum of |products| (measured):
// far below the output's rounding.  For an fp32 output that would be the
// largest error, so its codes are widened to bf16 (exact) and summed by the
// bf16 instruction in fp32, at half the rate.
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
};

// 16 bytes of a row from column k on, zero past K.
template <bool WIDE>
__device__ __forceinline__ uint4 row16(const uint8_t* __restrict__ row, int k, int K) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if constexpr (WIDE) {
    if (k < K) v = *(const uint4*)(row + k);
  } else {
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

// 64 tokens x 64 channels a workgroup, a 32 x 32 tile a wave, 64 codes of k
// at a time through LDS.
template <typename T, int SUM, int ACT, bool WIDE>
__global__ void __launch_bounds__(256) matmul8_kernel(const Mm p) {
  constexpr int PITCH = 80;  // bytes of an LDS row: 64 codes, and 16 to spread the banks
  __shared__ __attribute__((aligned(16))) uint8_t la[64 * PITCH];
  __shared__ __attribute__((aligned(16))) uint8_t lw[64 * PITCH];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tiles_n = (p.N + 63) / 64;
  const long long m0 = (long long)(blockIdx.x / tiles_n) * 64;
  const int n0 = (int)(blockIdx.x % tiles_n) * 64;
  const int r = tid >> 2, kc = (tid & 3) * 16;
  const long long ra = m0 + r < p.M ? m0 + r : p.M - 1;  // rows past the end repeat the last: not stored
  const int rw = n0 + r < p.N ? n0 + r : p.N - 1;
  const uint8_t* pa = p.a + ra * p.a_stride;
  const uint8_t* pw = p.w + rw * p.w_stride;
  const int wm = (wave & 1) * 32, wn = (wave >> 1) * 32;
  typename Acc<SUM>::type acc;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0;
  for (int k0 = 0; k0 < p.K; k0 += 64) {
    const uint4 va = row16<WIDE>(pa, k0 + kc, p.K), vw = row16<WIDE>(pw, k0 + kc, p.K);
    __syncthreads();
    *(uint4*)(la + r * PITCH + kc) = va;
    *(uint4*)(lw + r * PITCH + kc) = vw;
    __syncthreads();
    const uint8_t* fa = la + (wm + (lane & 31)) * PITCH + (lane >> 5) * 32;
    const uint8_t* fw = lw + (wn + (lane & 31)) * PITCH + (lane >> 5) * 32;
    const uint4 a0 = *(const uint4*)fa, a1 = *(const uint4*)(fa + 16);
    const uint4 w0 = *(const uint4*)fw, w1 = *(const uint4*)(fw + 16);
    mma64<SUM>(w0, w1, a0, a1, acc);
  }
  const long long m = m0 + wm + (lane & 31);
  if (m >= p.M) return;
  const float sa = p.a_scales[m];
  T* out = (T*)p.out + m * p.out_stride;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int n = n0 + wn + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
    if (n < p.N) {
      store1(out + n, act_fn<ACT>(fmaf((float)acc[e], sa * p.w_scales[n], p.bias ? p.bias[n] : 0.0f)));
    }
  }
}

template <typename T, int SUM, int ACT>
void launch(const Mm& p, bool wide, hipStream_t st) {
  const long long blocks = ((p.M + 63) / 64) * ((p.N + 63) / 64);
  if (wide)
    hipLaunchKernelGGL((matmul8_kernel<T, SUM, ACT, true>), dim3((unsigned)blocks), dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((matmul8_kernel<T, SUM, ACT, false>), dim3((unsigned)blocks), dim3(256), 0, st, p);
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
  if (((a->M + 63) / 64) * (((long long)a->N + 63) / 64) >= (1ll << 24)) return PD_ERR_UNSUPPORTED;
  Mm p;
  p.M = a->M, p.N = a->N, p.K = a->K;
  p.a = (const uint8_t*)a->a, p.w = (const uint8_t*)a->w;
  p.a_stride = a->a_stride, p.w_stride = a->w_stride, p.out_stride = a->out_stride;
  p.a_scales = a->a_scales, p.w_scales = a->w_scales, p.bias = a->bias, p.out = a->out;
  const bool wide = a->K % 16 == 0 && (uintptr_t)a->a % 16 == 0 && (uintptr_t)a->w % 16 == 0 &&
                    a->a_stride % 16 == 0 && a->w_stride % 16 == 0;
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
