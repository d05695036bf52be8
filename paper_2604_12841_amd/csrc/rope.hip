// rope.hip -- rotary positions with three axes (round, row, column).
//
// Pair m of a head turns by p f_m, p the token's position on the pair's axis.
// The angle is taken in turns, p f_m with f_m = base^(-k/n) / 2 pi split into
// two floats: a fused multiply-add drops the whole turns of p hi exactly and
// rounds what is left, and p lo is added, so the angle is as exact at round
// 100000 as at round 1.
//
// A work item is (token, head, chunk of pairs): neighbouring lanes hold
// neighbouring chunks, then heads, so a wave reads whole lines.  Bound by
// memory: each value is read and written once (163072 tokens x 10 heads x 64
// bf16: 77 us, 5.4 TB/s).
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/predecoder_ops.h"
#include "token_values.h"

namespace {

using namespace pd;

constexpr int MAX_PAIRS = 128;

struct Rope {
  long long tokens;
  int heads, pairs, turned, s0, s1;  // pairs [0, s0) turn with t, [s0, s1) with i, [s1, turned) with j
  int chunks;
  float sign;
  const int4* sites;
  const void* x;
  void* out;
  long long x_token, x_head, out_token, out_head;
  float hi[MAX_PAIRS], lo[MAX_PAIRS];  // turns of pair m for one step of its axis
};

// Sine and cosine of an angle in turns, |a| <= 1.
template <typename T>
__device__ __forceinline__ void sincos_turns(float a, float& s, float& c) {
  if constexpr (sizeof(T) == 4) {
    sincospif(2.0f * a, &s, &c);
  } else {  // within 2^-14, the result is rounded to bf16 (2^-8)
    s = __builtin_amdgcn_sinf(a);
    c = __builtin_amdgcn_cosf(a);
  }
}

// CP pairs a work item (8: wide loads; 1).  Interleaved pairs are neighbours,
// others half a head apart.
template <typename T, int CP, bool INTER>
__global__ void __launch_bounds__(256) rope_kernel(const Rope p) {
  const long long items = p.tokens * p.heads * p.chunks;
  for (long long w = (long long)blockIdx.x * 256 + threadIdx.x; w < items; w += (long long)gridDim.x * 256) {
    const int chunk = (int)(w % p.chunks);
    const long long wt = w / p.chunks;
    const int h = (int)(wt % p.heads);
    const long long token = wt / p.heads;
    const int4 at = p.sites[token];
    float c[CP], s[CP];
#pragma unroll
    for (int k = 0; k < CP; ++k) {
      const int m = chunk * CP + k;
      const float pos = (float)(m < p.s0 ? at.x : m < p.s1 ? at.y : at.z);
      const float turns = fmaf(pos, p.lo[m], fmaf(pos, p.hi[m], -__builtin_rintf(pos * p.hi[m])));
      sincos_turns<T>(turns, s[k], c[k]);
      s[k] *= p.sign;
    }
    const T* x = (const T*)p.x + token * p.x_token + h * p.x_head;
    T* out = (T*)p.out + token * p.out_token + h * p.out_head;
    const int first = INTER ? 2 * CP * chunk : CP * chunk;
    const int second = INTER ? first + CP : first + p.pairs;
    float v[2 * CP], o[2 * CP];
    if constexpr (CP == 8) {
      load8(x + first, v);
      load8(x + second, v + 8);
    } else {
      v[0] = load1(x + first);
      v[1] = load1(x + second);
    }
#pragma unroll
    for (int k = 0; k < CP; ++k) {
      const int a = INTER ? 2 * k : k, b = INTER ? 2 * k + 1 : k + CP;
      o[a] = v[a] * c[k] - v[b] * s[k];
      o[b] = v[b] * c[k] + v[a] * s[k];
      if (chunk * CP + k >= p.turned) o[a] = v[a], o[b] = v[b];
    }
    if constexpr (CP == 8) {
      store8(out + first, o);
      store8(out + second, o + 8);
    } else {
      store1(out + first, o[0]);
      store1(out + second, o[1]);
    }
  }
}

template <typename T, int CP>
void launch(const Rope& p, bool interleaved, hipStream_t st) {
  const long long items = p.tokens * p.heads * p.chunks;
  const long long want = (items + 255) / 256;
  const unsigned blocks = (unsigned)(want < (1 << 23) ? want : (1 << 23));  // threads stay below 2^32
  if (interleaved)
    hipLaunchKernelGGL((rope_kernel<T, CP, true>), dim3(blocks), dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((rope_kernel<T, CP, false>), dim3(blocks), dim3(256), 0, st, p);
}

}  // namespace

extern "C" pd_status predecoder_rope(void* hip_stream, const pd_rope_args* a) {
  if (!a || a->tokens < 0 || a->heads < 0 || a->head_dim < 2 || a->head_dim % 2) return PD_ERR_INVALID_ARG;
  if (a->dtype != PD_DTYPE_BF16 && a->dtype != PD_DTYPE_FP32) return PD_ERR_INVALID_ARG;
  if (!(a->base > 0.0) || !(a->base < INFINITY) || a->interleaved < 0 || a->interleaved > 1 || a->inverse < 0 ||
      a->inverse > 1)
    return PD_ERR_INVALID_ARG;
  const int pairs = a->head_dim / 2;
  long long turned = 0;
  for (int s : a->sections) {
    if (s < 0) return PD_ERR_INVALID_ARG;
    turned += s;
  }
  if (turned > pairs) return PD_ERR_INVALID_ARG;
  if (a->tokens == 0 || a->heads == 0) return PD_OK;
  if (!a->sites || (uintptr_t)a->sites % 16 || !a->x || !a->out) return PD_ERR_INVALID_ARG;
  const int elem = a->dtype == PD_DTYPE_BF16 ? 2 : 4;
  if ((uintptr_t)a->x % elem || (uintptr_t)a->out % elem) return PD_ERR_INVALID_ARG;
  if (a->head_dim > 2 * MAX_PAIRS) return PD_ERR_UNSUPPORTED;
  // work items are counted in 64 bits
  if (a->tokens > (1ll << 40) || a->heads > (1 << 20) || a->tokens > (1ll << 62) / ((long long)a->heads * pairs))
    return PD_ERR_UNSUPPORTED;
  // rows of out may not overlap, and out may be x only as it is
  if (!rows_apart(a->head_dim, {{a->tokens, a->out_token_stride}, {a->heads, a->out_head_stride}})) return PD_ERR_INVALID_ARG;
  if (a->out == a->x && ((a->tokens > 1 && a->out_token_stride != a->x_token_stride) ||
                         (a->heads > 1 && a->out_head_stride != a->x_head_stride)))
    return PD_ERR_INVALID_ARG;
  Rope p;
  p.tokens = a->tokens, p.heads = a->heads, p.pairs = pairs, p.turned = (int)turned;
  p.s0 = a->sections[0], p.s1 = a->sections[0] + a->sections[1];
  p.sign = a->inverse ? -1.0f : 1.0f;
  p.sites = (const int4*)a->sites;
  p.x = a->x, p.out = a->out;
  p.x_token = a->x_token_stride, p.x_head = a->x_head_stride;
  p.out_token = a->out_token_stride, p.out_head = a->out_head_stride;
  for (int axis = 0, m = 0; axis < 3; ++axis)
    for (int k = 0; k < a->sections[axis]; ++k, ++m) {
      const double f = pow(a->base, -(double)k / a->sections[axis]) / 6.283185307179586476925;
      p.hi[m] = (float)f;
      p.lo[m] = (float)(f - (double)p.hi[m]);
    }
  for (int m = (int)turned; m < MAX_PAIRS; ++m) p.hi[m] = p.lo[m] = 0.0f;
  auto rows16 = [&](const void* q, long long token, long long head) {
    return (uintptr_t)q % 16 == 0 && token * elem % 16 == 0 && head * elem % 16 == 0;
  };
  const bool wide = pairs % 8 == 0 && rows16(p.x, p.x_token, p.x_head) && rows16(p.out, p.out_token, p.out_head);
  p.chunks = wide ? pairs / 8 : pairs;
  const hipStream_t st = (hipStream_t)hip_stream;
  if (a->dtype == PD_DTYPE_BF16) {
    if (wide)
      launch<uint16_t, 8>(p, a->interleaved, st);
    else
      launch<uint16_t, 1>(p, a->interleaved, st);
  } else {
    if (wide)
      launch<float, 8>(p, a->interleaved, st);
    else
      launch<float, 1>(p, a->interleaved, st);
  }
  return hipGetLastError() == hipSuccess ? PD_OK : PD_ERR_DEVICE;
}
