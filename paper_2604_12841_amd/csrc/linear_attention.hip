// linear_attention.hip -- linear attention with a decay for each head, over
// rounds of tokens:
//   S_t = exp(-slope) S_(t-1) + sum over the tokens m of round t of k_m v_m^T
//   out_n = scale q_n S_t(n)
//
// The recurrent form: a workgroup holds the columns of S of one batch entry and
// key head, a thread some rows of one column.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/predecoder_ops.h"
#include "token_values.h"

namespace {

using namespace pd;

struct Linear {
  int batch, heads, kv_heads, group, head_dim, n, per_round;
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
};

// A workgroup of 16 x 16 threads: thread (r, c) holds rows r + 16 n of column c of sixteen.
__global__ void __launch_bounds__(256) linear_simple_kernel(const Linear p) {
  __shared__ float part[16][17];
  const int r = threadIdx.x >> 4, c = threadIdx.x & 15, D = p.head_dim;
  const int kvh = blockIdx.y % p.kv_heads, b = blockIdx.y / p.kv_heads, col = blockIdx.x * 16 + c;
  const int len = p.lengths ? min(max(p.lengths[b], 0), p.n) : p.n;
  const float fade = p.slopes ? expf(-p.slopes[kvh]) : 1.0f;
  const long long at = (long long)blockIdx.y * D * D;
  float s[8];
#pragma unroll
  for (int m = 0; m < 8; ++m) s[m] = p.state && r + 16 * m < D && col < D ? p.state[at + (r + 16 * m) * D + col] : 0.0f;
  for (long long n00 = 0; n00 < len; n00 += p.per_round) {
    const int n0 = (int)n00;
    const int n1 = (int)min((long long)len, (long long)n0 + p.per_round);
#pragma unroll
    for (int m = 0; m < 8; ++m) s[m] *= fade;
    for (int n = n0; n < n1; ++n) {
      const uint16_t* k = p.k + b * p.k_b + n * p.k_t + kvh * p.k_h;
      const float v = col < D ? load1(p.v + b * p.v_b + n * p.v_t + kvh * p.v_h + col) : 0.0f;
#pragma unroll
      for (int m = 0; m < 8; ++m)
        if (r + 16 * m < D) s[m] = fmaf(load1(k + r + 16 * m), v, s[m]);
    }
    for (int n = n0; n < n1; ++n)
      for (int g = 0; g < p.group; ++g) {
        const int h = kvh * p.group + g;
        const uint16_t* q = p.q + b * p.q_b + n * p.q_t + h * p.q_h;
        float sum = 0.0f;
#pragma unroll
        for (int m = 0; m < 8; ++m)
          if (r + 16 * m < D) sum = fmaf(load1(q + r + 16 * m), s[m], sum);
        part[r][c] = sum;
        __syncthreads();
        if (r == 0 && col < D) {
          for (int m = 1; m < 16; ++m) sum += part[m][c];
          store1(p.out + b * p.o_b + n * p.o_t + h * p.o_h + col, sum * p.scale);
        }
        __syncthreads();
      }
  }
#pragma unroll
  for (int m = 0; m < 8; ++m)
    if (p.state_out && r + 16 * m < D && col < D) p.state_out[at + (r + 16 * m) * D + col] = s[m];
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
  if ((long long)a->kv_heads * a->batch > 65535) return PD_ERR_UNSUPPORTED;
  if (!pointers || !a->batch || !a->heads) return PD_OK;
  if ((uintptr_t)a->slopes % 4 || (uintptr_t)a->lengths % 4 || (uintptr_t)a->state % 16 || (uintptr_t)a->state_out % 16) return PD_ERR_INVALID_ARG;
  if (!a->n) return PD_OK;
  if (!a->q || !a->k || !a->v || !a->out || a->out == a->q || a->out == a->k || a->out == a->v) return PD_ERR_INVALID_ARG;
  if (!rows16(a->q, a->q_batch_stride, a->q_token_stride, a->q_head_stride) ||
      !rows16(a->k, a->k_batch_stride, a->k_token_stride, a->k_head_stride) ||
      !rows16(a->v, a->v_batch_stride, a->v_token_stride, a->v_head_stride) ||
      !rows16(a->out, a->out_batch_stride, a->out_token_stride, a->out_head_stride))
    return PD_ERR_UNSUPPORTED;
  if (!rows_apart(a->head_dim, {{a->batch, a->out_batch_stride}, {a->n, a->out_token_stride}, {a->heads, a->out_head_stride}}))
    return PD_ERR_INVALID_ARG;
  return PD_OK;
}

}  // namespace

extern "C" size_t predecoder_linear_attention_workspace(const pd_linear_attention_args* a) { return 0; }

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
  hipLaunchKernelGGL(linear_simple_kernel, dim3((a->head_dim + 15) / 16, (unsigned)(a->kv_heads * a->batch)), dim3(256), 0,
                     (hipStream_t)hip_stream, p);
  return hipGetLastError() == hipSuccess ? PD_OK : PD_ERR_DEVICE;
}
