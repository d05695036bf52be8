// attention.hip -- grouped-head attention over the tokens of detector volumes:
// scores capped by a tanh, a bias by the distance of the sites, masks by
// volume, round and prefix.
//
// One pass over the keys with the running maximum and sum of the softmax.  The
// heads that share keys are rows of one query matrix: row r is token
// r / group, head r % group of the key head's group.  A workgroup takes 128
// rows, a wave 32, and 64 keys at a time come through LDS.  A wave computes
// the transposed scores K Q^T, so a lane holds 32 of the 64 scores of one row
// (the other half of the wave the rest): maximum and sum need one exchange.
// The same registers, rounded to bf16, are the right operand of
// out^T += V^T P^T, whose sum over keys may run in any order as long as V
// follows it.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/predecoder_ops.h"
#include "token_values.h"

namespace {

using namespace pd;

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr float LOG2E = 1.4426950408889634f;
constexpr int TK = 64;     // keys of a tile
constexpr int ROWS = 128;  // query rows of a workgroup

struct Attn {
  int heads, kv_heads, group, head_dim;
  int n_q, n_k;
  long long rows;  // n_q * group
  int causal, prefix;
  float scale, cap;  // cap 0: none
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* out;
  long long q_b, q_t, q_h, k_b, k_t, k_h, v_b, v_t, v_h, o_b, o_t, o_h;
  const int4* q_sites;
  const int4* k_sites;
  long long q_sites_b, k_sites_b;
  const float* slopes;
};

// |a - b| + c
__device__ __forceinline__ uint32_t far_add(int a, int b, uint32_t c) {
  return (uint32_t)((a > b ? a : b) - (a > b ? b : a)) + c;
}

template <int DP>
__global__ void __launch_bounds__(256) attention_kernel(const Attn p) {
  constexpr int KP = DP * 2 + 16;  // bytes of a key's row in LDS
  constexpr int VP = TK * 2 + 16;  // bytes of a row of V^T
  __shared__ __attribute__((aligned(16))) uint8_t lk[TK * KP];
  __shared__ __attribute__((aligned(16))) uint8_t lv[DP * VP];
  __shared__ int4 ls[TK];
  __shared__ int odd_v;  // the tile of V holds an infinity or a NaN
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  const int kvh = blockIdx.y, b = blockIdx.z;
  const long long row = (long long)blockIdx.x * ROWS + wave * 32 + (lane & 31);
  const long long r = row < p.rows ? row : p.rows - 1;
  const int token = (int)(r / p.group), head = kvh * p.group + (int)(r % p.group);
  const uint16_t* q = p.q + b * p.q_b + token * p.q_t + head * p.q_h;
  const uint16_t* kb = p.k + b * p.k_b + kvh * p.k_h;
  const uint16_t* vb = p.v + b * p.v_b + kvh * p.v_h;
  bf16x8 fq[DP / 16];
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    const int d = 16 * s + 8 * half;
    const uint4 w = d < p.head_dim ? *(const uint4*)(q + d) : make_uint4(0, 0, 0, 0);
    fq[s] = __builtin_bit_cast(bf16x8, w);
  }
  const int4 at = p.q_sites ? p.q_sites[b * p.q_sites_b + token] : make_int4(0, 0, 0, 0);
  const float slope = p.slopes ? p.slopes[head] : 0.0f;
  f32x16 o[DP / 32];
#pragma unroll
  for (int n = 0; n < DP / 32; ++n)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[n][e] = 0.0f;
  float top = -INFINITY, total = 0.0f;
  for (int k0 = 0; k0 < p.n_k; k0 += TK) {
    __syncthreads();
    if (tid == 0) odd_v = 0;
    if (tid < TK) {
      const int key = k0 + tid;
      int4 s = make_int4(0, 0, 0, -1);
      if (key < p.n_k) s = p.k_sites ? p.k_sites[b * p.k_sites_b + key] : make_int4(0, 0, 0, 0);
      ls[tid] = s;
    }
    __syncthreads();
    for (int c = tid; c < TK * (DP / 8); c += 256) {
      const int kk = c / (DP / 8), d = (c % (DP / 8)) * 8;
      const bool there = k0 + kk < p.n_k && d < p.head_dim;
      const long long key = k0 + kk;
      const uint4 wk = there ? *(const uint4*)(kb + key * p.k_t + d) : make_uint4(0, 0, 0, 0);
      const uint4 wv = there ? *(const uint4*)(vb + key * p.v_t + d) : make_uint4(0, 0, 0, 0);
      *(uint4*)(lk + kk * KP + d * 2) = wk;
      const uint32_t u[4] = {wv.x, wv.y, wv.z, wv.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint16_t x = (uint16_t)(u[e >> 1] >> (16 * (e & 1)));
        if ((x & 0x7f80) == 0x7f80) odd_v = 1;
        *(uint16_t*)(lv + (d + e) * VP + kk * 2) = x;
      }
    }
    __syncthreads();
    f32x16 z[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
#pragma unroll
      for (int e = 0; e < 16; ++e) z[n][e] = 0.0f;
#pragma unroll
      for (int s = 0; s < DP / 16; ++s) {
        const uint4 w = *(const uint4*)(lk + (32 * n + (lane & 31)) * KP + (16 * s + 8 * half) * 2);
        z[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), fq[s], z[n], 0, 0, 0);
      }
    }
    float most = -INFINITY;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int4 key = ls[32 * n + 8 * (e >> 2) + 4 * half + (e & 3)];
        float x = z[n][e] * p.scale;
        if (p.cap > 0.0f)
          x = p.cap - 2.0f * p.cap * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * (2.0f * LOG2E / p.cap)));
        if (p.slopes) x -= slope * (float)far_add(at.x, key.x, far_add(at.y, key.y, far_add(at.z, key.z, 0)));
        const bool seen = key.w == at.w && key.w >= 0 && (!p.causal || key.x <= at.x || key.x < p.prefix);
        x = seen ? x * LOG2E : -INFINITY;
        z[n][e] = x;
        most = fmaxf(most, x);
      }
    most = fmaxf(most, __shfl_xor(most, 32));
    const float was = top;
    top = fmaxf(top, most);
    const float base = top == -INFINITY ? 0.0f : top;
    const float alpha = __builtin_amdgcn_exp2f(was - base);
    total *= alpha;
#pragma unroll
    for (int n = 0; n < DP / 32; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[n][e] *= alpha;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        z[n][e] = __builtin_amdgcn_exp2f(z[n][e] - base);
        total += z[n][e];
      }
    if (odd_v) {
      // 0 x infinity: only the keys that a row sees may touch it
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          for (int h = 0; h < 2; ++h) {
            const float pr = bf16_round(__shfl(n ? z[1][e] : z[0][e], (lane & 31) + 32 * h));
            const int kk = 32 * n + 8 * (e >> 2) + 4 * h + (e & 3);
            if (pr != 0.0f) {
#pragma unroll
              for (int m = 0; m < DP / 32; ++m)
#pragma unroll
                for (int f = 0; f < 16; ++f) {
                  const int d = 32 * m + 8 * (f >> 2) + 4 * half + (f & 3);
                  o[m][f] = fmaf(pr, load1((const uint16_t*)(lv + d * VP + kk * 2)), o[m][f]);
                }
            }
          }
    } else {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          uint4 w;
          w.x = bf16_pack(z[n][8 * s], z[n][8 * s + 1]), w.y = bf16_pack(z[n][8 * s + 2], z[n][8 * s + 3]);
          w.z = bf16_pack(z[n][8 * s + 4], z[n][8 * s + 5]), w.w = bf16_pack(z[n][8 * s + 6], z[n][8 * s + 7]);
#pragma unroll
          for (int m = 0; m < DP / 32; ++m) {
            const uint8_t* f = lv + (32 * m + (lane & 31)) * VP + (32 * n + 16 * s + 4 * half) * 2;
            const uint2 lo = *(const uint2*)f, hi = *(const uint2*)(f + 16);
            o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                __builtin_bit_cast(bf16x8, make_uint4(lo.x, lo.y, hi.x, hi.y)), __builtin_bit_cast(bf16x8, w), o[m], 0,
                0, 0);
          }
        }
    }
  }
  total += __shfl_xor(total, 32);
  if (row >= p.rows) return;
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

bool rows16(const void* p, long long b, long long t, long long h) {
  return (uintptr_t)p % 16 == 0 && b % 8 == 0 && t % 8 == 0 && h % 8 == 0;
}

// The argument checks: sizes alone, or with the pointers.
pd_status check(const pd_attention_args* a, bool pointers) {
  if (!a || a->batch < 0 || a->heads < 0 || a->kv_heads < 0 || a->n_q < 0 || a->n_k < 0) return PD_ERR_INVALID_ARG;
  if (a->head_dim < 1 || !(fabsf(a->scale) < INFINITY) || !(a->cap >= 0.0f) || !(a->cap < INFINITY))
    return PD_ERR_INVALID_ARG;
  if (a->causal < 0 || a->causal > 1 || a->prefix < 0 || (a->prefix && !a->causal)) return PD_ERR_INVALID_ARG;
  if (a->heads && (!a->kv_heads || a->heads % a->kv_heads)) return PD_ERR_INVALID_ARG;
  if (a->head_dim % 8 || a->head_dim > 128) return PD_ERR_UNSUPPORTED;
  if (a->heads && a->heads / a->kv_heads > 64) return PD_ERR_UNSUPPORTED;
  if (a->kv_heads > 65535 || a->batch > 65535) return PD_ERR_UNSUPPORTED;  // the grid's axes
  if (a->heads && (long long)a->n_q * (a->heads / a->kv_heads) >= 1ll << 30) return PD_ERR_UNSUPPORTED;  // its threads
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
  const size_t need = predecoder_attention_workspace(a);
  if (need && (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < need)) return PD_ERR_INVALID_ARG;
  return PD_OK;
}

}  // namespace

extern "C" size_t predecoder_attention_workspace(const pd_attention_args* a) { return check(a, false) != PD_OK ? 0 : 0; }

extern "C" pd_status predecoder_attention(void* hip_stream, const pd_attention_args* a) {
  const pd_status ok = check(a, true);
  if (ok != PD_OK) return ok;
  if (!a->batch || !a->heads || !a->n_q) return PD_OK;
  Attn p;
  p.heads = a->heads, p.kv_heads = a->kv_heads, p.group = a->heads / a->kv_heads, p.head_dim = a->head_dim;
  p.n_q = a->n_q, p.n_k = a->n_k, p.rows = (long long)a->n_q * p.group;
  p.causal = a->causal, p.prefix = a->prefix, p.scale = a->scale, p.cap = a->cap;
  p.q = (const uint16_t*)a->q, p.k = (const uint16_t*)a->k, p.v = (const uint16_t*)a->v, p.out = (uint16_t*)a->out;
  p.q_b = a->q_batch_stride, p.q_t = a->q_token_stride, p.q_h = a->q_head_stride;
  p.k_b = a->k_batch_stride, p.k_t = a->k_token_stride, p.k_h = a->k_head_stride;
  p.v_b = a->v_batch_stride, p.v_t = a->v_token_stride, p.v_h = a->v_head_stride;
  p.o_b = a->out_batch_stride, p.o_t = a->out_token_stride, p.o_h = a->out_head_stride;
  p.q_sites = (const int4*)a->q_sites, p.k_sites = (const int4*)a->k_sites;
  p.q_sites_b = a->q_sites_batch_stride, p.k_sites_b = a->k_sites_batch_stride;
  p.slopes = a->slopes;
  const long long tiles = (p.rows + ROWS - 1) / ROWS;
  const dim3 grid((unsigned)tiles, (unsigned)a->kv_heads, (unsigned)a->batch);
  const hipStream_t st = (hipStream_t)hip_stream;
  if (a->head_dim <= 32)
    hipLaunchKernelGGL(attention_kernel<32>, grid, dim3(256), 0, st, p);
  else if (a->head_dim <= 64)
    hipLaunchKernelGGL(attention_kernel<64>, grid, dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL(attention_kernel<128>, grid, dim3(256), 0, st, p);
  return hipGetLastError() == hipSuccess ? PD_OK : PD_ERR_DEVICE;
}
