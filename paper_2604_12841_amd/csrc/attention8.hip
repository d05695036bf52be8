// attention8.hip -- attention of new tokens over a cache in 8 bits: scores
// capped by a tanh, a bias by the distance of the sites, masks by volume, round
// and prefix.
//
// One wave a query token and head, 64 keys at a time: a lane takes the score of
// one key, maximum and sum run over the tiles, then a lane holds one or two columns
// of the result.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>

#include "cache8.h"

namespace {

using namespace pd;

constexpr float LOG2E = 1.4426950408889634f;

struct Attn8 {
  int batch, heads, kv_heads, group, head_dim, n_q, capacity;
  int causal, prefix_last;
  float scale, cap;
  const uint16_t* q;
  uint16_t* out;
  long long q_b, q_t, q_h, o_b, o_t, o_h;
  const uint8_t* codes;
  const float* scales;
  const int4* sites;
  const int4* q_sites;
  long long q_sites_b;
  const float* slopes;
};

template <bool INT8>
__device__ __forceinline__ float decode1(uint8_t c) {
  if constexpr (INT8)
    return (float)(int8_t)c;
  else
    return __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
}

template <bool INT8>
__global__ void __launch_bounds__(64) attention8_simple_kernel(const Attn8 p) {
  __shared__ float qs[128], ps[64];
  const int lane = threadIdx.x;
  const int token = blockIdx.x % p.n_q, h = blockIdx.x / p.n_q % p.heads, b = blockIdx.x / p.n_q / p.heads, kvh = h / p.group;
  const uint16_t* q = p.q + b * p.q_b + token * p.q_t + h * p.q_h;
  for (int d = lane; d < p.head_dim; d += 64) qs[d] = load1(q + d);
  __syncthreads();
  const int4 at = p.q_sites[b * p.q_sites_b + token];
  const int last = p.causal ? max(at.x, p.prefix_last) : INT_MAX;
  const float slope = p.slopes ? p.slopes[h] : 0.0f;
  const long long k_row = ((long long)(b * 2) * p.kv_heads + kvh) * p.capacity, v_row = k_row + (long long)p.kv_heads * p.capacity;
  float top = -INFINITY, total = 0.0f, o[2] = {};
  for (int k0 = 0; k0 < p.capacity; k0 += 64) {
    const int key = k0 + lane;
    float z = -INFINITY;
    if (key < p.capacity) {
      const int4 s = p.sites[(long long)b * p.capacity + key];
      if (s.w == at.w && s.w >= 0 && s.x <= last) {
        float sum = 0.0f;
        for (int d = 0; d < p.head_dim; ++d) sum = fmaf(qs[d], decode1<INT8>(p.codes[(k_row + key) * p.head_dim + d]), sum);
        z = sum * p.scales[k_row + key] * p.scale;
        if (p.cap > 0.0f) z = p.cap * tanhf(z / p.cap);
        if (p.slopes) z -= slope * (float)(abs(s.x - at.x) + abs(s.y - at.y) + abs(s.z - at.z));
      }
    }
    const uint64_t seen = __ballot(!(z == -INFINITY));
    if (!seen) continue;
    float most = z;
    for (int n = 1; n < 64; n <<= 1) most = fmaxf(most, __shfl_xor(most, n));
    most = fmaxf(most, top);
    const float fade = top == -INFINITY ? 0.0f : exp2f((top - most) * LOG2E);
    const float e = z == -INFINITY ? 0.0f : exp2f((z - most) * LOG2E);
    total = total * fade + e;
    top = most;
    ps[lane] = key < p.capacity && e != 0.0f ? e * p.scales[v_row + key] : 0.0f;
    __syncthreads();
    for (int c = 0; c < 2; ++c) {
      const int d = lane + 64 * c;
      if (d >= p.head_dim) continue;
      o[c] *= fade;
      for (uint64_t left = seen; left; left &= left - 1) {
        const int n = __builtin_ctzll(left);
        o[c] = fmaf(ps[n], decode1<INT8>(p.codes[(v_row + k0 + n) * p.head_dim + d]), o[c]);
      }
    }
    __syncthreads();
  }
  for (int n = 1; n < 64; n <<= 1) total += __shfl_xor(total, n);
  const float inv = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : NAN;
  for (int c = 0; c < 2; ++c)
    if (lane + 64 * c < p.head_dim) store1(p.out + b * p.o_b + token * p.o_t + h * p.o_h + lane + 64 * c, o[c] * inv);
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
  if ((__int128)a->n_q * a->heads * c.batch >= 1ll << 24) return PD_ERR_UNSUPPORTED;
  if (!pointers || !c.batch || !a->heads || !a->n_q) return PD_OK;
  if (!a->q || !a->out || !a->q_sites || a->out == a->q) return PD_ERR_INVALID_ARG;
  if (c.capacity && check_cache(c, true) != PD_OK) return PD_ERR_INVALID_ARG;
  if ((uintptr_t)a->q_sites % 16 || (uintptr_t)a->slopes % 4) return PD_ERR_INVALID_ARG;
  if (!rows16(a->q, a->q_batch_stride, a->q_token_stride, a->q_head_stride) ||
      !rows16(a->out, a->out_batch_stride, a->out_token_stride, a->out_head_stride))
    return PD_ERR_UNSUPPORTED;
  if (!rows_apart(c.head_dim, {{c.batch, a->out_batch_stride}, {a->n_q, a->out_token_stride}, {a->heads, a->out_head_stride}}))
    return PD_ERR_INVALID_ARG;
  return PD_OK;
}

}  // namespace

extern "C" size_t predecoder_attention8_workspace(const pd_attention8_args* a) { return 0; }

extern "C" pd_status predecoder_attention8(void* hip_stream, const pd_attention8_args* a) {
  const pd_status ok = check(a, true);
  if (ok != PD_OK) return ok;
  const pd_cache& c = a->cache;
  if (!c.batch || !a->heads || !a->n_q) return PD_OK;
  Attn8 p;
  p.batch = c.batch, p.heads = a->heads, p.kv_heads = c.kv_heads, p.group = a->heads / c.kv_heads, p.head_dim = c.head_dim;
  p.n_q = a->n_q, p.capacity = c.capacity, p.causal = a->causal;
  p.prefix_last = a->prefix == PD_PREFIX_NONE ? INT_MIN : a->prefix - 1;
  p.scale = a->scale, p.cap = a->cap;
  p.q = (const uint16_t*)a->q, p.out = (uint16_t*)a->out;
  p.q_b = a->q_batch_stride, p.q_t = a->q_token_stride, p.q_h = a->q_head_stride;
  p.o_b = a->out_batch_stride, p.o_t = a->out_token_stride, p.o_h = a->out_head_stride;
  p.codes = (const uint8_t*)c.codes, p.scales = c.scales, p.sites = (const int4*)c.sites;
  p.q_sites = (const int4*)a->q_sites, p.q_sites_b = a->q_sites_batch_stride, p.slopes = a->slopes;
  const dim3 grid((unsigned)(a->n_q * a->heads * c.batch));
  if (c.codes_type == PD_CODES_INT8)
    hipLaunchKernelGGL(attention8_simple_kernel<true>, grid, dim3(64), 0, (hipStream_t)hip_stream, p);
  else
    hipLaunchKernelGGL(attention8_simple_kernel<false>, grid, dim3(64), 0, (hipStream_t)hip_stream, p);
  return hipGetLastError() == hipSuccess ? PD_OK : PD_ERR_DEVICE;
}
