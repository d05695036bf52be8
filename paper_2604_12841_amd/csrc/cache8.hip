// cache8.hip -- keys and values of tokens into a ring of places in 8 bits, and
// back.
//
// A row is the keys or the values of one token and head: its scale is
// max |x| / Q, its codes x / scale rounded to the format (Q its largest value).
// A write takes 16 values a lane, a read 8; as many lanes as hold a row (a power of two) find its
// largest value among themselves.  A wave takes neighbouring tokens of one head,
// whose rows lie one behind the other in the cache, so it writes whole lines.
//
// A read is bound by memory (four caches of up to 39200 tokens, 2 heads of 64, to
// bf16: 21 us, 5.2 TB/s), a write of many tokens too (16 of 9800, 4 heads of 64: 58 us, 4.2 TB/s); one of a
// round of 64 streams (12.5 us, 2.5 TB/s) by vector instructions, whose units are 0.75 busy: the exact quotients, and
// workgroups of 128 tokens' rows that 196 tokens fill to 0.77.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/predecoder_ops.h"
#include "cache8.h"

namespace {

using namespace pd;

// (arrays of HIP's own vectors, which are structures, would go to LDS)
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int MANY = 2;  // rows a thread, in large writes (16 streams of 9800 tokens, 4 x 64 bf16: 58 us, with four 60, with one 76)

struct Cache8 {
  int batch, kv_heads, head_dim, capacity, tokens;
  unsigned token_blocks;
  uint8_t* codes;
  float* scales;
  i32x4* sites;
  const long long* at;
  const void* x[2];  // k, v
  void* y[2];
  long long b_stride[2], t_stride[2], h_stride[2];
  const i32x4* in_sites;
  i32x4* out_sites;
  long long sites_b;
};

// at mod capacity, and the place of token m <= capacity from there on.
__device__ __forceinline__ int start_of(long long at, int capacity) {
  if (at >= 0 && at < capacity) return (int)at;
  const long long p = at % capacity;
  return (int)(p < 0 ? p + capacity : p);
}
__device__ __forceinline__ int place_of(int start, int m, int capacity) {
  const unsigned p = (unsigned)start + (unsigned)m;
  return (int)(p < (unsigned)capacity ? p : p - (unsigned)capacity);
}

// x / s to 23 bits, the last of which is set where more follow: another rounding, to fewer bits, is the only one.
// r = 1 / s rounded.
__device__ __forceinline__ float quotient_odd(float x, float s, float r) {
  float t = x * r;
  t = fmaf(fmaf(-t, s, x), r, t);  // rounded to nearest
  const float rest = fmaf(-t, s, x);
  const uint32_t u = __float_as_uint(t);
  // an even t that the quotient is not: the neighbour on the quotient's side
  const uint32_t side = (__float_as_uint(rest) ^ u) >> 31 ? u - 1 : u + 1;
  return rest != 0.0f && !(u & 1) ? __uint_as_float(side) : t;
}

template <typename T, bool WIDE>
__device__ __forceinline__ void load_row16(const T* p, float* v) {
  if constexpr (WIDE) {
    load8(p, v);
    load8(p + 8, v + 8);
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = load1(p + e);
  }
}

// most / q, rounded to nearest: with 1 / q rounded, one correction makes it so where the rest is a number of the range.
template <bool INT8>
__device__ __forceinline__ float scale_of(float most) {
  constexpr float q = INT8 ? 127.0f : 448.0f, part = 1.0f / q;
  if (!(most > 0x1p-80f)) return most / q;
  const float s = most * part;
  return fmaf(fmaf(-s, q, most), part, s);
}

// N: rows a thread, loaded together.
template <typename T, int LPR, int N, bool INT8, bool WIDE>
__global__ void __launch_bounds__(256) cache_write_kernel(const Cache8 p) {
  constexpr int ROWS = 256 / LPR;
  const unsigned group = blockIdx.x / p.token_blocks;
  const int m0 = (int)(blockIdx.x % p.token_blocks) * (ROWS * N) + threadIdx.x / LPR, lane = threadIdx.x % LPR;
  const int h = group % p.kv_heads, which = group / p.kv_heads % 2, b = group / p.kv_heads / 2;
  const int d = min(16 * lane, p.head_dim - 16);  // (lanes past the row's end repeat its last values)
  const T* x = (const T*)p.x[which] + b * p.b_stride[which] + h * p.h_stride[which] + d;
  i32x4 site[N];
  float v[N][16];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int m = min(m0 + n * ROWS, p.tokens - 1);
    site[n] = p.in_sites[b * p.sites_b + m];
    load_row16<T, WIDE>(x + m * p.t_stride[which], v[n]);
  }
  const int start = start_of(p.at[b], p.capacity);
  const long long rows = ((long long)(b * 2 + which) * p.kv_heads + h) * p.capacity;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int m = m0 + n * ROWS;
    const bool there = m < p.tokens && site[n].w >= 0;
    float most = 0.0f;
    bool finite = true;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      most = fmaxf(most, fabsf(v[n][e]));
      finite = finite && fabsf(v[n][e]) < INFINITY;
    }
    if (!finite) most = INFINITY;
#pragma unroll
    for (int k = 1; k < LPR; k <<= 1) most = fmaxf(most, __shfl_xor(most, k));
    if (!there) continue;
    const float q = INT8 ? 127.0f : 448.0f;
    const float scale = most < INFINITY ? scale_of<INT8>(most) : NAN;
    const int place = place_of(start, m, p.capacity);
    if (lane == 0) p.scales[rows + place] = scale;
    if (lane == 0 && which == 0 && h == 0) p.sites[(long long)b * p.capacity + place] = site[n];
    u32x4 w = {0, 0, 0, 0};
    if (scale > 0.0f) {
      // (rows of tiny values are lifted, so that the rest of a division is a number of the range)
      const float lift = scale < 0x1p-60f ? 0x1p64f : 1.0f, s = scale * lift, r = 1.0f / s;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float c[4];
        // (a scale of few bits, below the normal range, may be too small for its row)
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = fminf(fmaxf(quotient_odd(v[n][4 * g + e] * lift, s, r), -q), q);
        w[g] = INT8 ? int8_pack4(c[0], c[1], c[2], c[3]) : e4m3_pack4_within(c[0], c[1], c[2], c[3]);
      }
    }
    if (16 * lane < p.head_dim) *(u32x4*)(p.codes + (rows + place) * p.head_dim + d) = w;
  }
}

// The values of eight codes.
template <bool INT8>
__device__ __forceinline__ void decode8(const u32x2 w, float* v) {
  const uint32_t u[2] = {w.x, w.y};
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    if constexpr (INT8) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * n + e] = (float)(int8_t)(u[n] >> 8 * e);
    } else {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(u[n], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(u[n], true);
      v[4 * n] = lo[0], v[4 * n + 1] = lo[1], v[4 * n + 2] = hi[0], v[4 * n + 3] = hi[1];
    }
  }
}

template <typename T, int LPR, bool INT8, bool WIDE>
__global__ void __launch_bounds__(256) cache_read_kernel(const Cache8 p) {
  constexpr int ROWS = 256 / LPR;
  const unsigned group = blockIdx.x / p.token_blocks;
  const int m = (int)(blockIdx.x % p.token_blocks) * ROWS + threadIdx.x / LPR, lane = threadIdx.x % LPR;
  const int h = group % p.kv_heads, which = group / p.kv_heads % 2, b = group / p.kv_heads / 2;
  if (m >= p.tokens) return;
  const int d = min(8 * lane, p.head_dim - 8);  // (lanes past the row's end repeat its last values)
  const int place = place_of(start_of(p.at[b], p.capacity), m, p.capacity);
  const long long row = ((long long)(b * 2 + which) * p.kv_heads + h) * p.capacity + place;
  const i32x4 site = p.sites[(long long)b * p.capacity + place];
  const u32x2 w = *(const u32x2*)(p.codes + row * p.head_dim + d);
  const float scale = p.scales[row];
  if (lane == 0 && which == 0 && h == 0 && p.out_sites) p.out_sites[b * p.sites_b + m] = site;
  if (8 * lane >= p.head_dim) return;
  float v[8];
  decode8<INT8>(w, v);
  // (without a token codes and scale may be anything)
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = site.w >= 0 ? v[e] * scale : 0.0f;
  T* y = (T*)p.y[which] + b * p.b_stride[which] + m * p.t_stride[which] + h * p.h_stride[which] + d;
  if constexpr (WIDE) {
    store8(y, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) store1(y + e, v[e]);
  }
}

template <typename T, bool INT8, bool WIDE>
void launch(const Cache8& p, bool write, bool many, long long groups, hipStream_t st) {
  auto go = [&](auto lanes) {
    constexpr int LPR = decltype(lanes)::value;
    const dim3 blocks((unsigned)(groups * p.token_blocks));
    if (write && many)
      hipLaunchKernelGGL((cache_write_kernel<T, LPR / 2, MANY, INT8, WIDE>), blocks, dim3(256), 0, st, p);
    else if (write)
      hipLaunchKernelGGL((cache_write_kernel<T, LPR / 2, 1, INT8, WIDE>), blocks, dim3(256), 0, st, p);
    else
      hipLaunchKernelGGL((cache_read_kernel<T, LPR, INT8, WIDE>), blocks, dim3(256), 0, st, p);
  };
  if (p.head_dim <= 32)
    go(std::integral_constant<int, 4>());
  else if (p.head_dim <= 64)
    go(std::integral_constant<int, 8>());
  else
    go(std::integral_constant<int, 16>());
}

pd_status run(void* hip_stream, const pd_cache_args* a, bool write) {
  if (!a) return PD_ERR_INVALID_ARG;
  const pd_status ok = check_cache(a->cache, false);
  if (ok != PD_OK) return ok;
  const pd_cache& c = a->cache;
  if (a->tokens < 0 || a->tokens > c.capacity) return PD_ERR_INVALID_ARG;
  if (a->dtype != PD_DTYPE_BF16 && a->dtype != PD_DTYPE_FP32) return PD_ERR_INVALID_ARG;
  if (!c.batch || !c.kv_heads || !a->tokens) return PD_OK;
  // lanes of a row: 8 values each, a write's 16
  const int lanes = (c.head_dim <= 32 ? 4 : c.head_dim <= 64 ? 8 : 16) / (write ? 2 : 1);
  const long long groups = 2ll * c.batch * c.kv_heads;
  // A write takes several rows a thread where the card is full all the same.
  const bool many = write && groups * a->tokens * lanes >= 256ll * 1024 * MANY;
  const int rows = 256 / lanes * (many ? MANY : 1);
  const long long blocks = ((long long)a->tokens + rows - 1) / rows;
  // (threads below 2^32, tokens and a block's more in 31 bits)
  if (groups * blocks >= 1ll << 24 || a->tokens > 1 << 30) return PD_ERR_UNSUPPORTED;
  if (check_cache(c, true) != PD_OK || !a->at || (uintptr_t)a->at % 8 || !a->k || !a->v || (write && !a->sites)) return PD_ERR_INVALID_ARG;
  const int elem = a->dtype == PD_DTYPE_BF16 ? 2 : 4;
  if ((uintptr_t)a->k % elem || (uintptr_t)a->v % elem || (uintptr_t)a->sites % 16) return PD_ERR_INVALID_ARG;
  if (!write) {
    if (!rows_apart(c.head_dim, {{c.batch, a->k_batch_stride}, {a->tokens, a->k_token_stride}, {c.kv_heads, a->k_head_stride}}) ||
        !rows_apart(c.head_dim, {{c.batch, a->v_batch_stride}, {a->tokens, a->v_token_stride}, {c.kv_heads, a->v_head_stride}}) || a->k == a->v)
      return PD_ERR_INVALID_ARG;
    if (a->sites && !rows_apart(a->tokens, {{c.batch, a->sites_batch_stride}})) return PD_ERR_INVALID_ARG;
  }
  Cache8 p;
  p.batch = c.batch, p.kv_heads = c.kv_heads, p.head_dim = c.head_dim, p.capacity = c.capacity, p.tokens = a->tokens;
  p.token_blocks = (unsigned)blocks;
  p.codes = (uint8_t*)c.codes, p.scales = c.scales, p.sites = (i32x4*)c.sites, p.at = (const long long*)a->at;
  p.x[0] = p.y[0] = a->k, p.x[1] = p.y[1] = a->v;
  p.b_stride[0] = a->k_batch_stride, p.t_stride[0] = a->k_token_stride, p.h_stride[0] = a->k_head_stride;
  p.b_stride[1] = a->v_batch_stride, p.t_stride[1] = a->v_token_stride, p.h_stride[1] = a->v_head_stride;
  p.in_sites = (const i32x4*)a->sites, p.out_sites = (i32x4*)a->sites, p.sites_b = a->sites_batch_stride;
  bool wide = true;
  for (int n = 0; n < 2; ++n)
    wide = wide && (uintptr_t)p.x[n] % 16 == 0 && p.b_stride[n] * elem % 16 == 0 && p.t_stride[n] * elem % 16 == 0 && p.h_stride[n] * elem % 16 == 0;
  const hipStream_t st = (hipStream_t)hip_stream;
  auto go = [&](auto type, auto int8) {
    using T = decltype(type);
    if (wide)
      launch<T, decltype(int8)::value, true>(p, write, many, groups, st);
    else
      launch<T, decltype(int8)::value, false>(p, write, many, groups, st);
  };
  const bool int8 = c.codes_type == PD_CODES_INT8, bf16 = a->dtype == PD_DTYPE_BF16;
  if (bf16 && int8)
    go(uint16_t(), std::true_type());
  else if (bf16)
    go(uint16_t(), std::false_type());
  else if (int8)
    go(float(), std::true_type());
  else
    go(float(), std::false_type());
  return hipGetLastError() == hipSuccess ? PD_OK : PD_ERR_DEVICE;
}

}  // namespace

extern "C" pd_status predecoder_cache_write(void* hip_stream, const pd_cache_args* args) { return run(hip_stream, args, true); }

extern "C" pd_status predecoder_cache_read(void* hip_stream, const pd_cache_args* args) { return run(hip_stream, args, false); }
