// Attention of one new token per request over its cached rows: the packed cache of retained rows (cake_compact, or the
// decode cache), or the same rows in 4 bits (cake_compact_int4), and behind either the rows of tokens generated since.
//
//   O_h = sum_j softmax_j(q_h.k_j / sqrt d) v_j ,  lse_h = log sum_j exp(q_h.k_j / sqrt d)   over all rows j of h's KV head.
//
// One CTA per (request, KV head): a warp takes every eighth row, keeps a running maximum, sum and output of the head's
// query heads, and the warps' results are merged at the end.
#include "attend.cuh"

#include <algorithm>

namespace cake {
namespace {

constexpr int WARPS = 8;
constexpr int MAXG = 8;              // query heads per KV head (cake_create allows no more)

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void narrow(float* p, float x) { *p = x; }
__device__ __forceinline__ void narrow(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

template <typename T, int D, bool kInt4>
__global__ void __launch_bounds__(WARPS * 32) attend_rows(const CacheParams P) {
  constexpr int C = D / 32;                        // channels per lane
  __shared__ float s_m[WARPS][MAXG], s_l[WARPS][MAXG], s_o[WARPS][MAXG][D];
  const int g = blockIdx.x, r = blockIdx.y, G = P.Hq / P.Hkv, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t block = (int64_t)r * P.n_layers + P.layer, row0 = P.row_off[block];
  const int64_t n = (P.row_off[block + 1] - row0) / P.Hkv;
  const int64_t tail = P.tail_len ? max((int64_t)0, min((int64_t)P.tail_len[r], P.tail_cap)) : 0;
  const int64_t first = row0 + g * n;
  float q[MAXG][C], o[MAXG][C], m[MAXG], l[MAXG];
#pragma unroll
  for (int h = 0; h < MAXG; ++h) {
    m[h] = -CUDART_INF_F;
    l[h] = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      q[h][c] = h < G ? widen(((const T*)P.q)[((int64_t)r * P.Hq + g * G + h) * D + lane * C + c]) : 0.f;
      o[h][c] = 0.f;
    }
  }
  for (int64_t j = warp; j < n + tail; j += WARPS) {
    float k[C], v[C];
    if (j >= n) {
      const int64_t at = (((int64_t)r * P.Hkv + g) * P.tail_cap + (j - n)) * D + lane * C;
#pragma unroll
      for (int c = 0; c < C; ++c) { k[c] = widen(((const T*)P.k_tail)[at + c]); v[c] = widen(((const T*)P.v_tail)[at + c]); }
    } else if constexpr (kInt4) {
      const int64_t row = first + j, kg = P.group_off[block] + g * ((n + P.group - 1) / P.group) + j / P.group;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int ch = lane * C + c;
        const int kc = ((const uint8_t*)P.k)[row * (D / 2) + ch / 2] >> (4 * (ch & 1)) & 15;
        const int vc = ((const uint8_t*)P.v)[row * (D / 2) + ch / 2] >> (4 * (ch & 1)) & 15;
        k[c] = fmaf((float)kc, P.k_scale[kg * D + ch], P.k_zero[kg * D + ch]);
        const int64_t vg = row * (D / P.group) + ch / P.group;
        v[c] = fmaf((float)vc, P.v_scale[vg], P.v_zero[vg]);
      }
    } else {
      const int64_t at = (first + j) * D + lane * C;
#pragma unroll
      for (int c = 0; c < C; ++c) { k[c] = widen(((const T*)P.k)[at + c]); v[c] = widen(((const T*)P.v)[at + c]); }
    }
#pragma unroll
    for (int h = 0; h < MAXG; ++h) {
      if (h >= G) break;
      float s = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) s = fmaf(q[h][c], k[c], s);
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
      const float top = fmaxf(m[h], s), f = exp2f((m[h] - top) * P.scale2), e = exp2f((s - top) * P.scale2);
      m[h] = top;
      l[h] = fmaf(l[h], f, e);
#pragma unroll
      for (int c = 0; c < C; ++c) o[h][c] = fmaf(o[h][c], f, e * v[c]);
    }
  }
#pragma unroll
  for (int h = 0; h < MAXG; ++h) {
    if (lane == 0) { s_m[warp][h] = m[h]; s_l[warp][h] = l[h]; }
#pragma unroll
    for (int c = 0; c < C; ++c) s_o[warp][h][lane * C + c] = o[h][c];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < G * D; i += WARPS * 32) {
    const int h = i / D, c = i % D;
    float top = -CUDART_INF_F, sum = 0.f, acc = 0.f;
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, s_m[w][h]);
    for (int w = 0; w < WARPS; ++w) {
      if (s_l[w][h] == 0.f) continue;              // a warp without rows
      const float f = exp2f((s_m[w][h] - top) * P.scale2);
      sum = fmaf(s_l[w][h], f, sum);
      acc = fmaf(s_o[w][h][c], f, acc);
    }
    const int64_t at = (int64_t)r * P.Hq + g * G + h;
    // no rows at all: an output of zero and a log-sum-exp of -inf, which merges into nothing
    narrow((T*)P.out + at * D + c, n + tail > 0 ? acc / sum : 0.f);
    if (P.lse && c == 0) P.lse[at] = n + tail > 0 ? fmaf(top, P.scale, logf(sum)) : -CUDART_INF_F;
  }
}

template <bool kInt4>
int32_t launch_attend_rows(const cake_ctx* ctx, int32_t n_req, const CacheParams& P, cudaStream_t st) {
  const bool f32 = ctx->cfg.dtype == CAKE_DTYPE_FP32, wide = ctx->cfg.head_dim == 128;
  const dim3 grid((unsigned)P.Hkv, (unsigned)n_req);
  if (f32 && wide) attend_rows<float, 128, kInt4><<<grid, WARPS * 32, 0, st>>>(P);
  else if (f32) attend_rows<float, 64, kInt4><<<grid, WARPS * 32, 0, st>>>(P);
  else if (wide) attend_rows<__nv_bfloat16, 128, kInt4><<<grid, WARPS * 32, 0, st>>>(P);
  else attend_rows<__nv_bfloat16, 64, kInt4><<<grid, WARPS * 32, 0, st>>>(P);
  count_launch();
  return cuda_status(cudaGetLastError());
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Arguments that both forms of the cache have in common.
int32_t common_args(const cake_ctx* ctx, int32_t n_req, int32_t layer, const void* q, const int64_t* row_offsets,
                    const void* k_tail, const void* v_tail, const int32_t* tail_len, int64_t tail_capacity, void* out,
                    const void* workspace, int64_t workspace_bytes, CacheParams& P) {
  if (!ctx || n_req < 0 || n_req > 65535) return CAKE_ERR_ARG;
  const cake_config& c = ctx->cfg;
  if (layer < 0 || layer >= c.n_layers) return CAKE_ERR_ARG;
  if (n_req > 0 && (!q || !row_offsets || !out || !workspace)) return CAKE_ERR_ARG;
  if (workspace_bytes < cake_attend_workspace_bytes(ctx, n_req)) return CAKE_ERR_CAPACITY;
  if (tail_capacity < 0 || tail_capacity > INT32_MAX) return CAKE_ERR_ARG;
  if (tail_capacity > 0 && (!k_tail || !v_tail || !tail_len)) return CAKE_ERR_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace) || !aligned16(k_tail) || !aligned16(v_tail)) return CAKE_ERR_ARG;
  int dev = -1;
  CAKE_CUDA_TRY(cudaGetDevice(&dev));
  if (dev != ctx->device) return CAKE_ERR_ARG;
  P = {};
  P.q = q; P.row_off = row_offsets; P.out = out;
  if (tail_capacity > 0) { P.k_tail = k_tail; P.v_tail = v_tail; P.tail_len = tail_len; P.tail_cap = tail_capacity; }
  P.n_layers = c.n_layers; P.layer = layer; P.Hq = c.n_q_heads; P.Hkv = c.n_kv_heads;
  P.scale = 1.f / sqrtf((float)c.head_dim);
  P.scale2 = kLog2E / sqrtf((float)c.head_dim);
  return CAKE_OK;
}

}  // namespace
}  // namespace cake

using namespace cake;

extern "C" {

int64_t cake_attend_workspace_bytes(const cake_ctx* ctx, int32_t n_req) {
  if (!ctx || n_req < 0) return CAKE_ERR_ARG;
  return std::max<int64_t>(16, rows_workspace(ctx));
}

int32_t cake_attend_cache(const cake_ctx* ctx, int32_t n_req, int32_t layer, const void* q, const void* k_cache,
                          const void* v_cache, const int64_t* row_offsets, const void* k_tail, const void* v_tail,
                          const int32_t* tail_len, int64_t tail_capacity, void* out, float* lse, void* workspace,
                          int64_t workspace_bytes, void* stream) {
  CacheParams P;
  const int32_t rc = common_args(ctx, n_req, layer, q, row_offsets, k_tail, v_tail, tail_len, tail_capacity, out, workspace,
                                 workspace_bytes, P);
  if (rc != CAKE_OK || n_req == 0) return rc;
  if (!k_cache || !v_cache || !aligned16(k_cache) || !aligned16(v_cache)) return CAKE_ERR_ARG;
  P.k = k_cache; P.v = v_cache; P.lse = lse;
  if (ctx->cfg.dtype == CAKE_DTYPE_BF16) return launch_rows(ctx, n_req, P, workspace, (cudaStream_t)stream);
  return launch_attend_rows<false>(ctx, n_req, P, (cudaStream_t)stream);
}

int32_t cake_attend_int4(const cake_ctx* ctx, int32_t n_req, int32_t layer, const void* q, const uint8_t* k_codes,
                         const float* k_scale, const float* k_zero, const uint8_t* v_codes, const float* v_scale,
                         const float* v_zero, int32_t group, const int64_t* row_offsets, const int64_t* kgroup_offsets,
                         const void* k_tail, const void* v_tail, const int32_t* tail_len, int64_t tail_capacity, void* out,
                         float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  CacheParams P;
  const int32_t rc = common_args(ctx, n_req, layer, q, row_offsets, k_tail, v_tail, tail_len, tail_capacity, out, workspace,
                                 workspace_bytes, P);
  if (rc != CAKE_OK) return rc;
  if ((group != 32 && group != 64 && group != 128) || group > ctx->cfg.head_dim) return CAKE_ERR_ARG;
  if (n_req == 0) return CAKE_OK;
  if (!k_codes || !k_scale || !k_zero || !v_codes || !v_scale || !v_zero || !kgroup_offsets) return CAKE_ERR_ARG;
  if (!aligned16(k_codes) || !aligned16(v_codes) || !aligned16(k_scale) || !aligned16(k_zero) || !aligned16(v_scale) ||
      !aligned16(v_zero)) return CAKE_ERR_ARG;
  P.k = k_codes; P.v = v_codes; P.lse = lse;
  P.k_scale = k_scale; P.k_zero = k_zero; P.v_scale = v_scale; P.v_zero = v_zero; P.group = group;
  P.group_off = kgroup_offsets;
  if (ctx->cfg.dtype == CAKE_DTYPE_BF16) return launch_rows(ctx, n_req, P, workspace, (cudaStream_t)stream);
  return launch_attend_rows<true>(ctx, n_req, P, (cudaStream_t)stream);
}

}  // extern "C"
