// C-ABI of the cached attention: arguments of cake_attend_cache and cake_attend_int4 (kernels: attend_rows.cu).
#include "attend.cuh"

#include <algorithm>

namespace cake {
namespace {


// Arguments that both forms of the cache have in common.
int32_t common_args(const cake_ctx* ctx, int32_t n_req, int32_t layer, const void* q, const int64_t* row_offsets,
                    const void* k_tail, const void* v_tail, const int32_t* tail_len, int64_t tail_capacity, void* out,
                    float* lse, const void* workspace, int64_t workspace_bytes, CacheParams& P) {
  if (!ctx || n_req < 0 || n_req > 65535) return CAKE_ERR_ARG;
  const cake_config& c = ctx->cfg;
  if (layer < 0 || layer >= c.n_layers) return CAKE_ERR_ARG;
  if (n_req > 0 && (!q || !row_offsets || !out || !workspace)) return CAKE_ERR_ARG;
  if (workspace_bytes < cake_attend_workspace_bytes(ctx, n_req)) return CAKE_ERR_CAPACITY;
  if (tail_capacity < 0 || tail_capacity > INT32_MAX) return CAKE_ERR_ARG;
  if (tail_capacity > 0 && (!k_tail || !v_tail || !tail_len)) return CAKE_ERR_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16) || !aligned(k_tail, 16) || !aligned(v_tail, 16)) return CAKE_ERR_ARG;
  if (!aligned(lse, 4) || !aligned(row_offsets, 8) || !aligned(tail_len, 4)) return CAKE_ERR_ARG;
  int dev = -1;
  CAKE_CUDA_TRY(cudaGetDevice(&dev));
  if (dev != ctx->device) return CAKE_ERR_ARG;
  P = {};
  P.q = q; P.row_off = row_offsets; P.out = out; P.lse = lse;
  if (tail_capacity > 0) { P.k_tail = k_tail; P.v_tail = v_tail; P.tail_len = tail_len; P.tail_cap = tail_capacity; }
  P.n_layers = c.n_layers; P.layer = layer; P.Hq = c.n_q_heads; P.Hkv = c.n_kv_heads;
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
  const int32_t rc = common_args(ctx, n_req, layer, q, row_offsets, k_tail, v_tail, tail_len, tail_capacity, out, lse, workspace,
                                 workspace_bytes, P);
  if (rc != CAKE_OK || n_req == 0) return rc;
  if (!k_cache || !v_cache || !aligned(k_cache, 16) || !aligned(v_cache, 16)) return CAKE_ERR_ARG;
  P.k = k_cache; P.v = v_cache;
  return launch_rows(ctx, n_req, P, workspace, (cudaStream_t)stream);
}

int32_t cake_attend_int4(const cake_ctx* ctx, int32_t n_req, int32_t layer, const void* q, const uint8_t* k_codes,
                         const float* k_scale, const float* k_zero, const uint8_t* v_codes, const float* v_scale,
                         const float* v_zero, int32_t group, const int64_t* row_offsets, const int64_t* kgroup_offsets,
                         const void* k_tail, const void* v_tail, const int32_t* tail_len, int64_t tail_capacity, void* out,
                         float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  CacheParams P;
  const int32_t rc = common_args(ctx, n_req, layer, q, row_offsets, k_tail, v_tail, tail_len, tail_capacity, out, lse, workspace,
                                 workspace_bytes, P);
  if (rc != CAKE_OK) return rc;
  if ((group != 32 && group != 64 && group != 128) || group > ctx->cfg.head_dim) return CAKE_ERR_ARG;
  if (n_req == 0) return CAKE_OK;
  if (!k_codes || !k_scale || !k_zero || !v_codes || !v_scale || !v_zero || !kgroup_offsets) return CAKE_ERR_ARG;
  if (!aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(k_scale, 16) || !aligned(k_zero, 16) || !aligned(v_scale, 16) ||
      !aligned(v_zero, 16) || !aligned(kgroup_offsets, 8)) return CAKE_ERR_ARG;
  P.k = k_codes; P.v = v_codes;
  P.k_scale = k_scale; P.k_zero = k_zero; P.v_scale = v_scale; P.v_zero = v_zero; P.group = group;
  P.group_off = kgroup_offsets;
  return launch_rows(ctx, n_req, P, workspace, (cudaStream_t)stream);
}

}  // extern "C"
