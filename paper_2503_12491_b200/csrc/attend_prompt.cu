// C-ABI of the attention over prompts: arguments of cake_attend_prompt and cake_accumulate_attention (kernels: attend_tc.cu for
// bf16, attend_tc32.cu for fp32).
#include "attend.cuh"

#include <algorithm>

namespace cake {

void fill_prompt_batch(const cake_ctx* ctx, int lo, int rows, PromptBatch& b) {
  b.n = std::min(ctx->n_req - lo, kPromptReqs);
  int order[kPromptReqs];
  for (int i = 0; i < b.n; ++i) order[i] = lo + i;
  auto len = [&](int r) { return ctx->h_cu[r + 1] - ctx->h_cu[r]; };
  std::sort(order, order + b.n, [&](int x, int y) { return len(x) != len(y) ? len(x) > len(y) : x < y; });
  b.tiles = 0;
  for (int i = 0; i < b.n; ++i) {
    b.first[i] = b.tiles;
    b.len[i] = (int32_t)len(order[i]);
    b.req[i] = order[i];
    b.cu[i] = ctx->h_cu[order[i]];
    b.tiles += (b.len[i] + rows - 1) / rows;
  }
  b.first[b.n] = b.tiles;
}

}  // namespace cake

using namespace cake;

extern "C" {

// (bounds under which no product of a stride and a number of heads or tokens overflows)
static constexpr int64_t kMaxHeadStride = (int64_t)1 << 38, kMaxTokenStride = (int64_t)1 << 31;
// Rows that the kernels read and write in 16-byte pieces.
static bool rows_ok(const cake_ctx* ctx, const void* p, int64_t head, int64_t token) {
  const int64_t es = ctx->cfg.dtype == CAKE_DTYPE_FP32 ? 4 : 2;
  return aligned(p, 16) && head >= 0 && token >= 0 && head < kMaxHeadStride && token < kMaxTokenStride &&
         head * es % 16 == 0 && token * es % 16 == 0;
}

// (Tokens have rows of their own, and a row of K or V has a number of 31 bits: a box of a copy is 128 rows of either.)
static bool queries_ok(const cake_ctx* ctx, const void* q, int64_t head, int64_t token) {
  return rows_ok(ctx, q, head, token) && token >= ctx->cfg.head_dim &&
         (int64_t)ctx->cfg.n_kv_heads * ctx->total_tokens < ((int64_t)1 << 31);
}

// A batch is there, and the device is the context's.
static int32_t batch_ok(const cake_ctx* ctx) {
  if (!ctx) return CAKE_ERR_ARG;
  if (ctx->n_req < 0) return CAKE_ERR_STATE;
  int dev = -1;
  CAKE_CUDA_TRY(cudaGetDevice(&dev));
  return dev == ctx->device ? CAKE_OK : CAKE_ERR_ARG;
}

int32_t cake_attend_prompt(cake_ctx* ctx, const void* q, int64_t q_head_stride, int64_t q_token_stride, const void* k,
                           const void* v, void* out, int64_t out_head_stride, int64_t out_token_stride, float* lse,
                           float* lse_window, void* stream) {
  const int32_t ok = batch_ok(ctx);
  if (ok != CAKE_OK || ctx->n_req == 0) return ok;
  const int64_t d = ctx->cfg.head_dim;
  if (!q || !k || !v || !out) return CAKE_ERR_ARG;
  if (!queries_ok(ctx, q, q_head_stride, q_token_stride) || !rows_ok(ctx, k, 0, 0) || !rows_ok(ctx, v, 0, 0) ||
      !rows_ok(ctx, out, out_head_stride, out_token_stride)) return CAKE_ERR_ARG;
  if (!aligned(lse, 4) || !aligned(lse_window, 4)) return CAKE_ERR_ARG;
  // rows of the output that share memory would be written twice
  const int64_t heads = ctx->cfg.n_q_heads, tokens = ctx->total_tokens;
  const bool by_token = out_head_stride >= d && out_token_stride >= d && out_token_stride - d >= (heads - 1) * out_head_stride;
  const bool by_head = out_token_stride >= d && out_head_stride >= d && out_head_stride - d >= (tokens - 1) * out_token_stride;
  if (!by_token && !(heads == 1 && out_token_stride >= d) && !by_head) return CAKE_ERR_ARG;
  const Strided qs = {q_head_stride, q_token_stride}, os = {out_head_stride, out_token_stride};
  return (ctx->cfg.dtype == CAKE_DTYPE_FP32 ? launch_prompt_tc32 : launch_prompt_tc)(ctx, q, qs, k, v, out, os, lse, lse_window,
                                                                                (cudaStream_t)stream);
}

int32_t cake_accumulate_attention(cake_ctx* ctx, const void* q, int64_t q_head_stride, int64_t q_token_stride, const void* k,
                                  const float* lse, float* out, void* stream) {
  const int32_t ok = batch_ok(ctx);
  if (ok != CAKE_OK || ctx->n_req == 0) return ok;
  if (!q || !k || !lse || !out) return CAKE_ERR_ARG;
  if (!queries_ok(ctx, q, q_head_stride, q_token_stride) || !rows_ok(ctx, k, 0, 0)) return CAKE_ERR_ARG;
  if (!aligned(lse, 4) || !aligned(out, 4)) return CAKE_ERR_ARG;
  const Strided qs = {q_head_stride, q_token_stride};
  return (ctx->cfg.dtype == CAKE_DTYPE_FP32 ? launch_accumulate_tc32 : launch_accumulate_tc)(ctx, q, qs, k, lse, out, (cudaStream_t)stream);
}

}  // extern "C"
