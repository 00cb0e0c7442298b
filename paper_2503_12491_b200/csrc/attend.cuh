// What the attention kernels over prompts and caches share.
#pragma once

#include "cake_internal.cuh"

#include <math_constants.h>

namespace cake {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2E = 1.4426950408889634f;

// Up to kPromptReqs requests of a batch, longest first, as a kernel parameter: a launch needs no table in device
// memory, so a captured one stays valid whatever the context does next.
constexpr int kPromptReqs = 128;
struct PromptBatch {
  int32_t n, tiles;                    // requests; tiles of all of them
  int32_t first[kPromptReqs + 1];      // first tile of every request
  int32_t len[kPromptReqs];            // its tokens
  int32_t req[kPromptReqs];            // its place in the batch
  int64_t cu[kPromptReqs];             // its first token in the packed batch
};

// Requests [lo, lo + b.n) of the batch, cut into tiles of `rows` tokens.
void fill_prompt_batch(const cake_ctx* ctx, int lo, int rows, PromptBatch& b);

// The request of a tile (tile < b.tiles).
__device__ __forceinline__ int request_of(const PromptBatch& b, int tile) {
  int lo = 0, hi = b.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (b.first[mid] <= tile) lo = mid; else hi = mid;
  }
  return lo;
}

// Queries, or the output, of a prompt: element strides between heads and between tokens; channels are contiguous.
struct Strided {
  int64_t head, token;
};

// attend_tc.cu
bool prompt_tc_supported(const cake_ctx* ctx, Strided q);
int32_t launch_prompt_tc(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const void* v, void* out, Strided os,
                         float* lse, float* lse_window, cudaStream_t st);
int32_t launch_accumulate_tc(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const float* lse, float* out,
                             cudaStream_t st);
// attend_simt.cu
int32_t launch_prompt_simt(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const void* v, void* out, Strided os,
                           float* lse, float* lse_window, cudaStream_t st);
int32_t launch_accumulate_simt(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const float* lse, float* out,
                               cudaStream_t st);

}  // namespace cake
