// What the attention kernels over prompts and caches share.
#pragma once

#include "cake_internal.cuh"

#include <math_constants.h>

namespace cake {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2E = 1.4426950408889634f;
// Reference of a row of which no logit above -inf has come yet: those are then weighed as 0 beside later ones, not as NaN.
constexpr float kNoWeight = -3.402823466e38f;

// Programmatic dependent launch.  A kernel may take its places while the one before it in the stream ends, and touches global
// memory only after after_previous(), which waits for all of that one's work; it lets the next one in only then, so that what
// has run before its own predecessor is complete for whoever starts early behind it.
__device__ __forceinline__ void after_previous() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
// Launches a kernel that way, as clusters of `cluster` CTAs.
template <typename Kernel, typename... Args>
cudaError_t launch_early(Kernel kernel, unsigned grid, int threads, size_t smem, int cluster, cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3((unsigned)threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)cluster;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;              // (a cluster of one costs a CTA's turn more than none)
  count_launch();
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

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

// Requests [lo, lo + b.n) of the batch, cut into tiles of `rows` tokens (attend_prompt.cu).
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

// A null pointer is aligned: whether it may be null is another check.
inline bool aligned(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// Cached rows of one layer and the queries of one token per request.  group: channels (and rows) that share a scale in 4 bits,
// 0 for rows of the context's type.
struct CacheParams {
  const void *q, *k, *v;             // v, k: packed rows, or their codes
  const float *k_scale, *k_zero, *v_scale, *v_zero;
  const int64_t *row_off, *group_off;
  const void *k_tail, *v_tail;
  const int32_t* tail_len;
  int64_t tail_cap;
  void* out;
  float* lse;
  int n_layers, layer, Hq, Hkv, group;
  float scale2;
};

// attend_rows.cu
int64_t rows_workspace(const cake_ctx* ctx);
int32_t launch_rows(const cake_ctx* ctx, int32_t n_req, const CacheParams& c, void* workspace, cudaStream_t st);
// attend_tc.cu
int32_t launch_prompt_tc(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const void* v, void* out, Strided os,
                         float* lse, float* lse_window, cudaStream_t st);
int32_t launch_accumulate_tc(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const float* lse, float* out,
                             cudaStream_t st);
// attend_tc32.cu
int32_t launch_prompt_tc32(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const void* v, void* out, Strided os,
                           float* lse, float* lse_window, cudaStream_t st);
int32_t launch_accumulate_tc32(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const float* lse, float* out,
                               cudaStream_t st);

}  // namespace cake
