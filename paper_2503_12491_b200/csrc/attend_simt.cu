// Attention over whole prompts in fp32 FMA: causal, grouped heads, packed requests of different lengths.
//
//   prompt_simt       O_i = sum_{j<=i} softmax_j(q_i.k_j / sqrt d) v_j and lse_i = log sum_{j<=i} exp(q_i.k_j / sqrt d): one
//                     pass over the keys with a running maximum, sum and output per row.
//   accumulate_simt   A_j = 1/G sum_h sum_{i>=j} exp(q_hi.k_j / sqrt d - lse_hi): a CTA keeps a tile of keys and goes over the
//                     queries behind them, so that no sum is shared between CTAs and the result does not depend on
//                     their order.
//
// They take fp32 inputs, whose products the tensor cores do not give in fp32.  Every CTA of 256 threads works on a tile
// of R x 64 logits; a thread owns R/16 rows x 4 columns of it, rows and columns 16 apart, so that the 16-byte reads of
// the tiles in shared memory (rows padded by 16 bytes) meet no bank conflict.
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

namespace {

constexpr int KT = 64;               // keys of a tile
constexpr int THREADS = 256;
constexpr int PP = KT + 4;           // floats of a row of probabilities in shared memory

struct SimtParams {
  const void *q, *k, *v;
  void* out;
  float *lse, *lse_window;
  const float* lse_in;
  float* acc_out;
  Strided qs, os;
  int64_t T;
  int Hq, Hkv, window;
  float scale2, scale;               // log2(e) / sqrt(d), 1 / sqrt(d)
};

template <typename T> struct Row4;
template <> struct Row4<float> {
  static __device__ __forceinline__ float4 load(const float* p) { return *reinterpret_cast<const float4*>(p); }
  static __device__ __forceinline__ void store(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
};
template <> struct Row4<__nv_bfloat16> {
  static __device__ __forceinline__ float4 load(const __nv_bfloat16* p) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                       __uint_as_float(w.y & 0xFFFF0000u));
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, float4 v) {
    *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(v.x, v.y);
    *reinterpret_cast<__nv_bfloat162*>(p + 2) = __floats2bfloat162_rn(v.z, v.w);
  }
};

// Rows [row0, row0 + N) of a strided matrix into shared memory; rows from `valid` on read as zero, so that nothing of
// another request comes in.
template <typename T, int D, int N>
__device__ __forceinline__ void load_rows(float* dst, const T* src, int64_t stride, int row0, int valid) {
  for (int i = threadIdx.x; i < N * (D / 4); i += THREADS) {
    const int r = i / (D / 4), c = (i % (D / 4)) * 4;
    const float4 x = row0 + r < valid ? Row4<T>::load(src + (int64_t)(row0 + r) * stride + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    *reinterpret_cast<float4*>(dst + r * (D + 4) + c) = x;
  }
}

// Logits of rows ty + 16 i and columns tx + 16 j of the tile.
template <int D, int RT>
__device__ __forceinline__ void logits(const float* q, const float* k, int ty, int tx, float (&s)[RT][4]) {
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
  for (int c = 0; c < D; c += 4) {
    float4 kk[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) kk[j] = *reinterpret_cast<const float4*>(k + (tx + 16 * j) * (D + 4) + c);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const float4 a = *reinterpret_cast<const float4*>(q + (ty + 16 * i) * (D + 4) + c);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        s[i][j] = fmaf(a.x, kk[j].x, fmaf(a.y, kk[j].y, fmaf(a.z, kk[j].z, fmaf(a.w, kk[j].w, s[i][j]))));
    }
  }
}

template <typename T, int D, int RT>
__global__ void __launch_bounds__(THREADS, 1) prompt_simt(const __grid_constant__ PromptBatch B, const SimtParams P) {
  constexpr int R = 16 * RT, DC = D / 64;          // rows of the tile; 16-byte column groups of the output per thread
  extern __shared__ float sm[];
  float *qsm = sm, *ksm = qsm + R * (D + 4), *vsm = ksm + KT * (D + 4), *psm = vsm + KT * (D + 4);
  const int tile = blockIdx.x / P.Hq, h = blockIdx.x % P.Hq, g = h / (P.Hq / P.Hkv);
  const int r = request_of(B, tile), N = B.len[r];
  // the last rows have the most keys: they come first
  const int row0 = (B.first[r + 1] - 1 - tile) * R;
  const int64_t cu = B.cu[r];
  const T* q = (const T*)P.q + h * P.qs.head + cu * P.qs.token;
  const T* k = (const T*)P.k + (g * P.T + cu) * D;
  const T* v = (const T*)P.v + (g * P.T + cu) * D;
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  load_rows<T, D, R>(qsm, q, P.qs.token, row0, N);
  float m[RT], l[RT], o[RT][4 * DC];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    m[i] = -CUDART_INF_F;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < 4 * DC; ++c) o[i][c] = 0.f;
  }
  const int last = min(row0 + R, N);               // keys that some row sees
  for (int k0 = 0; k0 < last; k0 += KT) {
    __syncthreads();
    load_rows<T, D, KT>(ksm, k, D, k0, N);
    load_rows<T, D, KT>(vsm, v, D, k0, N);
    __syncthreads();
    float s[RT][4];
    logits<D, RT>(qsm, ksm, ty, tx, s);
    const bool edge = k0 + KT > row0 + 1 || k0 + KT > N;    // some key of the tile is behind some row, or beyond the prompt
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int row = row0 + ty + 16 * i;
      float top = m[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = k0 + tx + 16 * j;
        if (edge && (key > row || key >= N)) s[i][j] = -CUDART_INF_F;
        top = fmaxf(top, s[i][j]);
      }
#pragma unroll
      for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      // (a row of the padding may have seen nothing yet: its reference stays finite)
      const float ref = top == -CUDART_INF_F ? 0.f : top, f = exp2f((m[i] - ref) * P.scale2);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = exp2f((s[i][j] - ref) * P.scale2);
        sum += e;
        psm[(ty + 16 * i) * PP + tx + 16 * j] = e;
      }
      l[i] = fmaf(l[i], f, sum);                   // of this thread's columns
      m[i] = top;
#pragma unroll
      for (int c = 0; c < 4 * DC; ++c) o[i][c] *= f;
    }
    __syncwarp();                                  // a row's probabilities are written and read by one half-warp
#pragma unroll 2
    for (int j = 0; j < KT; j += 4) {
      float4 p[RT];
#pragma unroll
      for (int i = 0; i < RT; ++i) p[i] = *reinterpret_cast<const float4*>(psm + (ty + 16 * i) * PP + j);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
#pragma unroll
        for (int c = 0; c < DC; ++c) {
          const float4 x = *reinterpret_cast<const float4*>(vsm + (j + u) * (D + 4) + 64 * c + 4 * tx);
#pragma unroll
          for (int i = 0; i < RT; ++i) {
            const float e = u == 0 ? p[i].x : u == 1 ? p[i].y : u == 2 ? p[i].z : p[i].w;
            // a value behind the row may be anything (an infinity times the weight 0 is not 0): it is left out
            if (!edge || k0 + j + u <= row0 + ty + 16 * i) {
              o[i][4 * c] = fmaf(e, x.x, o[i][4 * c]);
              o[i][4 * c + 1] = fmaf(e, x.y, o[i][4 * c + 1]);
              o[i][4 * c + 2] = fmaf(e, x.z, o[i][4 * c + 2]);
              o[i][4 * c + 3] = fmaf(e, x.w, o[i][4 * c + 3]);
            }
          }
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int row = row0 + ty + 16 * i;
    float total = l[i];
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) total += __shfl_xor_sync(0xffffffffu, total, x);
    if (row >= N) continue;
    const float inv = 1.f / total;
    T* dst = (T*)P.out + h * P.os.head + (cu + row) * P.os.token;
#pragma unroll
    for (int c = 0; c < DC; ++c)
      Row4<T>::store(dst + 64 * c + 4 * tx,
                     make_float4(o[i][4 * c] * inv, o[i][4 * c + 1] * inv, o[i][4 * c + 2] * inv, o[i][4 * c + 3] * inv));
    if (tx == 0) {
      const float x = fmaf(m[i], P.scale, logf(total));
      if (P.lse) P.lse[h * P.T + cu + row] = x;
      const int w = row - (N - P.window);
      if (P.lse_window && w >= 0) P.lse_window[((int64_t)B.req[r] * P.Hq + h) * P.window + w] = x;
    }
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(THREADS, 1) accumulate_simt(const __grid_constant__ PromptBatch B, const SimtParams P) {
  constexpr int RT = 8, R = 16 * RT;
  extern __shared__ float sm[];
  float *ksm = sm, *qsm = ksm + KT * (D + 4), *lsm = qsm + R * (D + 4);
  const int tile = blockIdx.x / P.Hkv, g = blockIdx.x % P.Hkv, G = P.Hq / P.Hkv;
  const int r = request_of(B, tile), N = B.len[r], key0 = (tile - B.first[r]) * KT;
  const int64_t cu = B.cu[r];
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  load_rows<T, D, KT>(ksm, (const T*)P.k + (g * P.T + cu) * D, D, key0, N);
  // Two-part sums: up to G * N / 16 weights of very different size come together here.
  float hi[4] = {0.f, 0.f, 0.f, 0.f}, lo[4] = {0.f, 0.f, 0.f, 0.f};
  for (int h = g * G; h < (g + 1) * G; ++h) {
    const T* q = (const T*)P.q + h * P.qs.head + cu * P.qs.token;
    for (int row0 = key0 / R * R; row0 < N; row0 += R) {
      __syncthreads();
      load_rows<T, D, R>(qsm, q, P.qs.token, row0, N);
      for (int i = threadIdx.x; i < R; i += THREADS)
        lsm[i] = row0 + i < N ? P.lse_in[h * P.T + cu + row0 + i] * kLog2E : 0.f;
      __syncthreads();
      float s[RT][4];
      logits<D, RT>(qsm, ksm, ty, tx, s);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = key0 + tx + 16 * j;
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          const int row = row0 + ty + 16 * i;
          const float e = exp2f(fmaf(s[i][j], P.scale2, -lsm[ty + 16 * i]));
          x += row >= key && row < N ? e : 0.f;
        }
        const float t = hi[j] + x;
        lo[j] += hi[j] >= x ? (hi[j] - t) + x : (x - t) + hi[j];
        hi[j] = t;
      }
    }
  }
  __syncthreads();
  float* red = sm;                                 // [16][KT]
#pragma unroll
  for (int j = 0; j < 4; ++j) red[ty * KT + tx + 16 * j] = hi[j] + lo[j];
  __syncthreads();
  if ((int)threadIdx.x < KT && key0 + (int)threadIdx.x < N) {
    float x = 0.f;
    for (int i = 0; i < 16; ++i) x += red[i * KT + threadIdx.x];
    P.acc_out[g * P.T + cu + key0 + threadIdx.x] = x * (1.f / (float)G);
  }
}

SimtParams common(const cake_ctx* ctx) {
  const cake_config& c = ctx->cfg;
  SimtParams P = {};
  P.T = ctx->total_tokens;
  P.Hq = c.n_q_heads; P.Hkv = c.n_kv_heads; P.window = c.window;
  P.scale = 1.f / sqrtf((float)c.head_dim);
  P.scale2 = kLog2E / sqrtf((float)c.head_dim);
  return P;
}

template <typename T, int D, int RT>
cudaError_t run_prompt(const cake_ctx* ctx, const PromptBatch& B, const SimtParams& P, cudaStream_t st) {
  constexpr size_t smem = sizeof(float) * ((16 * RT + 2 * KT) * (D + 4) + 16 * RT * PP);
  static PerDeviceOnce once;
  if (once.need(ctx->device)) {
    const cudaError_t e = cudaFuncSetAttribute(prompt_simt<T, D, RT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    once.mark(ctx->device);
  }
  prompt_simt<T, D, RT><<<(unsigned)(B.tiles * P.Hq), THREADS, smem, st>>>(B, P);
  count_launch();
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t run_accumulate(const cake_ctx* ctx, const PromptBatch& B, const SimtParams& P, cudaStream_t st) {
  constexpr size_t smem = sizeof(float) * ((128 + KT) * (D + 4) + 128);
  static PerDeviceOnce once;
  if (once.need(ctx->device)) {
    const cudaError_t e = cudaFuncSetAttribute(accumulate_simt<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    once.mark(ctx->device);
  }
  accumulate_simt<T, D><<<(unsigned)(B.tiles * P.Hkv), THREADS, smem, st>>>(B, P);
  count_launch();
  return cudaGetLastError();
}

}  // namespace

int32_t launch_prompt_simt(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const void* v, void* out, Strided os,
                           float* lse, float* lse_window, cudaStream_t st) {
  SimtParams P = common(ctx);
  P.q = q; P.k = k; P.v = v; P.out = out; P.lse = lse; P.lse_window = lse_window; P.qs = qs; P.os = os;
  const bool f32 = ctx->cfg.dtype == CAKE_DTYPE_FP32, wide = ctx->cfg.head_dim == 128;
  PromptBatch B;
  for (int lo = 0; lo < ctx->n_req; lo += B.n) {
    fill_prompt_batch(ctx, lo, 128, B);
    CAKE_CUDA_TRY(f32 ? (wide ? run_prompt<float, 128, 8>(ctx, B, P, st) : run_prompt<float, 64, 8>(ctx, B, P, st))
                      : (wide ? run_prompt<__nv_bfloat16, 128, 8>(ctx, B, P, st) : run_prompt<__nv_bfloat16, 64, 8>(ctx, B, P, st)));
  }
  return CAKE_OK;
}

int32_t launch_accumulate_simt(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const float* lse, float* out,
                               cudaStream_t st) {
  SimtParams P = common(ctx);
  P.q = q; P.k = k; P.lse_in = lse; P.acc_out = out; P.qs = qs;
  const bool f32 = ctx->cfg.dtype == CAKE_DTYPE_FP32, wide = ctx->cfg.head_dim == 128;
  PromptBatch B;
  for (int lo = 0; lo < ctx->n_req; lo += B.n) {
    fill_prompt_batch(ctx, lo, KT, B);
    CAKE_CUDA_TRY(f32 ? (wide ? run_accumulate<float, 128>(ctx, B, P, st) : run_accumulate<float, 64>(ctx, B, P, st))
                      : (wide ? run_accumulate<__nv_bfloat16, 128>(ctx, B, P, st) : run_accumulate<__nv_bfloat16, 64>(ctx, B, P, st)));
  }
  return CAKE_OK;
}

}  // namespace cake

using namespace cake;

extern "C" {

// (bounds under which no product of a stride and a number of heads or tokens overflows)
static constexpr int64_t kMaxHeadStride = (int64_t)1 << 38, kMaxTokenStride = (int64_t)1 << 31;
// Rows that the kernels read and write in 16-byte pieces.
static bool rows_ok(const cake_ctx* ctx, const void* p, int64_t head, int64_t token) {
  const int64_t es = ctx->cfg.dtype == CAKE_DTYPE_FP32 ? 4 : 2;
  return ((uintptr_t)p & 15) == 0 && head >= 0 && token >= 0 && head < kMaxHeadStride && token < kMaxTokenStride &&
         head * es % 16 == 0 && token * es % 16 == 0;
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
  if (!rows_ok(ctx, q, q_head_stride, q_token_stride) || !rows_ok(ctx, k, 0, 0) || !rows_ok(ctx, v, 0, 0) ||
      !rows_ok(ctx, out, out_head_stride, out_token_stride)) return CAKE_ERR_ARG;
  // rows of the output that share memory would be written twice
  const int64_t heads = ctx->cfg.n_q_heads, tokens = ctx->total_tokens;
  const bool by_token = out_head_stride >= d && out_token_stride >= d && out_token_stride - d >= (heads - 1) * out_head_stride;
  const bool by_head = out_token_stride >= d && out_head_stride >= d && out_head_stride - d >= (tokens - 1) * out_token_stride;
  if (!by_token && !(heads == 1 && out_token_stride >= d) && !by_head) return CAKE_ERR_ARG;
  const Strided qs = {q_head_stride, q_token_stride}, os = {out_head_stride, out_token_stride};
  return (prompt_tc_supported(ctx, qs) ? launch_prompt_tc : launch_prompt_simt)(ctx, q, qs, k, v, out, os, lse, lse_window,
                                                                                (cudaStream_t)stream);
}

int32_t cake_accumulate_attention(cake_ctx* ctx, const void* q, int64_t q_head_stride, int64_t q_token_stride, const void* k,
                                  const float* lse, float* out, void* stream) {
  const int32_t ok = batch_ok(ctx);
  if (ok != CAKE_OK || ctx->n_req == 0) return ok;
  if (!q || !k || !lse || !out) return CAKE_ERR_ARG;
  if (!rows_ok(ctx, q, q_head_stride, q_token_stride) || !rows_ok(ctx, k, 0, 0)) return CAKE_ERR_ARG;
  const Strided qs = {q_head_stride, q_token_stride};
  return (prompt_tc_supported(ctx, qs) ? launch_accumulate_tc : launch_accumulate_simt)(ctx, q, qs, k, lse, out, (cudaStream_t)stream);
}

}  // extern "C"
