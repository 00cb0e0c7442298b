// Attention over whole prompts in fp32 FMA: causal, grouped heads, packed requests of different lengths.
//
//   prompt_simt       O_i = sum_{j<=i} softmax_j(q_i.k_j / sqrt d) v_j and lse_i = log sum_{j<=i} exp(q_i.k_j / sqrt d): one
//                     pass over the keys with a running maximum, sum and output per row.
//   accumulate_simt   A_j = 1/G sum_h sum_{i>=j} exp(q_hi.k_j / sqrt d - lse_hi): a CTA keeps a tile of keys and goes over the
//                     queries behind them, so that no sum is shared between CTAs and the result does not depend on
//                     their order.
//
// They take fp32 inputs, whose products the tensor cores do not give in fp32 (and the few layouts that prompt_tc does not).
// Every CTA of 256 threads works on a tile of R x 64 logits; a thread owns R/16 rows x 4 columns of it, rows and columns 16
// apart, so that the 16-byte reads of the tiles in shared memory (rows padded by 16 bytes) meet no bank conflict.  Products
// are packed two to an instruction (even and odd channels), copies of the next tiles run behind them (cp.async).  R is
// 128 where that gives every SM a tile, else as much smaller as does: a thread's reads of shared memory per product grow as its
// rows shrink.
#include "cache_mma.cuh"
#include "tc_ptx.cuh"

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
// another request comes in.  fp32 rows are copied asynchronously (one group of copies; done with copy_wait).
template <typename T, int D, int N>
__device__ __forceinline__ void load_rows(float* dst, const T* src, int64_t stride, int row0, int valid) {
#pragma unroll 4
  for (int i = threadIdx.x; i < N * (D / 4); i += THREADS) {
    const int r = i / (D / 4), c = (i % (D / 4)) * 4;
    const bool in = row0 + r < valid;
    const T* from = src + (in ? (int64_t)(row0 + r) * stride + c : 0);
    if constexpr (sizeof(T) == 4) copy_async16n(smem_addr(dst + r * (D + 4) + c), from, in ? 16 : 0);
    else *reinterpret_cast<float4*>(dst + r * (D + 4) + c) = in ? Row4<T>::load(from) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  copy_commit();
}

// Logits of rows ty + 16 i and columns tx + 16 j of the tile.
template <int D, int RT>
__device__ __forceinline__ void logits(const float* q, const float* k, int ty, int tx, float (&s)[RT][4]) {
  f32x2 t[RT][4];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) t[i][j] = pack2(0.f, 0.f);
  const uint32_t qa = smem_addr(q + ty * (D + 4)), ka = smem_addr(k + tx * (D + 4));
#pragma unroll 4
  for (int c = 0; c < D; c += 4) {
    f32x2 kk[4][2];
#pragma unroll
    for (int j = 0; j < 4; ++j) ld_shared(kk[j], ka + (uint32_t)(16 * j * (D + 4) + c) * 4);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      f32x2 a[2];
      ld_shared(a, qa + (uint32_t)(16 * i * (D + 4) + c) * 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) t[i][j] = fma2(a[1], kk[j][1], fma2(a[0], kk[j][0], t[i][j]));
    }
  }
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x, y;
      unpack2(t[i][j], x, y);
      s[i][j] = x + y;
    }
}

// o += p_j v_j for a run of four keys.  kEdge: a value behind the row may be anything (an infinity times the weight 0 is not 0):
// it is left out.
template <int D, int RT, bool kEdge>
__device__ __forceinline__ void add_values(f32x2 (&o)[RT][D / 32], const float* p, const float* v, int ty, int tx, int j, int first_row) {
  float4 e[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) e[i] = *reinterpret_cast<const float4*>(p + (ty + 16 * i) * PP + j);
#pragma unroll
  for (int u = 0; u < 4; ++u) {
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      f32x2 x[2];
      ld_shared(x, smem_addr(v + (j + u) * (D + 4) + 64 * c + 4 * tx));
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const float w = u == 0 ? e[i].x : u == 1 ? e[i].y : u == 2 ? e[i].z : e[i].w;
        if (!kEdge || j + u <= first_row + ty + 16 * i) {
          o[i][2 * c] = fma2(pack2(w, w), x[0], o[i][2 * c]);
          o[i][2 * c + 1] = fma2(pack2(w, w), x[1], o[i][2 * c + 1]);
        }
      }
    }
  }
}

template <typename T, int D, int RT>
__global__ void __launch_bounds__(THREADS, 1) prompt_simt(const __grid_constant__ PromptBatch B, const SimtParams P) {
  constexpr int R = 16 * RT;                       // rows of the tile
  extern __shared__ float sm[];
  float *qsm = sm, *ksm = qsm + R * (D + 4), *vsm = ksm + 2 * KT * (D + 4), *psm = vsm + KT * (D + 4);
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
  load_rows<T, D, KT>(ksm, k, D, 0, N);
  float m[RT], l[RT];
  f32x2 o[RT][D / 32];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    m[i] = -CUDART_INF_F;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) o[i][c] = pack2(0.f, 0.f);
  }
  const int last = min(row0 + R, N);               // keys that some row sees
  for (int k0 = 0, at = 0; k0 < last; k0 += KT, at ^= 1) {
    // this tile's values and the next one's keys are on their way while this one's keys are multiplied
    load_rows<T, D, KT>(vsm, v, D, k0, N);
    load_rows<T, D, KT>(ksm + (at ^ 1) * KT * (D + 4), k, D, k0 + KT, k0 + KT < last ? N : 0);
    copy_wait<2>();
    __syncthreads();
    float s[RT][4];
    logits<D, RT>(qsm, ksm + at * KT * (D + 4), ty, tx, s);
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
      for (int c = 0; c < D / 32; ++c) o[i][c] = mul2(o[i][c], pack2(f, f));
    }
    copy_wait<1>();
    __syncthreads();
    if (edge) {
#pragma unroll 2
      for (int j = 0; j < KT; j += 4) add_values<D, RT, true>(o, psm, vsm, ty, tx, j, row0 - k0);
    } else {
#pragma unroll 2
      for (int j = 0; j < KT; j += 4) add_values<D, RT, false>(o, psm, vsm, ty, tx, j, 0);
    }
    __syncthreads();
  }
  copy_wait<0>();
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
    for (int c = 0; c < D / 64; ++c) {
      float x0, x1, x2, x3;
      unpack2(o[i][2 * c], x0, x1);
      unpack2(o[i][2 * c + 1], x2, x3);
      Row4<T>::store(dst + 64 * c + 4 * tx, make_float4(x0 * inv, x1 * inv, x2 * inv, x3 * inv));
    }
    if (tx == 0) {
      const float x = fmaf(m[i], P.scale, logf(total));
      if (P.lse) P.lse[h * P.T + cu + row] = x;
      const int w = row - (N - P.window);
      if (P.lse_window && w >= 0) P.lse_window[((int64_t)B.req[r] * P.Hq + h) * P.window + w] = x;
    }
  }
}

// A cluster of G CTAs, one per query head of the group, works for a tile of keys; the first adds up what the others found.
template <typename T, int D, int RT>
__global__ void __launch_bounds__(THREADS, 2) accumulate_simt(const __grid_constant__ PromptBatch B, const SimtParams P) {
  constexpr int R = 16 * RT;
  extern __shared__ float sm[];
  float *ksm = sm, *qsm = ksm + KT * (D + 4), *lsm = qsm + 2 * R * (D + 4);
  __shared__ float part[KT];
  const int G = P.Hq / P.Hkv, mine = blockIdx.x % G, pair = blockIdx.x / G;
  const int tile = pair / P.Hkv, g = pair % P.Hkv, h = g * G + mine;
  const int r = request_of(B, tile), N = B.len[r], key0 = (tile - B.first[r]) * KT;
  const int64_t cu = B.cu[r];
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const T* q = (const T*)P.q + h * P.qs.head + cu * P.qs.token;
  const float* lse = P.lse_in + h * P.T + cu;
  load_rows<T, D, KT>(ksm, (const T*)P.k + (g * P.T + cu) * D, D, key0, N);
  const int first = key0 / R * R;
  auto load_q = [&](int row0, int at) {
    load_rows<T, D, R>(qsm + at * R * (D + 4), q, P.qs.token, row0, row0 < N ? N : 0);
    for (int i = threadIdx.x; i < R; i += THREADS) lsm[at * R + i] = row0 + i < N ? lse[row0 + i] * kLog2E : 0.f;
  };
  load_q(first, 0);
  // Two-part sums: up to N / 16 weights of very different size come together here.
  float hi[4] = {0.f, 0.f, 0.f, 0.f}, lo[4] = {0.f, 0.f, 0.f, 0.f};
  for (int row0 = first, at = 0; row0 < N; row0 += R, at ^= 1) {
    load_q(row0 + R, at ^ 1);
    copy_wait<1>();
    __syncthreads();
    float s[RT][4];
    logits<D, RT>(qsm + at * R * (D + 4), ksm, ty, tx, s);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int key = key0 + tx + 16 * j;
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const int row = row0 + ty + 16 * i;
        const float e = exp2f(fmaf(s[i][j], P.scale2, -lsm[at * R + ty + 16 * i]));
        x += row >= key && row < N ? e : 0.f;
      }
      const float t = hi[j] + x;
      lo[j] += hi[j] >= x ? (hi[j] - t) + x : (x - t) + hi[j];
      hi[j] = t;
    }
    __syncthreads();
  }
  copy_wait<0>();
  __syncthreads();
  float* red = sm;                                 // [16][KT]
#pragma unroll
  for (int j = 0; j < 4; ++j) red[ty * KT + tx + 16 * j] = hi[j] + lo[j];
  __syncthreads();
  if ((int)threadIdx.x < KT) {
    float x = 0.f;
    for (int i = 0; i < 16; ++i) x += red[i * KT + threadIdx.x];
    part[threadIdx.x] = x;
  }
  cluster_sync();
  if (cluster_rank() == 0 && (int)threadIdx.x < KT && key0 + (int)threadIdx.x < N) {
    float x = part[threadIdx.x];
    for (int y = 1; y < G; ++y) x += __uint_as_float(ld_peer(&part[threadIdx.x], (uint32_t)y));
    P.acc_out[g * P.T + cu + key0 + threadIdx.x] = x * (1.f / (float)G);
  }
  cluster_sync();                                  // nobody leaves while its sums may still be read
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
cudaError_t run_prompt(const cake_ctx* ctx, int lo, PromptBatch& B, const SimtParams& P, cudaStream_t st) {
  constexpr size_t smem = sizeof(float) * ((16 * RT + 3 * KT) * (D + 4) + 16 * RT * PP);
  static_assert(smem <= 227 * 1024, "a CTA has 227 KB of shared memory");
  static PerDeviceOnce once;
  if (once.need(ctx->device)) {
    const cudaError_t e = cudaFuncSetAttribute(prompt_simt<T, D, RT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    once.mark(ctx->device);
  }
  fill_prompt_batch(ctx, lo, 16 * RT, B);
  prompt_simt<T, D, RT><<<(unsigned)(B.tiles * P.Hq), THREADS, smem, st>>>(B, P);
  count_launch();
  return cudaGetLastError();
}

template <typename T, int D, int RT>
cudaError_t run_accumulate(const cake_ctx* ctx, int lo, PromptBatch& B, const SimtParams& P, cudaStream_t st) {
  constexpr size_t smem = sizeof(float) * ((2 * 16 * RT + KT) * (D + 4) + 2 * 16 * RT);
  static PerDeviceOnce once;
  if (once.need(ctx->device)) {
    const cudaError_t e = cudaFuncSetAttribute(accumulate_simt<T, D, RT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    once.mark(ctx->device);
  }
  fill_prompt_batch(ctx, lo, KT, B);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(B.tiles * P.Hq), 1, 1);
  cfg.blockDim = dim3(THREADS, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)(P.Hq / P.Hkv);             // (at most 8: portable)
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, accumulate_simt<T, D, RT>, B, P);
  count_launch();
  return e;
}

// Row tiles of `rows` tokens in requests [lo, lo + kPromptReqs).
int64_t row_tiles(const cake_ctx* ctx, int lo, int rows) {
  int64_t n = 0;
  for (int r = lo; r < std::min(ctx->n_req, lo + kPromptReqs); ++r) n += (ctx->h_cu[r + 1] - ctx->h_cu[r] + rows - 1) / rows;
  return n;
}
template <typename T, int D>
cudaError_t run_prompts(const cake_ctx* ctx, const SimtParams& P, cudaStream_t st) {
  PromptBatch B;
  for (int lo = 0; lo < ctx->n_req; lo += B.n) {
    const int64_t sms = ctx->n_sm;
    const cudaError_t e = sizeof(T) == 2 || row_tiles(ctx, lo, 128) * P.Hq >= sms ? run_prompt<T, D, 8>(ctx, lo, B, P, st)
                          : row_tiles(ctx, lo, 64) * P.Hq >= sms                  ? run_prompt<T, D, sizeof(T) == 2 ? 8 : 4>(ctx, lo, B, P, st)
                          : row_tiles(ctx, lo, 32) * P.Hq >= sms                  ? run_prompt<T, D, sizeof(T) == 2 ? 8 : 2>(ctx, lo, B, P, st)
                                                                                  : run_prompt<T, D, sizeof(T) == 2 ? 8 : 1>(ctx, lo, B, P, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}
template <typename T, int D>
cudaError_t run_accumulates(const cake_ctx* ctx, const SimtParams& P, cudaStream_t st) {
  PromptBatch B;
  for (int lo = 0; lo < ctx->n_req; lo += B.n) {
    const cudaError_t e = run_accumulate<T, D, 4>(ctx, lo, B, P, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

int32_t launch_prompt_simt(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const void* v, void* out, Strided os,
                           float* lse, float* lse_window, cudaStream_t st) {
  SimtParams P = common(ctx);
  P.q = q; P.k = k; P.v = v; P.out = out; P.lse = lse; P.lse_window = lse_window; P.qs = qs; P.os = os;
  const bool f32 = ctx->cfg.dtype == CAKE_DTYPE_FP32, wide = ctx->cfg.head_dim == 128;
  return cuda_status(f32 ? (wide ? run_prompts<float, 128>(ctx, P, st) : run_prompts<float, 64>(ctx, P, st))
                         : (wide ? run_prompts<__nv_bfloat16, 128>(ctx, P, st) : run_prompts<__nv_bfloat16, 64>(ctx, P, st)));
}

int32_t launch_accumulate_simt(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const float* lse, float* out,
                               cudaStream_t st) {
  SimtParams P = common(ctx);
  P.q = q; P.k = k; P.lse_in = lse; P.acc_out = out; P.qs = qs;
  const bool f32 = ctx->cfg.dtype == CAKE_DTYPE_FP32, wide = ctx->cfg.head_dim == 128;
  return cuda_status(f32 ? (wide ? run_accumulates<float, 128>(ctx, P, st) : run_accumulates<float, 64>(ctx, P, st))
                         : (wide ? run_accumulates<__nv_bfloat16, 128>(ctx, P, st) : run_accumulates<__nv_bfloat16, 64>(ctx, P, st)));
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
  return (ctx->cfg.dtype == CAKE_DTYPE_FP32 ? launch_prompt_tc32 : launch_prompt_tc)(ctx, q, qs, k, v, out, os, lse, lse_window,
                                                                                (cudaStream_t)stream);
}

int32_t cake_accumulate_attention(cake_ctx* ctx, const void* q, int64_t q_head_stride, int64_t q_token_stride, const void* k,
                                  const float* lse, float* out, void* stream) {
  const int32_t ok = batch_ok(ctx);
  if (ok != CAKE_OK || ctx->n_req == 0) return ok;
  if (!q || !k || !lse || !out) return CAKE_ERR_ARG;
  if (!rows_ok(ctx, q, q_head_stride, q_token_stride) || !rows_ok(ctx, k, 0, 0)) return CAKE_ERR_ARG;
  const Strided qs = {q_head_stride, q_token_stride};
  return (ctx->cfg.dtype == CAKE_DTYPE_FP32 ? launch_accumulate_tc32 : launch_accumulate_tc)(ctx, q, qs, k, lse, out, (cudaStream_t)stream);
}

}  // extern "C"
