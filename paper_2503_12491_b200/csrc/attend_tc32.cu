// Attention over whole prompts in fp32 on the sm_100a tensor cores.
//
//   prompt_tc32       O_i = sum_{j<=i} softmax_j(q_i.k_j / sqrt d) v_j and lse_i = log sum_{j<=i} exp(q_i.k_j / sqrt d).
//   accumulate_tc32   A_j = 1/G sum_h sum_{i>=j} exp(q_hi.k_j / sqrt d - lse_hi).
//
// An fp32 number is the exact sum of three bf16 ones (its 24 bits, eight at a time: split8), so a product of two fp32 operands
// is nine bf16 products, of which the six largest are taken, the smallest first:
//     x1 y3 + x3 y1 + x2 y2 + x1 y2 + x2 y1 + x1 y1 ,  summed in fp32 in tensor memory.
// Terms are cut, not rounded, so x2 is below 2^-7 of x and x3 below 2^-15, of its sign: x2 y3 and x3 y2, which are left out, are
// below 2^-22 of the product each and make it smaller.
// Six bf16 products are still five times as fast as one in fp32 FMA: 375 against 74 TFLOP/s of the device's nominal rates.
// (An infinity among what a row sees may make the row a NaN: its second and third terms are NaN.)
//
// The operand that a CTA keeps (128 queries, or keys of the accumulated attention) lies in tensor memory, three planes of d / 2
// columns, and so do the weights: with both operands in shared memory its bandwidth bounds tiles of this width (6 KB in the
// 32 cycles of a 128 x 64 x 16 product).  The others come through shared memory in the 128-byte swizzle; warps of their own
// read the fp32 rows ahead into registers, split them and write the planes while the tensor cores work on the tiles before.
// Tiles are 64 columns wide: three planes of more do not fit twice.
// Every wait is bounded; one that runs out raises CAKE_ERR_TIMEOUT and the CTA drains and exits.
#include "attend_tc.cuh"

#include <algorithm>

namespace cake {
namespace {

constexpr int STEP = 64;                         // columns of a tile of logits
constexpr int STEP_SLAB = STEP * 128;            // bytes of 64 channels of a plane of 64 rows

struct Tc32Params {
  const float *q, *k, *v;
  float *out, *lse, *lse_window;
  const float* lse_in;
  float* acc_out;
  Strided qs, os;
  int64_t T;
  int32_t* status;
  long long limit;
  int Hq, Hkv, G, window;
  float scale2;
};

// Eight channels: the upper eight bits of every number, the next eight, the rest.
__device__ __forceinline__ void split8(const float (&x)[8], uint4 (&p)[3]) {
  uint32_t w[3][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = x[2 * i], b = x[2 * i + 1];
    const float a1 = __uint_as_float(__float_as_uint(a) & 0xFFFF0000u), b1 = __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
    const float ra = a - a1, rb = b - b1;
    const float a2 = __uint_as_float(__float_as_uint(ra) & 0xFFFF0000u), b2 = __uint_as_float(__float_as_uint(rb) & 0xFFFF0000u);
    w[0][i] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
    w[1][i] = __byte_perm(__float_as_uint(ra), __float_as_uint(rb), 0x7632);
    w[2][i] = __byte_perm(__float_as_uint(ra - a2), __float_as_uint(rb - b2), 0x7632);
  }
#pragma unroll
  for (int e = 0; e < 3; ++e) p[e] = make_uint4(w[e][0], w[e][1], w[e][2], w[e][3]);
}
// Eight channels of a row, zeros where `in` is false (nothing is read then).
__device__ __forceinline__ void read8(float (&x)[8], const float* p, bool in) {
  const float4 a = in ? __ldg(reinterpret_cast<const float4*>(p)) : make_float4(0.f, 0.f, 0.f, 0.f);
  const float4 b = in ? __ldg(reinterpret_cast<const float4*>(p) + 1) : make_float4(0.f, 0.f, 0.f, 0.f);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
// Planes of piece c (eight channels) of a row, in tiles of ROWS rows.
template <int D, int ROWS>
__device__ __forceinline__ void put8(uint8_t* planes, int row, int c, const uint4 (&p)[3]) {
  uint8_t* at = planes + (c >> 3) * (ROWS * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4);
#pragma unroll
  for (int e = 0; e < 3; ++e) *reinterpret_cast<uint4*>(at + e * (ROWS * D * 2)) = p[e];
}
__device__ __forceinline__ void async_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A tile of STEP rows, read ahead by CONV threads: 16 to 64 numbers a thread.
template <int D, int CONV>
struct Ahead {
  static constexpr int PIECES = D / 8, N = STEP * PIECES / CONV;
  float x[N][8];
  __device__ __forceinline__ void read(const float* src, int64_t stride, int row0, int valid, int t) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = t + i * CONV, row = row0 + at / PIECES;
      read8(x[i], src + (int64_t)row * stride + (at % PIECES) * 8, row < valid);
    }
  }
  __device__ __forceinline__ void put(uint8_t* planes, int t) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint4 p[3];
      split8(x[i], p);
      put8<D, STEP>(planes, (t + i * CONV) / PIECES, (t + i * CONV) % PIECES, p);
    }
  }
};
// 64 numbers of this thread's lane as three planes of 32 columns, `apart` columns from one another.
__device__ __forceinline__ void put_planes(uint32_t (&w)[64], uint32_t at, uint32_t apart) {
#pragma unroll
  for (int e = 0; e < 3; ++e) {
    uint32_t p[32];
#pragma unroll
    for (int c = 0; c < 32; ++c) {
      p[c] = __byte_perm(w[2 * c], w[2 * c + 1], 0x7632);
      if (e < 2) {
        w[2 * c] = __float_as_uint(__uint_as_float(w[2 * c]) - __uint_as_float(w[2 * c] & 0xFFFF0000u));
        w[2 * c + 1] = __float_as_uint(__uint_as_float(w[2 * c + 1]) - __uint_as_float(w[2 * c + 1] & 0xFFFF0000u));
      }
    }
    tmem_st32(at + e * apart, p);
  }
}
// The row of this thread's lane (zeros if it is not there) as planes of D / 2 columns from `at` on.
template <int D>
__device__ __forceinline__ void put_row(const float* src, bool in, uint32_t at) {
#pragma unroll 1
  for (int c = 0; c < D; c += 64) {
    uint32_t w[64];
#pragma unroll
    for (int u = 0; u < 64; u += 4) {
      const float4 x = in ? __ldg(reinterpret_cast<const float4*>(src + c + u)) : make_float4(0.f, 0.f, 0.f, 0.f);
      w[u] = __float_as_uint(x.x); w[u + 1] = __float_as_uint(x.y); w[u + 2] = __float_as_uint(x.z); w[u + 3] = __float_as_uint(x.w);
    }
    put_planes(w, at + c / 2, D / 2);
  }
  tmem_wait_st();
}

// Planes of the six products.
__device__ constexpr int first_plane(int e) { return e == 1 ? 2 : e == 2 || e == 4 ? 1 : 0; }
__device__ constexpr int second_plane(int e) { return e == 0 ? 2 : e == 2 || e == 3 ? 1 : 0; }

// D[128][64] = A B^T over all channels: A in tensor memory, B planes of 64 rows in shared memory, K-major.
template <int D>
__device__ __forceinline__ void products(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc) {
#pragma unroll
  for (int e = 0; e < 6; ++e)
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      umma_ts(d, a + first_plane(e) * (uint32_t)(D / 2) + 8 * ks,
              b_lo + second_plane(e) * (uint32_t)(STEP * D * 2 >> 4) + (ks / 4) * (STEP_SLAB >> 4) + (ks % 4) * 2, idesc, (uint32_t)(e > 0 || ks > 0));
}

// ------------------------------------------------------------------ accumulated attention
constexpr int A_GROUPS = 2, A_CONV = A_GROUPS * 4, A_MMA = A_CONV + 4, A_LSE = A_MMA + 1, A_THREADS = 32 * (A_LSE + 1);
constexpr int A_BUFS = 4, A_STAGES = 4;          // tensor memory: four buffers of 64 logits, then the keys
constexpr uint32_t A_KEYS = A_BUFS * STEP;

template <int D> constexpr size_t acc32_smem() {
  return 1024 + (size_t)A_STAGES * STEP * D * 6 + (A_BUFS * STEP + A_GROUPS * TILE) * sizeof(float) + 256;
}

template <int D>
__global__ void __launch_bounds__(A_THREADS, 1) accumulate_tc32(const __grid_constant__ PromptBatch B, const Tc32Params P) {
  constexpr int Q_BYTES = STEP * D * 6;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* qs = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  float *nl = (float*)(qs + A_STAGES * Q_BYTES), *part = nl + A_BUFS * STEP;
  uint64_t *q_full = (uint64_t*)(part + A_GROUPS * TILE), *q_empty = q_full + A_STAGES, *acc_full = q_empty + A_STAGES,
           *acc_empty = acc_full + A_BUFS, *nl_full = acc_empty + A_BUFS, *k_full = nl_full + A_BUFS;
  uint32_t* s_tmem = (uint32_t*)(k_full + 1);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  // a cluster of G CTAs, one per query head of the group
  const int pair = blockIdx.x / P.G, tile = pair / P.Hkv, g = pair % P.Hkv, h = g * P.G + blockIdx.x % P.G;
  const int r = request_of(B, tile), N = B.len[r], key0 = (tile - B.first[r]) * TILE;      // the first keys have the most queries
  const int64_t cu = B.cu[r];
  const int n_tiles = (N - key0 + STEP - 1) / STEP;

  if (threadIdx.x == 0) {
    mbar_init(k_full, 4);
    for (int i = 0; i < A_STAGES; ++i) { mbar_init(&q_full[i], 4); mbar_init(&q_empty[i], 1); }
    for (int i = 0; i < A_BUFS; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], 4); mbar_init(&nl_full[i], 1); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == A_MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  after_previous();
  if (warp < 4) {
    const int key = key0 + warp * 32 + lane;
    put_row<D>(P.k + (g * P.T + cu + key) * D, key < N, tmem + ((uint32_t)(warp * 32) << 16) + A_KEYS);
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(k_full);
  }

  if (warp == A_MMA) {
    const uint32_t id = instr_desc(TILE, STEP), b = (smem_u32(qs) & 0x3FFFFu) >> 4;
    int last = -1;
    const bool ok = mbar_wait(k_full, 0, P.status, P.limit);
    for (int t = 0; ok && t < n_tiles; ++t) {
      const int s = t % A_STAGES, buf = t % A_BUFS;
      if (!mbar_wait(&acc_empty[buf], ((uint32_t)(t / A_BUFS) & 1u) ^ 1u, P.status, P.limit) ||
          !mbar_wait(&q_full[s], (uint32_t)(t / A_STAGES) & 1u, P.status, P.limit)) break;
      tc_fence_after();
      products<D>(tmem + STEP * buf, tmem + A_KEYS, b + (uint32_t)(s * Q_BYTES >> 4), id);
      umma_commit(&q_empty[s]);
      umma_commit(&acc_full[buf]);
      last = t;
    }
    // what was issued ends before tensor and shared memory are given back
    if (last >= 0) mbar_drain(&acc_full[last % A_BUFS], (uint32_t)(last / A_BUFS) & 1u, P.status);
  } else if (warp == A_LSE) {
    // -lse * log2(e) of the queries of every tile, three tiles ahead in registers
    constexpr int AHEAD = 3;
    float x[AHEAD][2];
    auto get = [&](int t, float (&v)[2]) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int i = key0 + t * STEP + 32 * e + lane;
        v[e] = i < N ? -P.lse_in[h * P.T + cu + i] * kLog2E : 0.f;
      }
    };
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) get(u, x[u]);
    bool ok = true;
    for (int t0 = 0; t0 < n_tiles && ok; t0 += AHEAD) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int t = t0 + u, buf = t % A_BUFS;
        if (t >= n_tiles || !ok) break;
        ok = mbar_wait(&acc_empty[buf], ((uint32_t)(t / A_BUFS) & 1u) ^ 1u, P.status, P.limit);
        if (!ok) break;
#pragma unroll
        for (int e = 0; e < 2; ++e) nl[buf * STEP + 32 * e + lane] = x[u][e];
        __syncwarp();
        if (lane == 0) mbar_arrive(&nl_full[buf]);
        get(t + AHEAD, x[u]);
      }
    }
  } else if (warp >= A_CONV) {
    const int t128 = threadIdx.x - A_CONV * 32;
    Ahead<D, 128> x;
    const float* q = P.q + h * P.qs.head + cu * P.qs.token;
    x.read(q, P.qs.token, key0, N, t128);
    for (int t = 0; t < n_tiles; ++t) {
      const int s = t % A_STAGES;
      if (!mbar_wait(&q_empty[s], ((uint32_t)(t / A_STAGES) & 1u) ^ 1u, P.status, P.limit)) break;
      x.put(qs + s * Q_BYTES, t128);
      async_proxy_fence();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_full[s]);
      if (t + 1 < n_tiles) x.read(q, P.qs.token, key0 + (t + 1) * STEP, N, t128);
    }
  } else {
    const int grp = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const f32x2 sc = splat(P.scale2);
    float hi = 0.f, lo = 0.f;
    for (int t = grp; t < n_tiles; t += A_GROUPS) {
      const int buf = t % A_BUFS, off = t * STEP, past = N - key0 - off;
      const uint32_t ph = (uint32_t)(t / A_BUFS) & 1u;
      if (!mbar_wait(&nl_full[buf], ph, P.status, P.limit) || !mbar_wait(&acc_full[buf], ph, P.status, P.limit)) break;
      tc_fence_after();
      const uint32_t at = tmem + lanes + STEP * buf;
      const float* n = nl + buf * STEP;
      f32x2 acc0 = splat(0.f), acc1 = splat(0.f);
      uint32_t a[32], b[32];
      tmem_ld32(at, a);
      tmem_wait_ld32(a);
      tmem_ld32(at + 32, b);
      if (off < TILE || past < STEP) {
        weigh32<true, false>(a, n, sc, row - off, past, acc0, acc1);
        tmem_wait_ld32(b);
        weigh32<true, false>(b, n + 32, sc, row - off - 32, past - 32, acc0, acc1);
      } else {
        weigh32<false, false>(a, n, sc, 0, 0, acc0, acc1);
        tmem_wait_ld32(b);
        weigh32<false, false>(b, n + 32, sc, 0, 0, acc0, acc1);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&acc_empty[buf]);
      float x0, x1, x2, x3;
      unpack2(acc0, x0, x1);
      unpack2(acc1, x2, x3);
      const float x = (x0 + x1) + (x2 + x3), y = hi + x;
      lo += hi >= x ? (hi - y) + x : (x - y) + hi;
      hi = y;
    }
    part[grp * TILE + row] = hi + lo;
  }
  tc_fence_before();
  __syncthreads();
  if (warp == A_MMA) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  } else if (threadIdx.x < TILE) {
    part[threadIdx.x] += part[TILE + threadIdx.x];
  }
  cluster_sync();
  if (cluster_rank() == 0 && threadIdx.x < TILE && key0 + (int)threadIdx.x < N) {
    float x = part[threadIdx.x];
    for (int y = 1; y < P.G; ++y) x += __uint_as_float(ld_peer(&part[threadIdx.x], (uint32_t)y));
    P.acc_out[g * P.T + cu + key0 + threadIdx.x] = x * (1.f / (float)P.G);
  }
  cluster_sync();                                // nobody leaves while its sums may still be read
}

// ------------------------------------------------------------------ prompt
// One tile of 128 rows of one query head.  Two buffers of logits: while the softmax of a tile runs, the tensor cores multiply
// the next tile's, then the weights of this one with its values.
//   tensor memory: two buffers of 96 columns (64 logits, over which the three planes of weights are written), O of one tile, the
//   queries.
// Sums in tensor memory are truncated, not rounded: half a step off per addition on average, and always downwards.  Over the
// tiles of a prompt that adds up (2.2e-6 relative at 512 keys), so the products of a tile of keys are added to the outputs so far
// in registers: a thread of the eight warps that split K and V has half of a row's channels.
//   Warps: 0-3 softmax, 4-11 K and V into planes and the outputs, 12 MMAs and tensor-memory allocation.
constexpr int P_CONV = 4, P_MMA = 12, P_THREADS = 32 * (P_MMA + 1), P_FACTORS = 4;
constexpr uint32_t P_BUF = 96, P_OUT = 192, P_QUERIES = P_OUT + 128;

template <int D> constexpr size_t prompt32_smem() { return 1024 + (size_t)4 * STEP * D * 6 + (P_FACTORS + 1) * TILE * sizeof(float) + 256; }

template <int D>
__global__ void __launch_bounds__(P_THREADS, 1) prompt_tc32(const __grid_constant__ PromptBatch B, const Tc32Params P) {
  constexpr int S_BYTES = STEP * D * 6;          // two stages each of K and V
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ks = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* vs = ks + 2 * S_BYTES;
  float* factors = (float*)(vs + 2 * S_BYTES);   // [P_FACTORS][128] what a row's outputs so far are multiplied with at a tile
  float* sums = factors + P_FACTORS * TILE;      // [128]
  uint64_t *k_full = (uint64_t*)(sums + TILE), *k_empty = k_full + 2, *v_full = k_full + 4, *v_empty = k_full + 6, *s_full = k_full + 8,
           *p_full = k_full + 10, *o_full = k_full + 12, *o_empty = k_full + 13, *q_full = k_full + 14;
  uint32_t* s_tmem = (uint32_t*)(k_full + 15);
  int* s_dirty = (int*)(k_full + 16);
  int* s_failed = s_dirty + 1;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int tile = blockIdx.x / P.Hq, h = blockIdx.x % P.Hq, g = h / P.G;
  const int r = request_of(B, tile), N = B.len[r];
  const int row0 = (B.first[r + 1] - 1 - tile) * TILE;               // the last rows have the most keys: they come first
  const int64_t cu = B.cu[r];
  const int n = (min(row0 + TILE, N) + STEP - 1) / STEP;             // key tiles
  const int row = (warp & 3) * 32 + lane, i = row0 + row;            // of a softmax or output thread: in the tile, in the request
  const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;

  if (threadIdx.x == 0) {
    mbar_init(o_full, 1); mbar_init(o_empty, 8); mbar_init(q_full, 4);
    for (int x = 0; x < 2; ++x) {
      mbar_init(&k_full[x], 8); mbar_init(&k_empty[x], 1); mbar_init(&v_full[x], 8); mbar_init(&v_empty[x], 1);
      mbar_init(&s_full[x], 1); mbar_init(&p_full[x], 4);
    }
    *s_dirty = *s_failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == P_MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  after_previous();
  constexpr int DH = D / 2;                      // channels of an output thread
  float o[DH];                                   // (warps 4 to 11)
#pragma unroll
  for (int c = 0; c < DH; ++c) o[c] = 0.f;

  if (warp == P_MMA) {
    const uint32_t id_s = instr_desc(TILE, STEP), id_o = instr_desc(TILE, D) | (1u << 16);     // values: N along the row
    const uint32_t k_lo = (smem_u32(ks) & 0x3FFFFu) >> 4;
    const uint32_t v_lo = ((smem_u32(vs) & 0x3FFFFu) >> 4) | ((uint32_t)(STEP_SLAB >> 4) << 16);
    bool ok = mbar_wait(q_full, 0, P.status, P.limit);
    auto qk = [&](int j) {
      if (!mbar_wait(&k_full[j & 1], (uint32_t)(j >> 1) & 1u, P.status, P.limit)) return false;
      tc_fence_after();
      products<D>(tmem + P_BUF * (j & 1), tmem + P_QUERIES, k_lo + (uint32_t)((j & 1) * S_BYTES >> 4), id_s);
      umma_commit(&k_empty[j & 1]);
      umma_commit(&s_full[j & 1]);
      return true;
    };
    if (ok) ok = qk(0);
    int done = 0;
    for (int j = 0; ok && j < n; ++j) {
      // (the next logits take the buffer of the tile before, whose weights the products issued before read)
      if (j + 1 < n) ok = qk(j + 1);
      if (ok) ok = mbar_wait(&v_full[j & 1], (uint32_t)(j >> 1) & 1u, P.status, P.limit);
      if (ok) ok = mbar_wait(&p_full[j & 1], (uint32_t)(j >> 1) & 1u, P.status, P.limit);
      if (ok) ok = mbar_wait(o_empty, ((uint32_t)j & 1u) ^ 1u, P.status, P.limit);
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (int e = 0; e < 6; ++e) {
        const uint32_t a = tmem + P_BUF * (j & 1) + 32u * first_plane(e);
        const uint32_t b = v_lo + (uint32_t)((j & 1) * S_BYTES >> 4) + second_plane(e) * (uint32_t)(S_BYTES / 3 >> 4);
#pragma unroll
        for (int kstep = 0; kstep < STEP / 16; ++kstep)
          umma_ts(tmem + P_OUT, a + 8 * kstep, b + (uint32_t)(kstep * 2048 >> 4), id_o, (uint32_t)(e > 0 || kstep > 0));
      }
      umma_commit(&v_empty[j & 1]);
      umma_commit(o_full);
      done = j + 1;
    }
    // what was issued ends before tensor and shared memory are given back, whether the others have waited for it or not
    // (one phase after the other: a parity does not tell a phase from the next but one)
    if (done > 0) mbar_drain(o_full, (uint32_t)(done - 1) & 1u, P.status);
    if (!ok) {
      umma_commit(o_full);
      mbar_drain(o_full, (uint32_t)done & 1u, P.status);
    }
  } else if (warp >= P_CONV) {
    const int t256 = threadIdx.x - P_CONV * 32, c0 = ((warp - P_CONV) >> 2) * DH;
    const float *k = P.k + (g * P.T + cu) * D, *v = P.v + (g * P.T + cu) * D;
    Ahead<D, 256> x;                             // the next tile: K of 0, then K of j + 1 and V of j in turn
    auto put = [&](uint8_t* planes, uint64_t* full, uint64_t* empty, int j) {
      if (!mbar_wait(&empty[j & 1], ((uint32_t)(j >> 1) & 1u) ^ 1u, P.status, P.limit)) return false;
      x.put(planes + (j & 1) * S_BYTES, t256);
      async_proxy_fence();
      __syncwarp();
      if (lane == 0) mbar_arrive(&full[j & 1]);
      return true;
    };
    // tile j's products to the outputs, which move to its reference
    auto add = [&](int j) {
      if (!mbar_wait(o_full, (uint32_t)j & 1u, P.status, P.limit)) return false;
      tc_fence_after();
      const float f = factors[(j % P_FACTORS) * TILE + row];
#pragma unroll
      for (int c = 0; c < DH; c += 16) {
        uint32_t w[16];
        tmem_ld16_issue(tmem + lanes + P_OUT + c0 + c, w);
        tmem_ld_wait(w);
#pragma unroll
        for (int u = 0; u < 16; ++u) o[c + u] = fmaf(o[c + u], f, __uint_as_float(w[u]));
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(o_empty);
      return true;
    };
    x.read(k, D, 0, N, t256);
    bool ok = put(ks, k_full, k_empty, 0);
    if (n > 1) x.read(k, D, STEP, N, t256);
    for (int j = 0; j < n && ok; ++j) {
      if (j + 1 < n) ok = put(ks, k_full, k_empty, j + 1);
      if (!ok) break;
      x.read(v, D, j * STEP, N, t256);
      if (j > 0) ok = add(j - 1);                // (the values are on their way)
      if (!ok) break;
      if ((j + 1) * STEP > row0) {
        // A value that some row of the tile must not see is multiplied by a weight of zero, which only helps if it is finite:
        // those that are not are added at the end, to the rows that do see them.
        bool found = false;
#pragma unroll
        for (int y = 0; y < Ahead<D, 256>::N; ++y)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!isfinite(x.x[y][e])) { x.x[y][e] = 0.f; found = true; }
        if (found) *s_dirty = 1;
      }
      ok = put(vs, v_full, v_empty, j);
      if (j + 2 < n) x.read(k, D, (j + 2) * STEP, N, t256);
    }
    if (ok) ok = add(n - 1);
    if (!ok) *s_failed = 1;
  } else {
    float ref = 0.f, sum = 0.f;
    bool ok = true;
    put_row<D>(P.q + h * P.qs.head + (cu + i) * P.qs.token, i < N, tmem + lanes + P_QUERIES);
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(q_full);
    for (int j = 0; j < n; ++j) {
      ok = mbar_wait(&s_full[j & 1], (uint32_t)(j >> 1) & 1u, P.status, P.limit);
      if (!ok) break;
      tc_fence_after();
      const uint32_t t_s = tmem + lanes + P_BUF * (j & 1);
      uint32_t w[64];
      tmem_ld32(t_s, w);
      tmem_ld32(t_s + 32, w + 32);
      tmem_wait_ld32(w);
      pin32(w + 32);
      float* s = reinterpret_cast<float*>(w);
      const int seen = i - j * STEP;             // keys of the tile up to this one are visible
      if ((j + 1) * STEP > row0 + 1) {
#pragma unroll
        for (int c = 0; c < 64; ++c) s[c] = c > seen ? -CUDART_INF_F : s[c];
      }
      float m0 = s[0], m1 = s[1];
#pragma unroll
      for (int c = 2; c < 64; c += 2) { m0 = fmaxf(m0, s[c]); m1 = fmaxf(m1, s[c + 1]); }
      const float top = fmaxf(m0, m1) * P.scale2;
      // The reference follows a maximum that is more than 2^kRefSlack above it.  (A factor is read before the logits of three
      // tiles on are issued, so that a ring of four is enough.)
      const float to = j == 0 ? fmaxf(top, kNoWeight) : top > ref + kRefSlack ? top : ref, f = j == 0 || to == ref ? 1.f : ex2(ref - to);
      ref = to;
      factors[(j % P_FACTORS) * TILE + row] = f;
      const float cf = coarse_factor(ref), sc = P.scale2 * cf, mr = -ref * cf;
      // weights, their sum, and their three planes
      float part[4] = {};
#pragma unroll
      for (int c = 0; c < 64; ++c) {
        s[c] = ex2(fmaf(s[c], sc, mr));
        part[c & 3] += s[c];
      }
      sum = fmaf(sum, f, (part[0] + part[1]) + (part[2] + part[3]));
      put_planes(w, t_s, 32);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_full[j & 1]);
    }
    if (!ok) *s_failed = 1;
    sums[row] = sum;
    if (ok && i < N) {
      const float l = (ref + log2f(sum)) * kLn2;
      if (P.lse) P.lse[h * P.T + cu + i] = l;
      const int x = i - (N - P.window);
      if (P.lse_window && x >= 0) P.lse_window[((int64_t)B.req[r] * P.Hq + h) * P.window + x] = l;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == P_MMA) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  } else if (warp >= P_CONV && i < N && !*s_failed) {
    const int c0 = ((warp - P_CONV) >> 2) * DH;
    const float inv = 1.f / sums[row];
    float* dst = P.out + h * P.os.head + (cu + i) * P.os.token + c0;
#pragma unroll
    for (int c = 0; c < DH; ++c) o[c] *= inv;
    if (*s_dirty) {
      const float* vals = P.v + (g * P.T + cu) * D + c0;
      for (int j = row0; j <= i; ++j)
#pragma unroll
        for (int c = 0; c < DH; ++c) {
          const float y = vals[(int64_t)j * D + c];
          if (!isfinite(y)) o[c] += y;
        }
    }
#pragma unroll
    for (int c = 0; c < DH; c += 4) *reinterpret_cast<float4*>(dst + c) = make_float4(o[c], o[c + 1], o[c + 2], o[c + 3]);
  }
}

// ------------------------------------------------------------------ host
Tc32Params common(const cake_ctx* ctx) {
  const cake_config& c = ctx->cfg;
  Tc32Params P = {};
  P.T = ctx->total_tokens; P.status = ctx->d_status;
  P.limit = ctx->wait_limit_cycles > 0 ? ctx->wait_limit_cycles : kSpinLimit;
  P.Hq = c.n_q_heads; P.Hkv = c.n_kv_heads; P.G = c.n_q_heads / c.n_kv_heads; P.window = c.window;
  P.scale2 = kLog2E / sqrtf((float)c.head_dim);
  return P;
}
template <int D, bool kPrompt>
int32_t run32(const cake_ctx* ctx, const Tc32Params& P, cudaStream_t st) {
  constexpr size_t smem = kPrompt ? prompt32_smem<D>() : acc32_smem<D>();
  static_assert(smem <= 227 * 1024, "a CTA has 227 KB of shared memory");
  const auto kernel = kPrompt ? prompt_tc32<D> : accumulate_tc32<D>;
  static PerDeviceOnce once;
  if (once.need(ctx->device)) {
    CAKE_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    once.mark(ctx->device);
  }
  PromptBatch B;
  for (int lo = 0; lo < ctx->n_req; lo += B.n) {
    fill_prompt_batch(ctx, lo, TILE, B);
    CAKE_CUDA_TRY(launch_early(kernel, (unsigned)(B.tiles * P.Hq), kPrompt ? P_THREADS : A_THREADS, smem, kPrompt ? 1 : P.G, st, B, P));
  }
  return CAKE_OK;
}

}  // namespace

int32_t launch_prompt_tc32(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const void* v, void* out, Strided os,
                           float* lse, float* lse_window, cudaStream_t st) {
  Tc32Params P = common(ctx);
  P.q = (const float*)q; P.k = (const float*)k; P.v = (const float*)v; P.out = (float*)out; P.lse = lse; P.lse_window = lse_window;
  P.qs = qs; P.os = os;
  return ctx->cfg.head_dim == 128 ? run32<128, true>(ctx, P, st) : run32<64, true>(ctx, P, st);
}

int32_t launch_accumulate_tc32(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const float* lse, float* out,
                               cudaStream_t st) {
  Tc32Params P = common(ctx);
  P.q = (const float*)q; P.k = (const float*)k; P.lse_in = lse; P.acc_out = out; P.qs = qs;
  return ctx->cfg.head_dim == 128 ? run32<128, false>(ctx, P, st) : run32<64, false>(ctx, P, st);
}

}  // namespace cake
