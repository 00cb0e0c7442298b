// Attention over whole prompts on the sm_100a tensor cores: bf16 inputs, causal, grouped heads, packed requests.
//
//   prompt_tc       O_i = sum_{j<=i} softmax_j(q_i.k_j / sqrt d) v_j and lse_i = log sum_{j<=i} exp(q_i.k_j / sqrt d).
//   accumulate_tc   A_j = 1/G sum_h sum_{i>=j} exp(q_hi.k_j / sqrt d - lse_hi): see there.
//
// prompt_tc.  A CTA works for 256 consecutive rows of one query head, as two tiles A and B of 128 rows, and goes over its key tiles of 128
// keys once, in ascending order:
//     S = Q K^T  (tcgen05, accumulator in tensor memory)  ->  P = 2^(s - ref), in bf16, back into tensor memory over S
//     O += P V   (tcgen05, P read from tensor memory, V as it lies in HBM: keys x channels)
// A thread of a softmax group owns one row: its logits come with tcgen05.ld, so a row's maximum and sum need no other
// thread.  While group A works on its logits, the tensor cores multiply for group B and the other way round.
//
// Reference.  P is taken against a reference that follows the row's running maximum only when that is more than 2^8 above
// it (the output would have to be rescaled in tensor memory for every new maximum): sums are exact in the reference, which
// cancels in O / sum and is added back in the log-sum-exp.
//
// Bound.  A tile pair is 2 x 128 x 128 logits: 2 x 2 products of 512 cycles at d = 128 on the tensor cores, and 32 768
// exponentials, 2048 cycles of the special-function unit; a share of the exponentials is computed by a polynomial on the
// FMA pipe (exp2_poly), so that the tensor cores set the pace.  Long prompts reach the board's power limit first: one of 32768
// tokens, 32 heads on 8, takes 7.7 ms, 1.15 PFLOP/s at 1.5 to 1.65 GHz; four of 4096, 32 heads, 150 us.
//
// Rounding.  P is rounded to bf16 as the operand of a bf16 product; its sum is taken before the rounding, in fp32; logits,
// sums and outputs are fp32.
//
// Warps: 0-3 softmax of tile A, 4-7 of tile B, 8 TMA loads, 9 MMAs and tensor-memory allocation, 10-11 look through the value
// tiles on the diagonal: a value that some row of the tile must not see is multiplied by a weight of zero, which only helps
// if it is finite, so those that are not are zeroed here and added to the rows that do see them at the end.
// Every wait is bounded; one that runs out raises CAKE_ERR_TIMEOUT and the CTA drains and exits.
#include "attend_tc.cuh"

#include <algorithm>

namespace cake {
namespace {

constexpr int P_THREADS = 384;
constexpr int W_TMA = 8, W_MMA = 9, W_SCAN = 10;

template <int D> struct PromptCfg {
  static constexpr int SLABS = D / 64;
  static constexpr int TILE_BYTES = SLABS * SLAB;
  static constexpr int STAGES = D == 128 ? 4 : 6;                    // K and V tiles in flight
  static constexpr size_t SMEM = 1024 + (size_t)(2 + STAGES) * TILE_BYTES + 256;
  static constexpr uint32_t O_COL = 256;                             // tensor memory: S/P of A, of B, O of A, of B
};
static_assert(PromptCfg<128>::SMEM <= 227 * 1024 && PromptCfg<64>::SMEM <= 227 * 1024, "a CTA has 227 KB of shared memory");

struct PromptParams {
  const __nv_bfloat16* v;                        // for the rows of the fix-up alone
  __nv_bfloat16* out;
  float *lse, *lse_window;
  Strided os;
  int64_t T;
  int32_t* status;
  long long limit;
  int Hq, G, window;
  int q_head_step;                               // 0 where all heads are the same rows in memory
  float scale2;
};

// ------------------------------------------------------------------ prompt
struct PromptSmem {
  uint8_t *q, *kv;
  uint64_t *q_full, *kv_full, *kv_empty, *s_full, *p_full, *o_full, *vd_full, *v_clean, *drained;
  uint32_t* tmem;
  int* dirty;                                    // [2] a value tile on the diagonal of A, of B had values that are not finite
};

template <int D>
__device__ __forceinline__ PromptSmem carve(uint8_t* base) {
  using C = PromptCfg<D>;
  PromptSmem s;
  uint8_t* p = (uint8_t*)(((uintptr_t)base + 1023) & ~(uintptr_t)1023);
  s.q = p;                      p += 2 * C::TILE_BYTES;
  s.kv = p;                     p += C::STAGES * C::TILE_BYTES;
  s.q_full = (uint64_t*)p;      p += 8;
  s.kv_full = (uint64_t*)p;     p += 8 * C::STAGES;
  s.kv_empty = (uint64_t*)p;    p += 8 * C::STAGES;
  s.s_full = (uint64_t*)p;      p += 16;
  s.p_full = (uint64_t*)p;      p += 32;         // [tile][half]
  s.o_full = (uint64_t*)p;      p += 16;
  s.vd_full = (uint64_t*)p;     p += 16;
  s.v_clean = (uint64_t*)p;     p += 16;
  s.drained = (uint64_t*)p;     p += 8;
  s.tmem = (uint32_t*)p;        p += 8;
  s.dirty = (int*)p;
  return s;
}

// A row's weights against its reference, into tensor memory over the logits.
template <bool kDiag>
__device__ __forceinline__ void weigh_row(const float* s, uint32_t t_s, float scale2, float ref, float& sum, uint64_t* p_full) {
  const f32x2 sc = splat(scale2), mr = splat(-ref);
  f32x2 acc0 = splat(0.f), acc1 = splat(0.f);
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    uint32_t p[32];
#pragma unroll
    for (int c = 0; c < 64; c += 8) {
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const f32x2 x = fma2(pack2(s[64 * half + c + i], s[64 * half + c + i + 1]), sc, mr);
        if (!kDiag && i == 6 && c % 16 == 0) {   // an eighth of the exponentials on the FMA pipe
          exp2_poly(x, e[i], e[i + 1]);
        } else {
          float a, b;
          unpack2(x, a, b);
          e[i] = ex2(a);
          e[i + 1] = ex2(b);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const __nv_bfloat162 w = __floats2bfloat162_rn(e[i], e[i + 1]);
        p[(c + i) / 2] = *reinterpret_cast<const uint32_t*>(&w);
      }
      acc0 = add2(acc0, pack2(e[0], e[1]));
      acc1 = add2(acc1, pack2(e[2], e[3]));
      acc0 = add2(acc0, pack2(e[4], e[5]));
      acc1 = add2(acc1, pack2(e[6], e[7]));
    }
    tmem_st32(t_s + 32 * half, p);
    tmem_wait_st();
    tc_fence_before();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(&p_full[half]);
  }
  float a, b, c, d;
  unpack2(acc0, a, b);
  unpack2(acc1, c, d);
  sum += (a + b) + (c + d);
}

// One row's tile of logits: reference, exponentials, P into tensor memory.  kDiag: keys behind the row are masked.
template <int D, bool kDiag>
__device__ __forceinline__ void softmax_tile(uint32_t t_s, uint32_t t_o, bool first, int row, float scale2, float& ref, float& sum,
                                             uint64_t* p_full) {
  uint32_t r[128];
#pragma unroll
  for (int c = 0; c < 4; ++c) tmem_ld32(t_s + 32 * c, r + 32 * c);
  tmem_wait_ld32(r);
  pin32(r + 32); pin32(r + 64); pin32(r + 96);
  float* s = reinterpret_cast<float*>(r);
  if constexpr (kDiag) {
#pragma unroll
    for (int c = 0; c < 128; ++c) s[c] = c > row ? -CUDART_INF_F : s[c];
  }
  float m0 = s[0], m1 = s[1], m2 = s[2], m3 = s[3];
#pragma unroll
  for (int c = 4; c < 128; c += 8) {
    m0 = max3(m0, s[c], s[c + 1]);
    m1 = max3(m1, s[c + 2], s[c + 3]);
    if (c + 4 < 128) {
      m2 = max3(m2, s[c + 4], s[c + 5]);
      m3 = max3(m3, s[c + 6], s[c + 7]);
    }
  }
  const float top = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)) * scale2;
  if (first) {
    ref = fmaxf(top, kNoWeight);
  } else if (__any_sync(0xffffffffu, top > ref + kRefSlack)) {
    // Some row's maximum left its reference behind: the warp's outputs move to the new ones.  (The products of the tile
    // before are done: this tile's logits were committed after them.)
    const float to = top > ref + kRefSlack ? top : ref, f = to == ref ? 1.f : ex2(ref - to);
    sum *= f;
    ref = to;
    uint32_t o[32];
#pragma unroll 1
    for (int c = 0; c < D; c += 32) {
      tmem_ld32(t_o + c, o);
      tmem_wait_ld32(o);
#pragma unroll
      for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
      tmem_st32(t_o + c, o);
    }
  }
  // (a copy of its own, so that the usual one keeps the scale in a register of the whole warp: with one for both long prompts were 2 %
  // slower)
  const float cf = coarse_factor(ref);
  if (__any_sync(0xffffffffu, cf != 1.f)) weigh_row<kDiag>(s, t_s, scale2 * cf, ref * cf, sum, p_full);
  else weigh_row<kDiag>(s, t_s, scale2, ref, sum, p_full);
}

template <int D>
__global__ void __launch_bounds__(P_THREADS, 1)
prompt_tc(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
          const __grid_constant__ CUtensorMap v_map, const __grid_constant__ PromptBatch B, const PromptParams P) {
  using C = PromptCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  const PromptSmem S = carve<D>(smem_raw);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int tile = blockIdx.x / P.Hq, h = blockIdx.x % P.Hq, g = h / P.G;
  const int r = request_of(B, tile), N = B.len[r];
  const int row0 = (B.first[r + 1] - 1 - tile) * 2 * TILE;           // the last rows have the most keys: they come first
  const int64_t cu = B.cu[r];
  const int n_a = row0 / TILE + 1, n_b = row0 + TILE < N ? n_a + 1 : 0, n_kv = max(n_a, n_b);   // key tiles of A, of B

  if (threadIdx.x == 0) {
    mbar_init(S.q_full, 1);
    for (int i = 0; i < C::STAGES; ++i) { mbar_init(&S.kv_full[i], 1); mbar_init(&S.kv_empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&S.s_full[i], 1); mbar_init(&S.o_full[i], 1); mbar_init(&S.vd_full[i], 1); mbar_init(&S.v_clean[i], 2); S.dirty[i] = 0; }
    for (int i = 0; i < 4; ++i) mbar_init(&S.p_full[i], 4);
    mbar_init(S.drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == W_MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(S.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *S.tmem;
  after_previous();
  // Item i of the ring: K of tile 0, then V of tile j and K of tile j + 1 in turn.
  const int n_items = 2 * n_kv;
  auto stage_of = [](int i) { return i % C::STAGES; };
  auto phase_of = [](int i) { return (uint32_t)(i / C::STAGES) & 1u; };
  auto k_item = [](int j) { return j == 0 ? 0 : 2 * j; };
  auto v_item = [](int j) { return 2 * j + 1; };
  // The value tiles on the diagonals of A and B, the last ones, arrive at barriers of their own, where the scan waits.  (Their
  // stages are not used again: at most two items come behind them.)
  static_assert(C::STAGES > 2, "");
  auto diag_of = [&](int i) { return (i & 1) == 0 ? -1 : i == v_item(n_a - 1) ? 0 : i == v_item(n_b - 1) ? 1 : -1; };
  auto full_of = [&](int i) { return diag_of(i) < 0 ? &S.kv_full[stage_of(i)] : &S.vd_full[diag_of(i)]; };

  if (warp == W_TMA) {
    mbar_expect_tx(S.q_full, (uint32_t)((n_b ? 2 : 1) * C::TILE_BYTES));
    for (int t = 0; t < (n_b ? 2 : 1); ++t)
      for (int sl = 0; sl < C::SLABS; ++sl)
        tma_load_4d(S.q + t * C::TILE_BYTES + sl * SLAB, &q_map, S.q_full, 64 * sl,
                    (int)(cu + row0) + t * TILE, h * P.q_head_step, 0);
    bool ok = true;
    int issued = 0;
    for (int i = 0; i < n_items; ++i) {
      ok = mbar_wait(&S.kv_empty[stage_of(i)], phase_of(i) ^ 1u, P.status, P.limit);
      if (!ok) break;
      const bool is_v = i & 1;
      const int j = i >> 1;
      mbar_expect_tx(full_of(i), C::TILE_BYTES);
      tma_load_3d(S.kv + stage_of(i) * C::TILE_BYTES, is_v ? &v_map : &k_map, full_of(i), 0, (int)(g * P.T + cu) + j * TILE, 0);
      issued = i + 1;
    }
    // do not leave the CTA while a copy may still be writing its shared memory
    mbar_drain(S.q_full, 0, P.status);
    for (int i = max(0, issued - C::STAGES); i < issued; ++i)
      mbar_drain(full_of(i), diag_of(i) < 0 ? phase_of(i) : 0u, P.status);
  } else if (warp == W_MMA) {
    const uint32_t id_s = instr_desc(TILE, TILE), id_o = instr_desc(TILE, D) | (1u << 16);   // B of the second: N along the row
    const uint32_t q_lo = (smem_u32(S.q) & 0x3FFFFu) >> 4, kv_lo = (smem_u32(S.kv) & 0x3FFFFu) >> 4;
    bool ok = mbar_wait(S.q_full, 0, P.status, P.limit);
    auto qk = [&](int t, int j) {                // S_t = Q_t K_j^T
      const uint32_t a = q_lo + (uint32_t)(t * C::TILE_BYTES >> 4), b = kv_lo + (uint32_t)(stage_of(k_item(j)) * C::TILE_BYTES >> 4);
      const uint32_t d = tmem + 128u * t;
      umma_ss<0>(d, a, b, id_s);
      umma_ss<1>(d, a + 2, b + 2, id_s);
      umma_ss<1>(d, a + 4, b + 4, id_s);
      umma_ss<1>(d, a + 6, b + 6, id_s);
      if constexpr (D == 128) {
        constexpr uint32_t o = SLAB >> 4;
        umma_ss<1>(d, a + o, b + o, id_s);
        umma_ss<1>(d, a + o + 2, b + o + 2, id_s);
        umma_ss<1>(d, a + o + 4, b + o + 4, id_s);
        umma_ss<1>(d, a + o + 6, b + o + 6, id_s);
      }
      umma_commit(&S.s_full[t]);
    };
    auto pv = [&](int t, int j) {                // O_t += P_t V_j, half of the keys as soon as its weights are there
      const uint32_t b = (kv_lo + (uint32_t)(stage_of(v_item(j)) * C::TILE_BYTES >> 4)) | ((uint32_t)(SLAB >> 4) << 16);
      const uint32_t d = tmem + C::O_COL + (uint32_t)(D * t), a = tmem + 128u * t;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (!mbar_wait(&S.p_full[2 * t + half], (uint32_t)j & 1u, P.status, P.limit)) return false;
        tc_fence_after();
#pragma unroll
        for (int ks = 4 * half; ks < 4 * half + 4; ++ks)
          umma_ts(d, a + 8 * ks, b + (uint32_t)(ks * 2048 >> 4), id_o, (uint32_t)(j > 0 || ks > 0));
      }
      return true;
    };
    if (ok) ok = mbar_wait(&S.kv_full[0], 0, P.status, P.limit);
    if (ok) {
      tc_fence_after();
      qk(0, 0);
      if (n_b) qk(1, 0);
      umma_commit(&S.kv_empty[0]);
    }
    for (int j = 0; ok && j < n_kv; ++j) {
      const int vi = v_item(j), ki = k_item(j + 1);
      const int diag = diag_of(vi);
      ok = mbar_wait(diag >= 0 ? &S.v_clean[diag] : &S.kv_full[stage_of(vi)], diag >= 0 ? 0u : phase_of(vi), P.status, P.limit);
      if (!ok) break;
      if (j < n_a) {
        ok = pv(0, j);
        if (!ok) break;
        if (j == n_a - 1) umma_commit(&S.o_full[0]);
      }
      if (j + 1 < n_kv) {
        ok = mbar_wait(&S.kv_full[stage_of(ki)], phase_of(ki), P.status, P.limit);
        if (!ok) break;
        tc_fence_after();
        if (j + 1 < n_a) qk(0, j + 1);
      }
      if (j < n_b) {
        ok = pv(1, j);
        if (!ok) break;
        if (j == n_b - 1) umma_commit(&S.o_full[1]);
      }
      umma_commit(&S.kv_empty[stage_of(vi)]);
      if (j + 1 < n_kv) {
        if (j + 1 < n_b) qk(1, j + 1);
        umma_commit(&S.kv_empty[stage_of(ki)]);
      }
    }
    // what was issued ends before tensor and shared memory are given back, whether the others have waited for it or not
    umma_commit(S.drained);
    mbar_drain(S.drained, 0, P.status);
  } else if (warp >= W_SCAN) {
    // the value tiles on the diagonals: j = n_a - 1 and n_b - 1
    for (int t = 0; t < (n_b ? 2 : 1); ++t) {
      const int vi = v_item(t ? n_b - 1 : n_a - 1);
      if (!mbar_wait(&S.vd_full[t], 0, P.status, P.limit)) break;
      uint4* x = reinterpret_cast<uint4*>(S.kv + stage_of(vi) * C::TILE_BYTES);
      bool found = false;
#pragma unroll 4
      for (int i = threadIdx.x - W_SCAN * 32; i < C::TILE_BYTES / 16; i += 64) {
        uint4 v = x[i];
        uint32_t* w = reinterpret_cast<uint32_t*>(&v);
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) bad |= (w[e] & 0x7F80u) == 0x7F80u || (w[e] & 0x7F800000u) == 0x7F800000u;
        if (bad) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if ((w[e] & 0x7F80u) == 0x7F80u) w[e] &= 0xFFFF0000u;
            if ((w[e] & 0x7F800000u) == 0x7F800000u) w[e] &= 0x0000FFFFu;
          }
          x[i] = v;
          found = true;
        }
      }
      if (found) S.dirty[t] = 1;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&S.v_clean[t]);
    }
  } else {
    const int t = warp >> 2, n = t ? n_b : n_a, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lanes + 128u * t, t_o = tmem + lanes + C::O_COL + (uint32_t)(D * t);
    float ref = 0.f, sum = 0.f;
    bool ok = true;
    for (int j = 0; j < n - 1 && ok; ++j) {
      ok = mbar_wait(&S.s_full[t], (uint32_t)j & 1u, P.status, P.limit);
      if (!ok) break;
      tc_fence_after();
      softmax_tile<D, false>(t_s, t_o, j == 0, row, P.scale2, ref, sum, S.p_full + 2 * t);
    }
    if (ok && n) {
      ok = mbar_wait(&S.s_full[t], (uint32_t)(n - 1) & 1u, P.status, P.limit);
      if (ok) {
        tc_fence_after();
        softmax_tile<D, true>(t_s, t_o, n == 1, row, P.scale2, ref, sum, S.p_full + 2 * t);
        ok = mbar_wait(&S.o_full[t], 0, P.status, P.limit);
      }
    }
    if (ok && n) {
      tc_fence_after();
      const int i = row0 + t * TILE + row;       // the row in its request
      // (logits of -inf alone: a sum of zero, no output and an lse of -inf; with a NaN among them the sum is one, and so is the lse)
      const float inv = sum == 0.f ? CUDART_NAN_F : 1.f / sum;
      const bool live = i < N;
      __nv_bfloat16* dst = P.out + h * P.os.head + (cu + i) * P.os.token;
      const __nv_bfloat16* vals = P.v + (g * P.T + cu) * D;
      const int dirty = S.dirty[0] | (t ? S.dirty[1] << 1 : 0);      // (a row of A sees nothing of B's diagonal tile)
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        uint32_t o[32];
        tmem_ld32(t_o + c, o);
        tmem_wait_ld32(o);
        float x[32];
#pragma unroll
        for (int u = 0; u < 32; ++u) x[u] = __uint_as_float(o[u]) * inv;
        if (dirty && live) {
          // values that are not finite and that this row sees: they decide its output, whatever their weight
          for (int j = (n_a - 1) * TILE; j <= i; ++j)
#pragma unroll
            for (int u = 0; u < 32; ++u) {
              const float w = __bfloat162float(vals[(int64_t)j * D + c + u]);
              if (!isfinite(w)) x[u] += w;
            }
        }
        if (live) {
#pragma unroll
          for (int u = 0; u < 32; u += 8) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const __nv_bfloat162 y = __floats2bfloat162_rn(x[u + 2 * e], x[u + 2 * e + 1]);
              w[e] = *reinterpret_cast<const uint32_t*>(&y);
            }
            *reinterpret_cast<uint4*>(dst + c + u) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
      if (live) {
        const float l = (ref + log2f(sum)) * kLn2;
        if (P.lse) P.lse[h * P.T + cu + i] = l;
        const int w = i - (N - P.window);
        if (P.lse_window && w >= 0) P.lse_window[((int64_t)B.req[r] * P.Hq + h) * P.window + w] = l;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == W_MMA) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// ------------------------------------------------------------------ accumulated attention
// A CTA keeps a tile of 128 keys of one KV head and goes over the query tiles of the group's heads from its own tokens on:
//     D[key][query] = K Q^T  (tcgen05)  ->  sum over the queries of 2^(d * scale - lse)
// A thread owns a key, so that its sum never leaves its registers; three groups of four warps take the query tiles in turn and
// are added up at the end in a fixed order.  The queries' log-sum-exps of a tile come through shared memory, where all
// threads of a warp read the same four at a time.  Where there are fewer tiles of keys than SMs, the heads of a group go to CTAs of
// their own, a cluster, whose first adds up the others' sums; with more the CTAs' beginnings and ends cost more than it gains.  Without
// and with, in us: 32 heads on 8, 1000 tokens (63 tiles) 23.7 and 16.4, 2000 (126) 43.5 and 42.1, 2500 (157) 53.4 and 57.9, 4096 (256)
// 95.7 and 119.9, 16384 1354 and 1586; 16 heads on 2, 1000 tokens (16) 43.9 and 12.2, 8192 (128) 305 and 215, 12000 (188) 458 and 447,
// 16384 (256) 711 and 785; four ragged requests, 32 on 8, 5000 tokens in all, 77 and 120.
//
// Bound.  128 x 128 logits are 512 cycles of the tensor cores and 1024 of the special-function unit: a share of the
// exponentials is computed on the FMA pipe (exp2_poly), until both units are busy.
//
// Sums.  A tile's 128 terms are added in fp32, the tiles' sums with their rounding errors kept (two-part sums).
constexpr int A_GROUPS = 3, A_THREADS = A_GROUPS * 128 + 128, A_BUFS = 4, A_STAGES = 4;
constexpr int A_TMA = A_GROUPS * 4, A_MMA = A_TMA + 1, A_LSE = A_TMA + 2;

template <int D> constexpr size_t acc_smem() {
  return 1024 + (size_t)(1 + A_STAGES) * (D / 64) * SLAB + A_BUFS * 128 * sizeof(float) + A_GROUPS * 128 * sizeof(float) + 256;
}
struct AccSmem {
  uint8_t *k, *q;
  float *nl, *part;                              // [A_BUFS][128] -lse * log2(e) of a tile's queries; [A_GROUPS][128] sums
  uint64_t *k_full, *q_full, *q_empty, *acc_full, *acc_empty, *nl_full;
  uint32_t* tmem;
};
template <int D>
__device__ __forceinline__ AccSmem carve_acc(uint8_t* base) {
  AccSmem s;
  constexpr int TB = (D / 64) * SLAB;
  uint8_t* p = (uint8_t*)(((uintptr_t)base + 1023) & ~(uintptr_t)1023);
  s.k = p;                      p += TB;
  s.q = p;                      p += A_STAGES * TB;
  s.nl = (float*)p;             p += A_BUFS * 128 * sizeof(float);
  s.part = (float*)p;           p += A_GROUPS * 128 * sizeof(float);
  s.k_full = (uint64_t*)p;      p += 8;
  s.q_full = (uint64_t*)p;      p += 8 * A_STAGES;
  s.q_empty = (uint64_t*)p;     p += 8 * A_STAGES;
  s.acc_full = (uint64_t*)p;    p += 8 * A_BUFS;
  s.acc_empty = (uint64_t*)p;   p += 8 * A_BUFS;
  s.nl_full = (uint64_t*)p;     p += 8 * A_BUFS;
  s.tmem = (uint32_t*)p;
  return s;
}

struct AccParams {
  const float* lse;
  float* out;
  int64_t T;
  int32_t* status;
  long long limit;
  int Hq, Hkv, G;
  int q_head_step;
  float scale2;
};

template <bool kEdge>
__device__ __forceinline__ float weigh_tile(uint32_t taddr, const float* nl, float scale2, int first, int past) {
  const f32x2 sc = splat(scale2);
  f32x2 acc0 = splat(0.f), acc1 = splat(0.f);
  uint32_t a[32], b[32];
  tmem_ld32(taddr, a);
  tmem_wait_ld32(a);
  tmem_ld32(taddr + 32, b);                      // the next columns are on their way during the arithmetic
  weigh32<kEdge, true>(a, nl, sc, first, past, acc0, acc1);
  tmem_wait_ld32(b);
  tmem_ld32(taddr + 64, a);
  weigh32<kEdge, true>(b, nl + 32, sc, first - 32, past - 32, acc0, acc1);
  tmem_wait_ld32(a);
  tmem_ld32(taddr + 96, b);
  weigh32<kEdge, true>(a, nl + 64, sc, first - 64, past - 64, acc0, acc1);
  tmem_wait_ld32(b);
  weigh32<kEdge, true>(b, nl + 96, sc, first - 96, past - 96, acc0, acc1);
  float x0, x1, x2, x3;
  unpack2(acc0, x0, x1);
  unpack2(acc1, x2, x3);
  return (x0 + x1) + (x2 + x3);
}

// kSplit: a cluster of G CTAs, one per query head of the group.
template <int D, bool kSplit>
__global__ void __launch_bounds__(A_THREADS, 1)
accumulate_tc(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ PromptBatch B,
              const AccParams P) {
  constexpr int SLABS = D / 64, TB = SLABS * SLAB;
  extern __shared__ uint8_t smem_raw[];
  const AccSmem S = carve_acc<D>(smem_raw);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int share = kSplit ? blockIdx.x % P.G : 0, pair = kSplit ? blockIdx.x / P.G : blockIdx.x;
  const int tile = pair / P.Hkv, g = pair % P.Hkv, h0 = g * P.G + share, heads = kSplit ? 1 : P.G;      // this CTA's query heads
  const int r = request_of(B, tile), N = B.len[r], key0 = (tile - B.first[r]) * TILE;      // the first keys have the most queries
  const int64_t cu = B.cu[r];
  const int per_head = (N - key0 + TILE - 1) / TILE, n_tiles = per_head * heads;    // query tiles: head by head

  if (threadIdx.x == 0) {
    mbar_init(S.k_full, 1);
    for (int i = 0; i < A_STAGES; ++i) { mbar_init(&S.q_full[i], 1); mbar_init(&S.q_empty[i], 1); }
    for (int i = 0; i < A_BUFS; ++i) { mbar_init(&S.acc_full[i], 1); mbar_init(&S.acc_empty[i], 4); mbar_init(&S.nl_full[i], 1); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == A_MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(S.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *S.tmem;
  after_previous();

  if (warp == A_TMA) {
    mbar_expect_tx(S.k_full, TB);
    tma_load_3d(S.k, &k_map, S.k_full, 0, (int)(g * P.T + cu) + key0, 0);
    bool ok = true;
    int issued = 0, h = h0, q0 = key0;
    for (int t = 0; t < n_tiles; ++t) {
      const int s = t % A_STAGES;
      ok = mbar_wait(&S.q_empty[s], ((uint32_t)(t / A_STAGES) & 1u) ^ 1u, P.status, P.limit);
      if (!ok) break;
      mbar_expect_tx(&S.q_full[s], TB);
#pragma unroll
      for (int sl = 0; sl < SLABS; ++sl)
        tma_load_4d(S.q + s * TB + sl * SLAB, &q_map, &S.q_full[s], 64 * sl, (int)cu + q0, h * P.q_head_step, 0);
      issued = t + 1;
      q0 += TILE;
      if (q0 >= N) { q0 = key0; ++h; }
    }
    // do not leave the CTA while a copy may still be writing its shared memory
    mbar_drain(S.k_full, 0, P.status);
    for (int t = max(0, issued - A_STAGES); t < issued; ++t)
      mbar_drain(&S.q_full[t % A_STAGES], (uint32_t)(t / A_STAGES) & 1u, P.status);
  } else if (warp == A_MMA) {
    const uint32_t id = instr_desc(TILE, TILE);
    const uint32_t a = (smem_u32(S.k) & 0x3FFFFu) >> 4, q_lo = (smem_u32(S.q) & 0x3FFFFu) >> 4;
    bool ok = mbar_wait(S.k_full, 0, P.status, P.limit);
    int last = -1;
    for (int t = 0; ok && t < n_tiles; ++t) {
      const int s = t % A_STAGES, buf = t % A_BUFS;
      ok = mbar_wait(&S.acc_empty[buf], ((uint32_t)(t / A_BUFS) & 1u) ^ 1u, P.status, P.limit);
      if (ok) ok = mbar_wait(&S.q_full[s], (uint32_t)(t / A_STAGES) & 1u, P.status, P.limit);
      if (!ok) break;
      tc_fence_after();
      const uint32_t b = q_lo + (uint32_t)(s * TB >> 4), d = tmem + 128u * buf;
      umma_ss<0>(d, a, b, id);
      umma_ss<1>(d, a + 2, b + 2, id);
      umma_ss<1>(d, a + 4, b + 4, id);
      umma_ss<1>(d, a + 6, b + 6, id);
      if constexpr (D == 128) {
        constexpr uint32_t o = SLAB >> 4;
        umma_ss<1>(d, a + o, b + o, id);
        umma_ss<1>(d, a + o + 2, b + o + 2, id);
        umma_ss<1>(d, a + o + 4, b + o + 4, id);
        umma_ss<1>(d, a + o + 6, b + o + 6, id);
      }
      umma_commit(&S.q_empty[s]);
      umma_commit(&S.acc_full[buf]);
      last = t;
    }
    // what was issued ends before tensor and shared memory are given back
    if (last >= 0) mbar_drain(&S.acc_full[last % A_BUFS], (uint32_t)(last / A_BUFS) & 1u, P.status);
  } else if (warp == A_LSE) {
    // -lse * log2(e) of the queries of every tile, three tiles ahead in registers
    constexpr int AHEAD = 3;
    float x[AHEAD][4];
    auto get = [&](int t, float (&v)[4]) {
      const int h = h0 + t / per_head, q0 = key0 + (t % per_head) * TILE;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = q0 + 32 * e + lane;
        v[e] = t < n_tiles && i < N ? -P.lse[h * P.T + cu + i] * kLog2E : 0.f;
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
        ok = mbar_wait(&S.acc_empty[buf], ((uint32_t)(t / A_BUFS) & 1u) ^ 1u, P.status, P.limit);
        if (!ok) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) S.nl[buf * 128 + 32 * e + lane] = x[u][e];
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.nl_full[buf]);
        get(t + AHEAD, x[u]);
      }
    }
  } else if (warp < A_TMA) {
    const int grp = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    float hi = 0.f, lo = 0.f;
    for (int t = grp; t < n_tiles; t += A_GROUPS) {
      const int buf = t % A_BUFS, q0 = key0 + (t % per_head) * TILE;
      const uint32_t ph = (uint32_t)(t / A_BUFS) & 1u;
      if (!mbar_wait(&S.nl_full[buf], ph, P.status, P.limit) || !mbar_wait(&S.acc_full[buf], ph, P.status, P.limit)) break;
      tc_fence_after();
      const uint32_t at = tmem + lanes + 128u * buf;
      const float x = q0 == key0 || q0 + TILE > N ? weigh_tile<true>(at, S.nl + buf * 128, P.scale2, q0 == key0 ? row : 0, N - q0)
                                                  : weigh_tile<false>(at, S.nl + buf * 128, P.scale2, 0, 0);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&S.acc_empty[buf]);
      const float y = hi + x;
      lo += hi >= x ? (hi - y) + x : (x - y) + hi;
      hi = y;
    }
    S.part[grp * 128 + row] = hi + lo;
  }
  tc_fence_before();
  __syncthreads();
  if (warp == A_MMA) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  } else if (threadIdx.x < TILE) {
    S.part[threadIdx.x] = (S.part[threadIdx.x] + S.part[128 + threadIdx.x]) + S.part[256 + threadIdx.x];
  }
  if constexpr (kSplit) cluster_sync();
  else __syncthreads();
  if (share == 0 && threadIdx.x < TILE && key0 + (int)threadIdx.x < N) {
    float x = S.part[threadIdx.x];
    for (int y = 1; kSplit && y < P.G; ++y) x += __uint_as_float(ld_peer(&S.part[threadIdx.x], (uint32_t)y));
    P.out[g * P.T + cu + key0 + threadIdx.x] = x * (1.f / (float)P.G);
  }
  if constexpr (kSplit) cluster_sync();          // nobody leaves while its sums may still be read
}

// ------------------------------------------------------------------ host
bool encode(CUtensorMap* map, const void* p, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  const EncodeTiledFn enc = encode_fn();
  const cuuint32_t es[4] = {1, 1, 1, 1};
  return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(p), dims, strides, box, es,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// K or V [rows][d] as (64 channels, rows, slabs): a box is a tile, slab by slab
bool encode_rows(CUtensorMap* map, const void* p, int64_t rows, int d) {
  const cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)(d / 64)}, strides[2] = {(cuuint64_t)d * 2, 128};
  const cuuint32_t box[3] = {64, TILE, (cuuint32_t)(d / 64)};
  return encode(map, p, 3, dims, strides, box);
}
// Queries as (channels, tokens, heads, 1); heads that are the same rows in memory are one
bool encode_q(CUtensorMap* map, const void* p, const cake_ctx* ctx, Strided s) {
  const cake_config& c = ctx->cfg;
  const cuuint64_t any = 16;
  const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)ctx->total_tokens, s.head ? (cuuint64_t)c.n_q_heads : 1, 1};
  const cuuint64_t strides[3] = {(cuuint64_t)s.token * 2, s.head ? (cuuint64_t)s.head * 2 : any, any};
  const cuuint32_t box[4] = {64, TILE, 1, 1};
  return encode(map, p, 4, dims, strides, box);
}

}  // namespace

template <int D>
static cudaError_t run_prompt_tc(const cake_ctx* ctx, const CUtensorMap& qm, const CUtensorMap& km, const CUtensorMap& vm,
                                 const PromptBatch& B, const PromptParams& P, cudaStream_t st) {
  static PerDeviceOnce once;
  if (once.need(ctx->device)) {
    const cudaError_t e = cudaFuncSetAttribute(prompt_tc<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PromptCfg<D>::SMEM);
    if (e != cudaSuccess) return e;
    once.mark(ctx->device);
  }
  return launch_early(prompt_tc<D>, (unsigned)(B.tiles * P.Hq), P_THREADS, PromptCfg<D>::SMEM, 1, st, qm, km, vm, B, P);
}

int32_t launch_prompt_tc(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const void* v, void* out, Strided os,
                         float* lse, float* lse_window, cudaStream_t st) {
  const cake_config& c = ctx->cfg;
  CUtensorMap qm, km, vm;
  const int64_t rows = c.n_kv_heads * ctx->total_tokens;
  if (!encode_q(&qm, q, ctx, qs) || !encode_rows(&km, k, rows, c.head_dim) || !encode_rows(&vm, v, rows, c.head_dim))
    return CAKE_ERR_CUDA;
  PromptParams P;
  P.v = (const __nv_bfloat16*)v; P.out = (__nv_bfloat16*)out; P.lse = lse; P.lse_window = lse_window; P.os = os;
  P.T = ctx->total_tokens; P.status = ctx->d_status;
  P.limit = ctx->wait_limit_cycles > 0 ? ctx->wait_limit_cycles : kSpinLimit;
  P.Hq = c.n_q_heads; P.G = c.n_q_heads / c.n_kv_heads; P.window = c.window;
  P.q_head_step = qs.head != 0;
  P.scale2 = kLog2E / sqrtf((float)c.head_dim);
  PromptBatch B;
  for (int lo = 0; lo < ctx->n_req; lo += B.n) {
    fill_prompt_batch(ctx, lo, 2 * TILE, B);
    CAKE_CUDA_TRY(c.head_dim == 128 ? run_prompt_tc<128>(ctx, qm, km, vm, B, P, st) : run_prompt_tc<64>(ctx, qm, km, vm, B, P, st));
  }
  return CAKE_OK;
}

template <int D, bool kSplit>
static cudaError_t run_accumulate_tc(const cake_ctx* ctx, const CUtensorMap& qm, const CUtensorMap& km, const PromptBatch& B,
                                     const AccParams& P, cudaStream_t st) {
  static PerDeviceOnce once;
  if (once.need(ctx->device)) {
    const cudaError_t e = cudaFuncSetAttribute(accumulate_tc<D, kSplit>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)acc_smem<D>());
    if (e != cudaSuccess) return e;
    once.mark(ctx->device);
  }
  return launch_early(accumulate_tc<D, kSplit>, (unsigned)(B.tiles * (kSplit ? P.Hq : P.Hkv)), A_THREADS, acc_smem<D>(), kSplit ? P.G : 1,
                      st, qm, km, B, P);               // (G is at most 8: portable)
}

int32_t launch_accumulate_tc(const cake_ctx* ctx, const void* q, Strided qs, const void* k, const float* lse, float* out,
                             cudaStream_t st) {
  const cake_config& c = ctx->cfg;
  CUtensorMap qm, km;
  if (!encode_q(&qm, q, ctx, qs) || !encode_rows(&km, k, c.n_kv_heads * ctx->total_tokens, c.head_dim)) return CAKE_ERR_CUDA;
  AccParams P;
  P.lse = lse; P.out = out; P.T = ctx->total_tokens; P.status = ctx->d_status;
  P.limit = ctx->wait_limit_cycles > 0 ? ctx->wait_limit_cycles : kSpinLimit;
  P.Hq = c.n_q_heads; P.Hkv = c.n_kv_heads; P.G = c.n_q_heads / c.n_kv_heads;
  P.q_head_step = qs.head != 0;
  P.scale2 = kLog2E / sqrtf((float)c.head_dim);
  PromptBatch B;
  for (int lo = 0; lo < ctx->n_req; lo += B.n) {
    fill_prompt_batch(ctx, lo, TILE, B);
    const bool split = P.G > 1 && B.tiles * P.Hkv < ctx->n_sm;
    CAKE_CUDA_TRY(c.head_dim == 128 ? (split ? run_accumulate_tc<128, true>(ctx, qm, km, B, P, st) : run_accumulate_tc<128, false>(ctx, qm, km, B, P, st))
                                    : (split ? run_accumulate_tc<64, true>(ctx, qm, km, B, P, st) : run_accumulate_tc<64, false>(ctx, qm, km, B, P, st)));
  }
  return CAKE_OK;
}

}  // namespace cake
