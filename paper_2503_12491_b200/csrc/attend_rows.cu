// Attention of one new token per request over its cached rows: the rows in the context's type (bf16 or fp32) or in 4 bits, and behind
// either the rows of tokens generated since.
//
//   O_h = sum_j softmax_j(q_h.k_j / sqrt d) v_j ,  lse_h = log sum_j exp(q_h.k_j / sqrt d)   over all rows j of h's KV head.
//
// Work.  The (request, KV head) pairs of the layer are cut into units of 32 rows (the tail's rows behind the packed ones; 8 rows
// a unit in the 4-bit kernel, whose stages are smaller), and every CTA of one per SM takes the same number of consecutive
// units, whatever pairs they belong to: the device works evenly on ragged batches, and on one long request.  Lengths lie on
// the device, so each CTA adds up the units of all requests for itself.  Inside a CTA the warps take the units in turn, each
// with copies of its own units in flight (cp.async) and its own running softmax.  Where a pair ends they leave their results in one
// of two places in turn, without waiting, and the first warp that wants the place again puts them together: the one that is
// ahead.  (With a barrier at each end 256 requests of 560 rows in 4 bits took 131 us, where this takes 109; the last warp
// doing it, which is the one behind, 117.)  A pair that lies in one CTA is finished there; of the others a CTA leaves its share in the workspace (at most one share at either end
// of its run), and merge_shares, a CTA per boundary between two runs, puts them together: no CTA waits for another, and the
// workspace needs no initialisation.  (In one launch instead: by clusters of 16 CTAs per head 11.2 us for one request of 2048 rows
// and 8 heads, where this takes 8.6; by the CTA that leaves a pair's last share, counted with atomics, 16.4.)
//
// bf16 queries: products on the tensor cores (mma m16n8k16).  S^T[key][col] = K Q^T and O^T[channel][col] = V^T P^T with the
// query heads as the 8 columns.  With up to four heads the columns 4 to 7 hold the same heads once more, for the second term of
// what is held in two bf16 terms (kTwo): weights, and queries and weights times scales, are then exact to 2^-16.  With more heads
// the 4-bit kernel multiplies twice, and the weights of bf16 rows are rounded to bf16.
//
// 4-bit rows.  A code c becomes the bf16 16 + c (or 128 + c) by a logical operation per pair and at most one shift; scales and
// zeros are never applied to a row but to the other operand: q_c s_c for the keys, p_j s_j for the values, and
//     q.k = sum_c (q_c s_c)(code - 8) + sum_c q_c (z_c + 8 s_c) ,   p.v = sum_j (p_j s_j)(code - 8) + sum_j p_j (z_j + 8 s_j) .
// What was added to the codes, and the 8, which makes the rounding of the other operand count as little as it can, comes off by
// products of that rounded operand with a constant (the tensor cores are idle for the most part; logical operations set the
// pace).  Channels and keys are taken in whatever order the words bring them, the same one in both operands; a value tile's 16
// channels come from one group of 32, which has one scale per row.
//
// Bound, for 8 KV heads of 32 query heads.  bf16 rows: DRAM, 5.8 TB/s of the 6.5 that a copy reaches (75 us for 32 requests of 1000 to
// 6000 rows of 128 channels; 64 channels 4.4, 49 us).  fp32 rows: three warps per SM with chains of FMA
// behind reads of shared memory (a 16-byte piece of a query per four of them): 5.1 TB/s (172 us; 64 channels 3.0, 148 us).  4-bit rows, bf16 queries: a unit of 32 rows and 128 channels
// is about 1050 instructions of a warp, half of them logical operations or additions of whole numbers at two cycles each, 1050 cycles of
// that pipe, beside 56 products at eight (112 with more than four heads), 450 of the tensor cores: 2.7 TB/s (78 us for 32 requests of
// 1000 to 8000 rows; 32 us of DRAM).  4-bit rows, fp32 queries: FMA and conversions of codes, 1.3 TB/s (166 us of the same rows).
#include "cache_mma.cuh"
#include "tc_ptx.cuh"

namespace cake {
namespace {

constexpr float kRefSlack = 8.f;                 // powers of two a maximum may lie above the reference before all is rescaled

template <typename T, int D, int GROUP> struct RowsCfg {
  static constexpr bool INT4 = GROUP != 0, F32 = sizeof(T) == 4;
  static constexpr int UNIT = 32, TAIL = !INT4 ? 32 : F32 ? 4 : 8;               // rows of a unit
  static constexpr int NG = INT4 ? D / GROUP : 1;                                // channel groups of a row
  static constexpr int K_BYTES = INT4 ? UNIT * D / 2 : UNIT * D * (int)sizeof(T);
  static constexpr int VS_BYTES = INT4 ? UNIT * NG * 4 : 0, KS_BYTES = INT4 ? D * 4 : 0;
  static constexpr int STAGE = 2 * (K_BYTES + VS_BYTES + KS_BYTES);
  static_assert(2 * TAIL * D * (int)sizeof(T) <= STAGE, "tail rows fit a stage");
};

struct RowsParams {
  CacheParams c;
  float* shares;                                 // [CTA][2][G][D], then [CTA][2][G][2] (reference, sum)
  int32_t* status;
  long long limit;                               // cycles that a wait may take
  int n_req;
};
__host__ __device__ inline int64_t share_stats(int ctas, int G, int D) { return (int64_t)ctas * 2 * G * D; }

// Rows of a request's pairs.
struct Lengths {
  int64_t first, n;                              // first row of head 0; packed rows per head
  int64_t kgroup;                                // first key group of head 0 (4-bit rows)
  int32_t tail;
};
__device__ __forceinline__ Lengths lengths_of(const CacheParams& c, int r) {
  const int64_t block = (int64_t)r * c.n_layers + c.layer;
  Lengths x;
  x.first = c.row_off[block];
  const int64_t rows = max((int64_t)0, c.row_off[block + 1] - x.first);
  x.n = rows >> 32 ? rows / c.Hkv : (int64_t)((uint32_t)rows / (uint32_t)c.Hkv);
  x.kgroup = c.group_off ? c.group_off[block] : 0;
  x.tail = c.tail_cap ? (int32_t)max((int64_t)0, min((int64_t)c.tail_len[r], c.tail_cap)) : 0;
  return x;
}
template <int UNIT, int TAIL>
__device__ __forceinline__ int units_of(const Lengths& x) { return (int)((x.n + UNIT - 1) / UNIT) + (x.tail + TAIL - 1) / TAIL; }

// Sum of v over the lanes up to this one.
__device__ __forceinline__ int lanes_before(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += x;
  }
  return v;
}
// Units of 32 requests at a time, by a whole warp: the lengths of this lane's request, the sum of units up to it, all requests'.
template <int UNIT, int TAIL>
struct Requests {
  Lengths len;
  int units, upto, all;
  __device__ __forceinline__ void read(const CacheParams& c, int n_req, int base, int lane) {
    len = Lengths{};
    units = 0;
    if (base + lane < n_req) {
      len = lengths_of(c, base + lane);
      units = units_of<UNIT, TAIL>(len);
    }
    upto = lanes_before(units, lane);
  }
  // All of them, the first ones last (they stay); each(base) after every 32.  (A trip to memory per 32 requests, in both kernels: 8192
  // requests of one row take 0.31 ms for that, 65 535 2.9.)
  template <typename F>
  __device__ __forceinline__ void read_all(const CacheParams& c, int n_req, int lane, F each) {
    all = 0;
    for (int base = (n_req - 1) / 32 * 32; base >= 0; base -= 32) {
      read(c, n_req, base, lane);
      all += __shfl_sync(0xffffffffu, upto, 31);
      each(base);
    }
  }
};
// (Units are counted in 32 bits: 2^31 of them are 4 TB of 4-bit rows.)
__device__ __forceinline__ int per_cta(int units, int ctas) { return max(1, (units + ctas - 1) / ctas); }

// A place in the sequence of units: moves forward only.
template <typename T, int D, int GROUP>
struct Cursor {
  using C = RowsCfg<T, D, GROUP>;
  int r, g;
  int start, units;                              // first unit of the pair, and how many it has
  Lengths len;
  // At the pair of unit u, by a whole warp.
  __device__ __forceinline__ void open(const CacheParams& c, int n_req, Requests<C::UNIT, C::TAIL>& Q, int u, int lane) {
    int before = 0;
    for (int base = 0; ; base += 32) {
      const uint32_t found = __ballot_sync(0xffffffffu, (before + Q.upto) * c.Hkv > u);
      if (found) {
        const int at = __ffs(found) - 1;
        r = base + at; g = 0;
        units = __shfl_sync(0xffffffffu, Q.units, at);
        start = (before + __shfl_sync(0xffffffffu, Q.upto, at) - units) * c.Hkv;
        len.first = __shfl_sync(0xffffffffu, Q.len.first, at);
        len.n = __shfl_sync(0xffffffffu, Q.len.n, at);
        len.kgroup = __shfl_sync(0xffffffffu, Q.len.kgroup, at);
        len.tail = __shfl_sync(0xffffffffu, Q.len.tail, at);
        const int heads = (u - start) / units;
        g = heads;
        start += heads * units;
        return;
      }
      before += __shfl_sync(0xffffffffu, Q.upto, 31);
      if (base + 32 >= n_req) return;                // (u is one of the units: not reached)
      Q.read(c, n_req, base + 32, lane);
    }
  }
  __device__ __forceinline__ void next(const CacheParams& c, int n_req) {
    start += units;
    if (++g < c.Hkv) return;
    g = 0;
    if (++r >= n_req) { units = 1 << 30; return; }
    len = lengths_of(c, r);
    units = units_of<C::UNIT, C::TAIL>(len);
  }
  __device__ __forceinline__ void seek(const CacheParams& c, int n_req, int u) { while (u - start >= units) next(c, n_req); }
};

__device__ __forceinline__ void narrow(float* p, float x) { *p = x; }
__device__ __forceinline__ void narrow(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
// Two or four consecutive numbers, from shared memory and to where they are stored.
__device__ __forceinline__ void ld_floats(float (&x)[2], const float* p) { const float2 a = *reinterpret_cast<const float2*>(p); x[0] = a.x; x[1] = a.y; }
__device__ __forceinline__ void ld_floats(float (&x)[4], const float* p) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
}
__device__ __forceinline__ void st_row(float* p, const float (&x)[2]) { *reinterpret_cast<float2*>(p) = make_float2(x[0], x[1]); }
__device__ __forceinline__ void st_row(float* p, const float (&x)[4]) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void st_row(__nv_bfloat16* p, const float (&x)[2]) { *reinterpret_cast<uint32_t*>(p) = bf16_pair(x[0], x[1]); }
__device__ __forceinline__ void st_row(__nv_bfloat16* p, const float (&x)[4]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]));
}

// Counters in shared memory through which warps hand results to one another.
__device__ __forceinline__ void arrive(int* p, int n) {
  asm volatile("red.release.cta.shared::cta.add.s32 [%0], %1;" ::"r"(smem_addr(p)), "r"(n) : "memory");
}
// Of n + (n << 8), all of the warps: marks them as taken, for one caller.
__device__ __forceinline__ bool take_full(int* p) {
  int x, old;
  asm volatile("ld.acquire.cta.shared::cta.s32 %0, [%1];" : "=r"(x) : "r"(smem_addr(p)) : "memory");
  if (x == 0 || (x & 255) != x >> 8) return false;
  asm volatile("atom.acquire.cta.shared::cta.cas.b32 %0, [%1], %2, %3;" : "=r"(old) : "r"(smem_addr(p)), "r"(x), "r"(1 << 30) : "memory");
  return old == x;
}
__device__ __forceinline__ void set_count(int* p, int n) {
  asm volatile("st.release.cta.shared::cta.s32 [%0], %1;" ::"r"(smem_addr(p)), "r"(n) : "memory");
}
// Until the counter is at least n, by every lane; false after `limit` cycles.
__device__ __forceinline__ bool wait_count(const int* p, int n, int32_t* status, long long limit) {
  const long long t0 = clock64();
  for (;;) {
    int x;
    asm volatile("ld.acquire.cta.shared::cta.s32 %0, [%1];" : "=r"(x) : "r"(smem_addr(p)) : "memory");
    const bool there = x >= n;
    if (__all_sync(0xffffffffu, there)) return true;
    const bool late = clock64() - t0 > limit;
    if (__any_sync(0xffffffffu, late)) {
      atomicCAS(status, 0, CAKE_ERR_TIMEOUT);
      return false;
    }
  }
}

__device__ __forceinline__ float ex2a(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <typename T, int D, int GROUP, bool kTwo, int W, int ST>
struct RowsSmem {
  using C = RowsCfg<T, D, GROUP>;
  static constexpr int HEADS = kTwo ? 4 : 8, PK = 36;                            // floats of a head's weights of a unit (padded)
  // a warp's results of a pair: outputs [head][channel], sums of weights times zeros [head][group], (reference, sum) [head]
  static constexpr int ZEROS = HEADS * D, STATS = ZEROS + HEADS * C::NG, RESULT = (STATS + 2 * HEADS + 3) / 4 * 4;
  static constexpr size_t RING = (size_t)W * ST * C::STAGE, WEIGHTS = (size_t)W * (HEADS * PK + (C::F32 ? HEADS * D : 0)) * 4,
                          CURSORS = (size_t)W * sizeof(Cursor<T, D, GROUP>), RESULTS = (size_t)W * RESULT * 4;
  // places for all warps' results of a pair: two if they fit
  static constexpr int PLACES = RING + WEIGHTS + CURSORS + 2 * RESULTS + 48 <= 227 * 1024 ? 2 : 1;
  static constexpr size_t BYTES = RING + WEIGHTS + CURSORS + PLACES * RESULTS + 48;
  static_assert(C::STAGE >= RESULT * 4 && WEIGHTS % 16 == 0 && CURSORS % 16 == 0, "a warp's results fit a stage; 16-byte pieces");
};

// A warp's running softmax: reference and (this lane's part of the) sum of the two heads of its columns 2 j, 2 j + 1, outputs
// as the products leave them, and for 4-bit rows the sums of weights times zeros of the head of column lane / 4.
template <int D, int NG>
struct Running {
  float ref[2], sum[2], o[D / 16][4];
  f32x2 z[(NG + 1) / 2];
  __device__ __forceinline__ void clear() {
    ref[0] = ref[1] = kNoWeight;
    sum[0] = sum[1] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
#pragma unroll
    for (int i = 0; i < (NG + 1) / 2; ++i) z[i] = pack2(0.f, 0.f);
  }
};

// Weights of a unit's keys against the reference, which moves up first if a maximum lies too far above it; into shared
// memory as [head][key].  s: logits of keys 16 m + lane / 4 (+ 8).
template <int D, int NG, bool kTwo, int MT, int PK>
__device__ __forceinline__ void weigh(Running<D, NG>& R, float (&s)[MT][4], int valid, float scale2, float* sp, int lane) {
  float top[2] = {-CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[m][e] *= scale2;
      if (valid < 16 * MT && 16 * m + (lane >> 2) + 8 * (e >> 1) >= valid) s[m][e] = -CUDART_INF_F;
      top[e & 1] = fmaxf(top[e & 1], s[m][e]);
    }
#pragma unroll
  for (int x = 4; x < 32; x <<= 1) {
    top[0] = fmaxf(top[0], __shfl_xor_sync(0xffffffffu, top[0], x));
    top[1] = fmaxf(top[1], __shfl_xor_sync(0xffffffffu, top[1], x));
  }
  if (__any_sync(0xffffffffu, top[0] > R.ref[0] + kRefSlack || top[1] > R.ref[1] + kRefSlack)) {
    float f[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float to = top[h] > R.ref[h] + kRefSlack ? top[h] : R.ref[h];
      f[h] = to == R.ref[h] ? 1.f : ex2a(R.ref[h] - to);
      R.ref[h] = to;
      R.sum[h] *= f[h];
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) R.o[i][e] *= f[e & 1];
    // the factor of the head of column lane / 4: from a lane that has this column
    const int col = kTwo ? (lane >> 2) & 3 : lane >> 2;
    const float a = __shfl_sync(0xffffffffu, f[0], col >> 1), b = __shfl_sync(0xffffffffu, f[1], col >> 1);
#pragma unroll
    for (int i = 0; i < (NG + 1) / 2; ++i) R.z[i] = mul2(R.z[i], pack2(col & 1 ? b : a, col & 1 ? b : a));
  }
  const int j = lane & 3;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = ex2a(s[m][e] - R.ref[e & 1]);
      R.sum[e & 1] += p;
      if (!kTwo || j < 2) sp[(2 * j + (e & 1)) * PK + 16 * m + (lane >> 2) + 8 * (e >> 1)] = p;
    }
  __syncwarp();
}

// A pair of weights as this lane's column takes them: with kTwo the leading bits for columns 0-3, the rest for 4-7.
template <bool kTwo>
__device__ __forceinline__ uint32_t weight_pair(float a, float b, bool second) {
  if constexpr (!kTwo) return bf16_pair(a, b);
  const float x = bf16_floor(a), y = bf16_floor(b);
  return bf16_pair(second ? a - x : x, second ? b - y : y);
}

// 32 rows (MT = 2), or up to 8 (MT = 1) behind 4-bit rows, whose outputs' order of channels they take: rows i and i + 8 of
// output tile t are channels 32 (t / 2) + 4 i + 2 (t % 2) and the one after it.
template <int D, int NG, bool kTwo, int MT, int PK>
__device__ __forceinline__ void dense_unit(Running<D, NG>& R, const uint32_t (&q)[D / 16][2], uint32_t k_at, uint32_t v_at, int valid,
                                           float scale2, float* sp, int lane) {
  const int i8 = lane >> 3, l8 = lane & 7;
  float s[MT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    s[m][0] = s[m][1] = s[m][2] = s[m][3] = 0.f;
    const int row = 16 * m + l8 + 8 * (MT == 2 ? i8 & 1 : 0);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      uint32_t a[4];
      ldmatrix4(a, k_at + (uint32_t)(row * D * 2 + (((2 * ks + (i8 >> 1)) ^ (row & 7)) << 4)));
      if (MT == 1) a[1] = a[3] = 0u;               // eight rows: the lower half of the tile
      mma16816(s[m], a[0], a[1], a[2], a[3], q[ks][0], q[ks][1]);
    }
  }
  weigh<D, NG, kTwo, MT, PK>(R, s, valid, scale2, sp, lane);
  const int n = lane >> 2, j = lane & 3, h = kTwo ? n & 3 : n;
#pragma unroll
  for (int ks = 0; ks < MT; ++ks) {
    const float* p = sp + h * PK + 16 * ks + 2 * j;
    const float2 lo = *reinterpret_cast<const float2*>(p), hi = MT == 2 ? *reinterpret_cast<const float2*>(p + 8) : make_float2(0.f, 0.f);
    const uint32_t b0 = weight_pair<kTwo>(lo.x, lo.y, n >= 4), b1 = weight_pair<kTwo>(hi.x, hi.y, n >= 4);
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) {
      if constexpr (MT == 2) {
        const int row = 16 * ks + l8 + 8 * (i8 >> 1);
        uint32_t a[4];
        ldmatrix4t(a, v_at + (uint32_t)(row * D * 2 + (((2 * ct + (i8 & 1)) ^ (row & 7)) << 4)));
        mma16816(R.o[ct], a[0], a[1], a[2], a[3], b0, b1);
      } else {
        const int ch = 32 * (ct / 2) + 4 * n + 2 * (ct & 1);
        uint32_t w[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int row = 2 * j + u;
          asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[u]) : "r"(v_at + (uint32_t)(row * D * 2 + (((ch >> 3) ^ (row & 7)) << 4) + (ch & 7) * 2)) : "memory");
        }
        mma16816(R.o[ct], __byte_perm(w[0], w[1], 0x5410), __byte_perm(w[0], w[1], 0x7632), 0u, 0u, b0, b1);
      }
    }
  }
  __syncwarp();
}

// Nibbles I and I + 4 of a word as bf16: 128 + code for the first (in the mantissa's lowest bits, no shift), else 16 + code; and
// minus what that is for a code of 8.
template <int I> __device__ __forceinline__ uint32_t codes(uint32_t w) {
  return I == 0 ? (w & 0x000F000Fu) | 0x43004300u : ((w >> (I ? 4 * I - 3 : 0)) & 0x00780078u) | 0x41804180u;
}
template <int I> constexpr uint32_t kMinusMid = I == 0 ? 0xC308C308u : 0xC1C0C1C0u;      // -136, -24

// 32 rows in 4 bits.  qf: queries of the head of column lane / 4, pairs of channels of quarter lane % 4 of a row (with kTwo the
// half of them that this lane works on).  With kTwo the
// lanes of columns i and i + 4, which have the same head, share the work on the other operands: each takes half of the channels (of
// the keys) and hands the other the part of its results that this one multiplies with.
template <int D, int GROUP, bool kTwo, int PK>
__device__ __forceinline__ void int4_unit(Running<D, D / GROUP>& R, const f32x2 (&qf)[D / (kTwo ? 16 : 8)], uint32_t st, int valid, float scale2, float* sp,
                                          int lane) {
  using C = RowsCfg<__nv_bfloat16, D, GROUP>;
  constexpr int NG = C::NG, WORDS = D / 32;        // words of a quarter of a row
  const int n = lane >> 2, j = lane & 3;
  const bool second = n >= 4;
  const uint32_t kc = st, vc = st + C::K_BYTES, ks = st + 2 * C::K_BYTES, vs = ks + 2 * D * 4;
  // --- keys: the queries times the scales of the unit's group in two bf16 terms, and what the zeros and middles give
  uint32_t b[D / 16][2], b2[D / 16][2];              // (kTwo: b alone is multiplied with)
  f32x2 bias = pack2(0.f, 0.f);
  constexpr int MINE = kTwo ? WORDS / 2 : WORDS;
  // pieces of this lane's quarter: t at t ^ j among four (128 channels; 64: see load_int4)
  const uint32_t ks_at = ks + (D == 128 ? j * 128 + (kTwo && second ? 64 : 0) : (j >> 1) * 128);
#pragma unroll
  for (int u = 0; u < MINE; ++u) {
    float x[8], r[8];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      uint32_t at;
      if constexpr (D == 128) {
        at = ks_at + ((((2 * u + e) & 3) ^ j) << 4) + ((2 * u + e) >> 2) * 64;
      } else {
        at = ks_at + ((((j & 1) * 4 + 2 * (u + (kTwo && second ? WORDS / 2 : 0)) + e) ^ (j >> 1)) << 4);
      }
      f32x2 sc[2], ze[2];
      ld_shared(sc, at);
      ld_shared<D * 4>(ze, at);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f32x2 q = qf[4 * u + 2 * e + i];
        const f32x2 y = mul2(q, sc[i]);
        bias = fma2(q, fma2(pack2(8.f, 8.f), sc[i], ze[i]), bias);
        float y0, y1;
        unpack2(y, y0, y1);
        const int at8 = 4 * e + 2 * i;
        x[at8] = bf16_floor(y0); x[at8 + 1] = bf16_floor(y1);
        unpack2(fma2(pack2(x[at8], x[at8 + 1]), pack2(-1.f, -1.f), y), r[at8], r[at8 + 1]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {                  // channels i and i + 4 of the word
      const uint32_t lead = bf16_pair(x[i], x[i + 4]), rest = bf16_pair(r[i], r[i + 4]);
      if constexpr (kTwo) {
        const uint32_t keep = second ? rest : lead, got = __shfl_xor_sync(0xffffffffu, second ? lead : rest, 16);
        // the first lane worked on word u and gets word u + WORDS / 2, the second the other way round
        b[2 * u + i / 2][i & 1] = second ? got : keep;
        b[2 * (u + WORDS / 2) + i / 2][i & 1] = second ? keep : got;
      } else {
        b[2 * u + i / 2][i & 1] = lead;
        b2[2 * u + i / 2][i & 1] = rest;
      }
    }
  }
  float bi, bi1;
  unpack2(bias, bi, bi1);
  bi += bi1;
  bi += __shfl_xor_sync(0xffffffffu, bi, 1);
  bi += __shfl_xor_sync(0xffffffffu, bi, 2);
  if constexpr (kTwo) bi += __shfl_xor_sync(0xffffffffu, bi, 16);
  const int c0 = kTwo ? (2 * j) & 3 : 2 * j;
  float bias0 = __shfl_sync(0xffffffffu, bi, 4 * c0), bias1 = __shfl_sync(0xffffffffu, bi, 4 * c0 + 4);
  // with kTwo both terms are added up below, and these must come in once
  if (kTwo && j >= 2) bias0 = bias1 = 0.f;
  float s[2][4] = {}, mid[4] = {bias0, bias1, bias0, bias1};
  const uint32_t k_at = D == 128 ? kc + n * 64 + ((j ^ ((n >> 1) & 3)) << 4) : kc + n * 32 + j * 8;
  for_n<2>([&](auto m) {
    uint32_t a[WORDS], c[WORDS];
    ld_shared<m.value * 8 * D>(a, k_at);
    ld_shared<m.value * 8 * D + 4 * D>(c, k_at);
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      constexpr uint32_t m0 = kMinusMid<0>, m1 = kMinusMid<1>;
      const uint32_t a0 = codes<0>(a[w]), a1 = codes<0>(c[w]), a2 = codes<1>(a[w]), a3 = codes<1>(c[w]);
      const uint32_t d0 = codes<2>(a[w]), d1 = codes<2>(c[w]), d2 = codes<3>(a[w]), d3 = codes<3>(c[w]);
      mma16816(s[m], a0, a1, a2, a3, b[2 * w][0], b[2 * w][1]);
      mma16816(s[m], d0, d1, d2, d3, b[2 * w + 1][0], b[2 * w + 1][1]);
      if (m == 0) {
        mma16816(mid, m0, m0, m1, m1, b[2 * w][0], b[2 * w][1]);
        mma16816(mid, m1, m1, m1, m1, b[2 * w + 1][0], b[2 * w + 1][1]);
      }
      if constexpr (!kTwo) {
        mma16816(s[m], a0, a1, a2, a3, b2[2 * w][0], b2[2 * w][1]);
        mma16816(s[m], d0, d1, d2, d3, b2[2 * w + 1][0], b2[2 * w + 1][1]);
        if (m == 0) {
          mma16816(mid, m0, m0, m1, m1, b2[2 * w][0], b2[2 * w][1]);
          mma16816(mid, m1, m1, m1, m1, b2[2 * w + 1][0], b2[2 * w + 1][1]);
        }
      }
    }
  });
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[m][e] += mid[e];
      if (kTwo) s[m][e] += __shfl_xor_sync(0xffffffffu, s[m][e], 2);
    }
  weigh<D, NG, kTwo, 2, PK>(R, s, valid, scale2, sp, lane);
  // --- values: keys j, j + 4, j + 8, j + 12 of 16; the weights times the scales
  const float* p = sp + (kTwo ? n & 3 : n) * PK;
  uint32_t bb[2][NG][2], b3[2][NG][2];               // leading terms and the rest (kTwo: as this lane's column takes them, in bb)
#pragma unroll
  for (int half = 0; half < (kTwo ? 1 : 2); ++half) {
    const int kstep = kTwo ? second : half;
    float x[NG][4];
    const uint32_t p_at = smem_addr(p) + (16 * kstep + j) * 4, vs_at = vs + (16 * kstep + j) * NG * 4;
    for_n<4>([&](auto i) {                           // (zeros lie 32 rows of scales further)
      const float w = ld_shared_f<i.value * 16>(p_at);
      if constexpr (NG > 1) {
        f32x2 sc[NG / 2], ze[NG / 2];
        ld_shared<i.value * 16 * NG>(sc, vs_at);
        ld_shared<(i.value * 4 + 32) * NG * 4>(ze, vs_at);
#pragma unroll
        for (int g = 0; g < NG / 2; ++g) {
          unpack2(mul2(pack2(w, w), sc[g]), x[2 * g][i], x[2 * g + 1][i]);
          R.z[g] = fma2(pack2(w, w), fma2(pack2(8.f, 8.f), sc[g], ze[g]), R.z[g]);
        }
      } else {
        const float sc = ld_shared_f<i.value * 16>(vs_at), ze = ld_shared_f<(i.value * 4 + 32) * 4>(vs_at);
        x[0][i] = w * sc;
        R.z[0] = fma2(pack2(w, 0.f), pack2(fmaf(8.f, sc, ze), 0.f), R.z[0]);
      }
    });
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float a = bf16_floor(x[g][2 * u]), b = bf16_floor(x[g][2 * u + 1]);
        const uint32_t lead = bf16_pair(a, b), rest = bf16_pair(x[g][2 * u] - a, x[g][2 * u + 1] - b);
        if constexpr (kTwo) {
          const uint32_t got = __shfl_xor_sync(0xffffffffu, second ? lead : rest, 16);
          bb[0][g][u] = second ? got : lead;
          bb[1][g][u] = second ? rest : got;
        } else {
          bb[half][g][u] = lead;
          b3[half][g][u] = rest;
        }
      }
  }
  // row 16 kstep + j + 4 i, piece blk: at blk ^ (2 (i % 2)) ^ (j / 2) (128 channels)
  const uint32_t v_at = vc + j * (D / 2) + 2 * n, v_even = v_at + (D == 128 ? (j >> 1) * 16 : 0), v_odd = v_at - (D == 128 ? (j >> 1) * 16 : 0);
  for_n<2>([&](auto kstep) {
    for_n<D / 32>([&](auto blk) {                    // 32 channels: two bytes of this lane's per row
      uint32_t h[4];
      for_n<4>([&](auto i) {
        constexpr int piece = D == 128 ? blk.value ^ (2 * (i.value & 1)) : blk.value;
        h[i] = ld_shared_u16<(16 * kstep.value + 4 * i.value) * (D / 2) + piece * 16>(piece & 1 ? v_odd : v_even);
      });
      const uint32_t w0 = __byte_perm(h[0], h[1], 0x5410), w1 = __byte_perm(h[2], h[3], 0x5410);
      constexpr int g = blk.value / ((D / 32) / NG);
      float (&o0)[4] = R.o[2 * blk], (&o1)[4] = R.o[2 * blk + 1];
      mma16816(o0, codes<0>(w0), codes<1>(w0), codes<0>(w1), codes<1>(w1), bb[kstep][g][0], bb[kstep][g][1]);
      mma16816(o1, codes<2>(w0), codes<3>(w0), codes<2>(w1), codes<3>(w1), bb[kstep][g][0], bb[kstep][g][1]);
      mma16816(o0, kMinusMid<0>, kMinusMid<1>, kMinusMid<0>, kMinusMid<1>, bb[kstep][g][0], bb[kstep][g][1]);
      mma16816(o1, kMinusMid<1>, kMinusMid<1>, kMinusMid<1>, kMinusMid<1>, bb[kstep][g][0], bb[kstep][g][1]);
      if constexpr (!kTwo) {
        mma16816(o0, codes<0>(w0), codes<1>(w0), codes<0>(w1), codes<1>(w1), b3[kstep][g][0], b3[kstep][g][1]);
        mma16816(o1, codes<2>(w0), codes<3>(w0), codes<2>(w1), codes<3>(w1), b3[kstep][g][0], b3[kstep][g][1]);
        mma16816(o0, kMinusMid<0>, kMinusMid<1>, kMinusMid<0>, kMinusMid<1>, b3[kstep][g][0], b3[kstep][g][1]);
        mma16816(o1, kMinusMid<1>, kMinusMid<1>, kMinusMid<1>, kMinusMid<1>, b3[kstep][g][0], b3[kstep][g][1]);
      }
    });
  });
  __syncwarp();
}

// Copies of ROWS rows of the context's type (those from `valid` on read as zeros) into shared memory, 16-byte piece c of a row at
// c ^ (row % 8).
template <typename T, int D, int ROWS>
__device__ __forceinline__ void load_dense(uint32_t dst, const T* src, int valid, int lane) {
  constexpr int CH = D * (int)sizeof(T) / 16, STEP = 32 / CH;
  const int r0 = lane / CH, c = lane % CH;
  for_n<ROWS / STEP>([&](auto i) {
    const int r = r0 + i * STEP;
    copy_async16n<0, i.value * 512>(dst + (uint32_t)(r * D * (int)sizeof(T) + ((c ^ (r & 7)) << 4)), (const uint8_t*)src + lane * 16,
                                    r < valid ? 16 : 0);
  });
}
// Copies of a unit of 4-bit rows: codes (128 channels: piece c of a row at c ^ (row / 2 % 4), so that neither the keys' 16-byte
// nor the values' 2-byte reads meet bank conflicts), the keys' scales and zeros of their group (piece c at c ^ (c / 8) within eight
// pieces, for the same reason), the values' scales and zeros.
template <int D, int GROUP>
__device__ __forceinline__ void load_int4(uint32_t at, const CacheParams& c, int64_t row, int64_t kgroup, int valid, int lane) {
  using C = RowsCfg<float, D, GROUP>;                // (4-bit rows lie in shared memory alike for both types)
  constexpr int NG = C::NG, CH = D / 32, ROWS = 32 / CH;                         // pieces of a row; rows of a pass of the warp
  const uint8_t *k = (const uint8_t*)c.k + row * (D / 2) + lane * 16, *v = (const uint8_t*)c.v + row * (D / 2) + lane * 16;
  const int r0 = lane / CH, p = lane % CH;
  // (the rows of a lane are 8 or 16 apart: their pieces are turned alike)
  const uint32_t to = at + (uint32_t)(r0 * (D / 2) + ((D == 128 ? p ^ ((r0 >> 1) & 3) : p) << 4));
  for_n<C::UNIT / ROWS>([&](auto i) {
    const int n = r0 + i * ROWS < valid ? 16 : 0;                                // beyond: zeros, nothing is read
    copy_async16n<i.value * 512, i.value * 512>(to, k, n);
    copy_async16n<i.value * 512 + C::K_BYTES, i.value * 512>(to, v, n);
  });
  const uint32_t ks = at + 2 * C::K_BYTES, vs = ks + 2 * C::KS_BYTES;
  if (lane < D / 4) {
    const uint32_t to = ks + ((lane & ~7) | ((lane ^ (lane >> 3)) & 7)) * 16;
    const int64_t from = kgroup * D + lane * 4;
    copy_async16n(to, c.k_scale + from, 16);
    copy_async16n<C::KS_BYTES>(to, c.k_zero + from, 16);
  }
  if constexpr (NG == 4) {                           // a row's scales start on a 16-byte boundary
    const int n = lane < valid ? 16 : 0;
    const int64_t from = (row + lane) * 4;
    copy_async16n(vs + lane * 16, c.v_scale + from, n);
    copy_async16n<C::VS_BYTES>(vs + lane * 16, c.v_zero + from, n);
  } else {
    const int64_t from = row * NG + lane;
    for_n<NG>([&](auto i) {
      const int n = (lane + 32 * i) / NG < valid ? 4 : 0;
      copy_async4n<i.value * 128, i.value * 128>(vs + lane * 4, c.v_scale + from, n);
      copy_async4n<i.value * 128 + C::VS_BYTES, i.value * 128>(vs + lane * 4, c.v_zero + from, n);
    });
  }
}

// ------------------------------------------------------------------ fp32 queries
// Products in fp32 FMA.  For the logits a lane is a key, for the outputs it owns D / 32 channels: the keys' weights go through
// shared memory in between, and the queries come from there too, as 16-byte pieces that all lanes read at once.
template <int D, int HEADS>
struct Running32 {
  float ref[HEADS], sum[HEADS], o[HEADS][D / 32];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      ref[h] = kNoWeight;
      sum[h] = 0.f;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) o[h][c] = 0.f;
    }
  }
};
// Weights of a unit's keys (this lane's: s) into shared memory as [key][head].
template <int D, int HEADS>
__device__ __forceinline__ void weigh32(Running32<D, HEADS>& R, float (&s)[HEADS], int valid, float scale2, float* sp, int lane) {
#pragma unroll
  for (int h = 0; h < HEADS; ++h) {
    s[h] = lane < valid ? s[h] * scale2 : -CUDART_INF_F;
    float top = s[h];
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
    if (top > R.ref[h] + kRefSlack) {                // (the whole warp has the same values)
      const float f = exp2f(R.ref[h] - top);
      R.ref[h] = top;
      R.sum[h] *= f;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) R.o[h][c] *= f;
    }
    const float p = exp2f(s[h] - R.ref[h]);
    R.sum[h] += p;                                   // of this lane's keys
    sp[lane * HEADS + h] = p;
  }
  __syncwarp();
}
// v: this lane's channels of key `j`.
template <int D, int HEADS>
__device__ __forceinline__ void add_row(Running32<D, HEADS>& R, const float* sp, int j, const float (&v)[D / 32]) {
#pragma unroll
  for (int h = 0; h < HEADS; h += 4) {
    const float4 p = *reinterpret_cast<const float4*>(sp + j * HEADS + h);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      R.o[h][c] = fmaf(p.x, v[c], R.o[h][c]);
      R.o[h + 1][c] = fmaf(p.y, v[c], R.o[h + 1][c]);
      R.o[h + 2][c] = fmaf(p.z, v[c], R.o[h + 2][c]);
      R.o[h + 3][c] = fmaf(p.w, v[c], R.o[h + 3][c]);
    }
  }
}
// ROWS rows in fp32; qs: queries [head][channel].
template <int D, int HEADS, int ROWS>
__device__ __forceinline__ void dense32_unit(Running32<D, HEADS>& R, const float* qs, const uint8_t* k, const uint8_t* v, int valid, float scale2,
                                             float* sp, int lane) {
  const int row = min(lane, ROWS - 1);
  float s[HEADS] = {};
#pragma unroll 4
  for (int c = 0; c < D / 4; ++c) {
    const float4 x = *reinterpret_cast<const float4*>(k + row * D * 4 + ((c ^ (row & 7)) << 4));
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      const float4 q = *reinterpret_cast<const float4*>(qs + h * D + 4 * c);
      s[h] = fmaf(q.x, x.x, fmaf(q.y, x.y, fmaf(q.z, x.z, fmaf(q.w, x.w, s[h]))));
    }
  }
  weigh32<D, HEADS>(R, s, valid, scale2, sp, lane);
#pragma unroll 4
  for (int j = 0; j < min(valid, ROWS); ++j) {
    float x[D / 32];
    if constexpr (D == 128) {
      const float4 y = *reinterpret_cast<const float4*>(v + j * 512 + ((lane ^ (j & 7)) << 4));
      x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w;
    } else {
      const float2 y = *reinterpret_cast<const float2*>(v + j * 256 + (((lane >> 1) ^ (j & 7)) << 4) + (lane & 1) * 8);
      x[0] = y.x; x[1] = y.y;
    }
    add_row<D, HEADS>(R, sp, j, x);
  }
  __syncwarp();
}
// The nibble at bit 4 i less 8, in fp32: 16 + code by the mantissa's upper four bits, and an exact difference.  (With 16 + code in the
// products and 16 off at the end the outputs of a few hundred rows were 9e-7 from 64 bits; plain fp32: 2e-7.)
__device__ __forceinline__ float code32(uint32_t w, int i) {
  return __uint_as_float(((4 * i < 19 ? w << (19 - 4 * i) : w >> (4 * i - 19)) & 0x00780000u) | 0x41800000u) - 24.f;
}
// 32 rows in 4 bits, in the layout of load_int4; q: this lane's channels of the queries, qs: room for them times the unit's scales.
template <int D, int GROUP, int HEADS>
__device__ __forceinline__ void int4_unit32(Running32<D, HEADS>& R, const float (&q)[HEADS][D / 32], float* qs, const uint8_t* st, int valid,
                                            float scale2, float* sp, int lane) {
  using C = RowsCfg<float, D, GROUP>;
  constexpr int NG = C::NG, CL = D / 32;
  const uint8_t *kc = st, *vc = st + C::K_BYTES;
  const float *ks = (const float*)(st + 2 * C::K_BYTES), *kz = ks + D, *vs = kz + D, *vz = vs + C::UNIT * NG;
  const int piece = lane * CL / 4, at = ((piece & ~7) | ((piece ^ (piece >> 3)) & 7)) * 4 + (lane * CL & 3);
  float s[HEADS];
#pragma unroll
  for (int h = 0; h < HEADS; ++h) {
    s[h] = 0.f;
#pragma unroll
    for (int c = 0; c < CL; ++c) {
      const float sc = ks[at + c];
      qs[h * D + lane * CL + c] = q[h][c] * sc;
      s[h] = fmaf(q[h][c], fmaf(8.f, sc, kz[at + c]), s[h]);
    }
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) s[h] += __shfl_xor_sync(0xffffffffu, s[h], x);
  }
  __syncwarp();
#pragma unroll
  for (int p = 0; p < D / 32; ++p) {                 // 32 channels of this lane's key
    const uint4 w4 = *reinterpret_cast<const uint4*>(kc + lane * (D / 2) + ((D == 128 ? p ^ ((lane >> 1) & 3) : p) << 4));
    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = code32(w[e], i);
#pragma unroll
      for (int h = 0; h < HEADS; ++h) {
        const float4 a = *reinterpret_cast<const float4*>(qs + h * D + 32 * p + 8 * e), b = *reinterpret_cast<const float4*>(qs + h * D + 32 * p + 8 * e + 4);
        s[h] = fmaf(a.x, x[0], fmaf(a.y, x[1], fmaf(a.z, x[2], fmaf(a.w, x[3], s[h]))));
        s[h] = fmaf(b.x, x[4], fmaf(b.y, x[5], fmaf(b.z, x[6], fmaf(b.w, x[7], s[h]))));
      }
    }
  }
  weigh32<D, HEADS>(R, s, valid, scale2, sp, lane);
  const int g = lane * CL / GROUP;
#pragma unroll 4
  for (int j = 0; j < valid; ++j) {
    const float sc = vs[j * NG + g], ze = fmaf(8.f, sc, vz[j * NG + g]);
    float x[CL];
    const int byte = lane * CL / 2, from = j * (D / 2) + ((D == 128 ? (byte >> 4) ^ ((j >> 1) & 3) : byte >> 4) << 4) + (byte & 15);
    const uint32_t w = CL == 4 ? *reinterpret_cast<const uint16_t*>(vc + from) : vc[from];
#pragma unroll
    for (int c = 0; c < CL; ++c) x[c] = fmaf(code32(w, c), sc, ze);
    add_row<D, HEADS>(R, sp, j, x);
  }
  __syncwarp();
}

// ------------------------------------------------------------------ the kernel
// Results of the warps that had units of a pair: warp w's at of + w * RESULT.
struct Entry {
  const float* of;
  int r, g, flags;                               // flags: how many warps, << 8 the first, << 16 the whole pair, << 17 it begins here
};
template <typename T, int D, int GROUP, bool kTwo, int W, int ST>
__global__ void __launch_bounds__(W * 32, 1) attend_units(const RowsParams P) {
  using C = RowsCfg<T, D, GROUP>;
  using M = RowsSmem<T, D, GROUP, kTwo, W, ST>;
  constexpr int HEADS = M::HEADS, NG = C::NG, PK = M::PK;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* ring = smem_raw;
  float* weights = (float*)(smem_raw + M::RING);
  Cursor<T, D, GROUP>* cursors = (Cursor<T, D, GROUP>*)(smem_raw + M::RING + M::WEIGHTS);
  float* results = (float*)(smem_raw + M::RING + M::WEIGHTS + M::CURSORS);       // [place][warp][RESULT]
  int4* entries = (int4*)(results + M::PLACES * W * M::RESULT);                 // per place: r, g, flags of an Entry
  int *arrived = (int*)(entries + 2), *merged = arrived + 2;                     // per place: how many warps and, << 8, of how many
  const CacheParams& c = P.c;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, G = c.Hq / c.Hkv;
  if (threadIdx.x < 4) arrived[threadIdx.x] = 0;
  __syncthreads();
  after_previous();                                  // (merge_shares may take its places now)

  // --- this CTA's units, and the pair of the first
  Requests<C::UNIT, C::TAIL> Q;
  Q.read_all(c, P.n_req, lane, [](int) {});
  const int total = Q.all * c.Hkv, per = per_cta(total, gridDim.x);
  const int u0 = (int)min((int64_t)total, (int64_t)blockIdx.x * per), u1 = min(u0 + per, total);
  if (u0 >= u1) return;
  Cursor<T, D, GROUP> work;
  work.open(c, P.n_req, Q, u0, lane);
  // the place of the copies, which run ahead, lies in shared memory: it is read once per unit, registers are short
  Cursor<T, D, GROUP>& load = cursors[warp];
  if (lane == 0) load = work;
  __syncwarp();

  uint8_t* my_ring = ring + (size_t)warp * ST * C::STAGE;
  auto issue = [&](int k) {                          // copies of this warp's k-th unit
    const int u = u0 + warp + k * W;
    if (u < u1) {
      if (u - load.start >= load.units) {
        Cursor<T, D, GROUP> to = load;
        to.seek(c, P.n_req, u);
        __syncwarp();
        if (lane == 0) load = to;
        __syncwarp();
      }
      const int packed = (int)((load.len.n + C::UNIT - 1) / C::UNIT), at = u - load.start;
      uint8_t* st = my_ring + (size_t)(k % ST) * C::STAGE;
      if (at < packed) {
        const int valid = (int)min((int64_t)C::UNIT, load.len.n - (int64_t)at * C::UNIT);
        const int64_t row = load.len.first + load.g * load.len.n + (int64_t)at * C::UNIT;
        if constexpr (C::INT4) {
          load_int4<D, GROUP>(smem_addr(st), c, row, load.len.kgroup + load.g * ((load.len.n + GROUP - 1) / GROUP) + (int64_t)at * C::UNIT / GROUP,
                              valid, lane);
        } else {
          load_dense<T, D, C::UNIT>(smem_addr(st), (const T*)c.k + row * D, valid, lane);
          load_dense<T, D, C::UNIT>(smem_addr(st) + C::K_BYTES, (const T*)c.v + row * D, valid, lane);
        }
      } else {
        const int t0 = (at - packed) * C::TAIL, valid = min(C::TAIL, load.len.tail - t0);
        const int64_t row = ((int64_t)load.r * c.Hkv + load.g) * c.tail_cap + t0;
        load_dense<T, D, C::TAIL>(smem_addr(st), (const T*)c.k_tail + row * D, valid, lane);
        load_dense<T, D, C::TAIL>(smem_addr(st) + C::TAIL * D * (int)sizeof(T), (const T*)c.v_tail + row * D, valid, lane);
      }
    }
    copy_commit();
  };
#pragma unroll
  for (int k = 0; k < ST - 1; ++k) issue(k);

  const int n = lane >> 2, j = lane & 3, head = kTwo ? n & 3 : n;
  float* sp = weights + warp * HEADS * PK;
  float* qs = weights + W * HEADS * PK + warp * HEADS * D;                       // (fp32: queries)
  // Puts the results of a pair's warps together, in their order.
  auto merge = [&](const Entry& e) {
    const float* of = e.of;
    const bool whole = e.flags >> 16 & 1;
    const int64_t share = (int64_t)blockIdx.x * 2 + (e.flags >> 17 & 1), at = (int64_t)e.r * c.Hq + e.g * G;
    // a lane per warp and head: the warp's factor to the head's largest reference, that and the head's sum; they go where the weights
    // were.  (Short loops: code that runs once per pair is not in the instruction cache.)
    constexpr int PW = W <= 4 ? 4 : W <= 8 ? 8 : 16, HP = 32 / PW;
    static_assert(HEADS * (PW + 2) <= HEADS * PK, "room");
    float2* of_head = reinterpret_cast<float2*>(sp + HEADS * PW);
    const int w0 = lane % PW;
    const bool has = w0 < W && (w0 + W - (e.flags >> 8 & 255)) % W < (e.flags & 255);
    const uint32_t live = __ballot_sync(0xffffffffu, has);
#pragma unroll 1
    for (int h = lane / PW; h < (HEADS > HP ? HEADS : HP); h += HP) {            // (whole warps)
      const float2 t = has && h < G ? *reinterpret_cast<const float2*>(of + w0 * M::RESULT + M::STATS + 2 * h) : make_float2(kNoWeight, 0.f);
      float top = t.x;
#pragma unroll
      for (int y = PW / 2; y > 0; y >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, y));
      const float f = ex2a(t.x - top);
      float sum = t.y * f;
#pragma unroll
      for (int y = PW / 2; y > 0; y >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, y);
      if (h < HEADS) {
        sp[h * PW + w0] = f;
        if (w0 == 0) of_head[h] = make_float2(top, sum);
      }
    }
    __syncwarp();
    constexpr int CL = D / 32;                       // channels of a lane
#pragma unroll 1
    for (int h = 0; h < G; ++h) {
      // (all loads first, so that they are on their way together)
      float x[W][CL], z[W], f[PW], acc[CL] = {};
#pragma unroll
      for (int w = 0; w < W; w += 4) {
        const float4 y = *reinterpret_cast<const float4*>(sp + h * PW + w);
        f[w] = y.x; f[w + 1] = y.y; f[w + 2] = y.z; f[w + 3] = y.w;
      }
      const float2 total = of_head[h];
#pragma unroll
      for (int w = 0; w < W; ++w) {
#pragma unroll
        for (int i = 0; i < CL; ++i) x[w][i] = 0.f;
        z[w] = 0.f;
        if (live >> w & 1) {
          ld_floats(x[w], of + w * M::RESULT + h * D + lane * CL);
          if constexpr (C::INT4 && !C::F32) z[w] = of[w * M::RESULT + M::ZEROS + h * NG + lane * CL / GROUP];
        }
      }
#pragma unroll
      for (int w = 0; w < W; ++w)
#pragma unroll
        for (int i = 0; i < CL; ++i) acc[i] = fmaf(x[w][i] + z[w], f[w], acc[i]);
      if (whole) {
        const float inv = 1.f / total.y;
#pragma unroll
        for (int i = 0; i < CL; ++i) acc[i] *= inv;
        st_row((T*)c.out + (at + h) * D + lane * CL, acc);
        if (c.lse && lane == 0) c.lse[at + h] = (total.x + log2f(total.y)) * kLn2;
      } else {
        st_row(P.shares + (share * G + h) * D + lane * CL, acc);
        if (lane == 0) *reinterpret_cast<float2*>(P.shares + share_stats(gridDim.x, G, D) + (share * G + h) * 2) = total;
      }
    }
    __syncwarp();
  };
  // The results in a place, if all are there and nobody else has taken them.
  auto take = [&](int place, Entry& e) {
    int got = 0;
    if (lane == 0) got = take_full(arrived + place);
    if (!__shfl_sync(0xffffffffu, got, 0)) return false;
    __syncwarp();                                    // (a shuffle orders no memory: what lane 0 has acquired, the others read below)
    const int4 x = entries[place];
    e.r = x.x; e.g = x.y; e.flags = x.z;
    e.of = results + place * W * M::RESULT;
    return true;
  };
  auto leave = [&](int place) {
    if (lane == 0) {
      arrived[place] = 0;
      set_count(merged + place, merged[place] + 1);
    }
  };
  int k = 0, shared = 0;                             // this warp's units so far; pairs so far that several warps had
  Entry own;
  bool alone = false, late = false;                  // (alone: `own` is to be put together)
  for (int u = u0, end; u < u1; u = end) {           // pair by pair
    work.seek(c, P.n_req, u);
    end = min(work.start + work.units, u1);
    const int packed = (int)((work.len.n + C::UNIT - 1) / C::UNIT);
    // the warps that have units of it, from warp `head_warp` on in turn
    const int parts = min(W, end - u), head_warp = (u - u0) % W;
    const int place = shared % M::PLACES, before = shared / M::PLACES;
    if (parts > 1) ++shared;
    // Where its results go: by itself a warp takes the one stage of its ring that holds no unit to come, otherwise its part of a
    // place.  The first warp that finds the place's last pair complete puts that together: it is the one with the most time.
#pragma unroll 1
    for (;;) {
      Entry e;
      const bool taken = !alone && parts > 1 && before > 0 && take(place, e);
      if (!alone && !taken) break;
      if (alone) e = own;
      merge(e);
      if (taken) leave(place);
      alone = false;
    }
    if ((warp + W - head_warp) % W >= parts) continue;
    float* mine;
    auto open_place = [&]() {
      mine = parts == 1 ? (float*)(my_ring + (size_t)((k + ST - 1) % ST) * C::STAGE) : results + (place * W + warp) * M::RESULT;
      return parts == 1 || before == 0 || wait_count(merged + place, before, P.status, P.limit);
    };
    if constexpr (C::F32) {
      Running32<D, HEADS> R;
      R.clear();
      const float* q = (const float*)c.q + ((int64_t)work.r * c.Hq + work.g * G) * D;
      float qr[HEADS][D / 32];                       // this lane's channels
#pragma unroll
      for (int h = 0; h < HEADS; ++h)
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          qr[h][i] = h < G ? q[h * D + lane * (D / 32) + i] : 0.f;
          if (!C::INT4) qs[h * D + lane * (D / 32) + i] = qr[h][i];
        }
      __syncwarp();
      for (; u0 + warp + k * W < end; ++k) {
        issue(k + ST - 1);
        copy_wait<ST - 1>();
        __syncwarp();
        const int at = u0 + warp + k * W - work.start;
        uint8_t* st = my_ring + (size_t)(k % ST) * C::STAGE;
        if (at < packed) {
          const int valid = (int)min((int64_t)C::UNIT, work.len.n - (int64_t)at * C::UNIT);
          if constexpr (C::INT4) int4_unit32<D, GROUP, HEADS>(R, qr, qs, st, valid, c.scale2, sp, lane);
          else dense32_unit<D, HEADS, C::UNIT>(R, qs, st, st + C::K_BYTES, valid, c.scale2, sp, lane);
        } else {
          const int valid = min(C::TAIL, work.len.tail - (at - packed) * C::TAIL);
          if constexpr (C::INT4) {                   // (the room for the queries holds them times some unit's scales)
#pragma unroll
            for (int h = 0; h < HEADS; ++h)
#pragma unroll
              for (int i = 0; i < D / 32; ++i) qs[h * D + lane * (D / 32) + i] = qr[h][i];
            __syncwarp();
          }
          dense32_unit<D, HEADS, C::TAIL>(R, qs, st, st + C::TAIL * D * 4, valid, c.scale2, sp, lane);
        }
      }
      late = !open_place();
      if (late) break;
#pragma unroll
      for (int h = 0; h < HEADS; ++h) {
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) R.sum[h] += __shfl_xor_sync(0xffffffffu, R.sum[h], x);
        if (lane == 0) *reinterpret_cast<float2*>(mine + M::STATS + 2 * h) = make_float2(R.ref[h], R.sum[h]);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) mine[h * D + lane * (D / 32) + i] = R.o[h][i];
      }
    } else {
      Running<D, NG> R;
      R.clear();
      // the queries of this lane's column, as the products take them
      const __nv_bfloat16* q = (const __nv_bfloat16*)c.q + ((int64_t)work.r * c.Hq + work.g * G + head) * D;
      const bool live = head < G;
      uint32_t qd[C::INT4 ? 1 : D / 16][2];
      constexpr int QW = D / (kTwo ? 64 : 32);         // pieces of eight channels
      f32x2 qf[C::INT4 ? 4 * QW : 1];
      if constexpr (C::INT4) {
#pragma unroll
        for (int i = 0; i < QW; ++i) {
          const uint4 w = live ? *reinterpret_cast<const uint4*>(q + j * (D / 4) + 8 * (i + (kTwo && n >= 4 ? QW : 0))) : make_uint4(0, 0, 0, 0);
          qf[4 * i] = pack2(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u));
          qf[4 * i + 1] = pack2(__uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u));
          qf[4 * i + 2] = pack2(__uint_as_float(w.z << 16), __uint_as_float(w.z & 0xFFFF0000u));
          qf[4 * i + 3] = pack2(__uint_as_float(w.w << 16), __uint_as_float(w.w & 0xFFFF0000u));
        }
      }
      auto dense_queries = [&](uint32_t (&x)[D / 16][2]) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          x[i][0] = live ? *reinterpret_cast<const uint32_t*>(q + 16 * i + 2 * j) : 0u;
          x[i][1] = live ? *reinterpret_cast<const uint32_t*>(q + 16 * i + 2 * j + 8) : 0u;
        }
      };
      if constexpr (!C::INT4) dense_queries(qd);
      for (; u0 + warp + k * W < end; ++k) {
        issue(k + ST - 1);
        copy_wait<ST - 1>();
        __syncwarp();
        const int at = u0 + warp + k * W - work.start;
        uint8_t* st = my_ring + (size_t)(k % ST) * C::STAGE;
        if (at < packed) {
          const int valid = (int)min((int64_t)C::UNIT, work.len.n - (int64_t)at * C::UNIT);
          if constexpr (C::INT4) int4_unit<D, GROUP, kTwo, PK>(R, qf, smem_addr(st), valid, c.scale2, sp, lane);
          else dense_unit<D, NG, kTwo, 2, PK>(R, qd, smem_addr(st), smem_addr(st) + C::K_BYTES, valid, c.scale2, sp, lane);
        } else {
          const int valid = min(C::TAIL, work.len.tail - (at - packed) * C::TAIL);
          if constexpr (C::INT4) {                     // few rows: their queries are read again rather than kept
            uint32_t x[D / 16][2];
            dense_queries(x);
            dense_unit<D, NG, kTwo, 1, PK>(R, x, smem_addr(st), smem_addr(st) + C::TAIL * D * 2, valid, c.scale2, sp, lane);
          } else {
            dense_unit<D, NG, kTwo, 2, PK>(R, qd, smem_addr(st), smem_addr(st) + C::TAIL * D * 2, valid, c.scale2, sp, lane);
          }
        }
      }
      late = !open_place();
      if (late) break;
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) {
        R.sum[0] += __shfl_xor_sync(0xffffffffu, R.sum[0], x);
        R.sum[1] += __shfl_xor_sync(0xffffffffu, R.sum[1], x);
      }
      if (n == 0 && (!kTwo || j < 2)) {
        *reinterpret_cast<float4*>(mine + M::STATS + 4 * j) = make_float4(R.ref[0], R.sum[0], R.ref[1], R.sum[1]);
      }
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        // channels of the tile's rows lane / 4 and + 8
        const int ch0 = C::INT4 ? 32 * (i / 2) + 4 * n + 2 * (i & 1) : 16 * i + n, ch1 = C::INT4 ? ch0 + 1 : ch0 + 8;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = R.o[i][e];
          if (kTwo) x += __shfl_xor_sync(0xffffffffu, x, 2);
          if (!kTwo || j < 2) mine[(2 * j + (e & 1)) * D + (e >> 1 ? ch1 : ch0)] = x;
        }
      }
      if constexpr (C::INT4) {
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          float x, y;
          unpack2(R.z[i / 2], x, y);
          if (i & 1) x = y;
          x += __shfl_xor_sync(0xffffffffu, x, 1);
          x += __shfl_xor_sync(0xffffffffu, x, 2);
          if (kTwo) x += __shfl_xor_sync(0xffffffffu, x, 16);
          if (j == 0 && (!kTwo || n < 4)) mine[M::ZEROS + head * NG + i] = x;
        }
      }
    }
    own.r = work.r; own.g = work.g;
    own.flags = parts | head_warp << 8 | (work.start >= u0 && work.start + work.units <= u1) << 16 | (work.start >= u0) << 17;
    own.of = mine - warp * M::RESULT;
    __syncwarp();
    alone = parts == 1;
    if (!alone && lane == 0) {
      if (warp == head_warp) entries[place] = make_int4(own.r, own.g, own.flags, 0);
      arrive(arrived + place, warp == head_warp ? 1 + (parts << 8) : 1);
    }
  }
  copy_wait<0>();
  // What is left.  (Every warp looks at a place at least once after its last contribution to it, here or above: no result stays.)
#pragma unroll 1
  for (int place = -1; place < min(M::PLACES, shared) && !late; ++place) {
    Entry e = own;
    if (place < 0 ? !alone : !take(place, e)) continue;
    merge(e);
    if (place >= 0) leave(place);
  }
}

// Pairs that lie in several CTAs, from the shares these left: a CTA per pair where there are fewer pairs than CTAs, else one per
// boundary, for the pair that goes on from CTA blockIdx.x to the next, if it began in that CTA.  A thread sums four channels of
// every `parts`-th share; what it reads first is on its way while the shares' references are compared.  And the outputs of
// requests without any row.
constexpr int M_THREADS = 512, M_AHEAD = 6;
template <typename T, int D, int GROUP>
__global__ void __launch_bounds__(M_THREADS) merge_shares(const RowsParams P, int ctas, bool by_pair) {
  using C = RowsCfg<T, D, GROUP>;
  extern __shared__ float m_smem[];                  // [CTAs][G] factors; [M_THREADS] partial sums of four channels
  __shared__ float s_top[8], s_sum[8];
  const CacheParams& c = P.c;
  const int G = c.Hq / c.Hkv, lane = threadIdx.x & 31;
  Requests<C::UNIT, C::TAIL> Q = {};
  Q.read_all(c, P.n_req, lane, [&](int base) {
    // no rows at all: an output of zero and a log-sum-exp of -inf, which merges into nothing
    uint32_t none = __ballot_sync(0xffffffffu, base + lane < P.n_req && Q.units == 0 && (base + lane) % gridDim.x == blockIdx.x);
    for (; threadIdx.x < 32 && none; none &= none - 1) {
      const int64_t at = (int64_t)(base + __ffs(none) - 1) * c.Hq;
      for (int i = lane; i < c.Hq * D; i += 32) narrow((T*)c.out + at * D + i, 0.f);
      for (int i = lane; c.lse && i < c.Hq; i += 32) c.lse[at + i] = -CUDART_INF_F;
    }
  });
  const int total = Q.all * c.Hkv, per = per_cta(total, ctas);
  Cursor<T, D, GROUP> pair = {};
  bool mine;
  if (by_pair) {
    const int r = blockIdx.x / c.Hkv;
    int before = 0;
    for (int base = 0; base < r / 32 * 32; base += 32) {
      before += __shfl_sync(0xffffffffu, Q.upto, 31);
      Q.read(c, P.n_req, base + 32, lane);
    }
    pair.r = r; pair.g = blockIdx.x % c.Hkv;
    pair.units = __shfl_sync(0xffffffffu, Q.units, r % 32);
    pair.start = (before + __shfl_sync(0xffffffffu, Q.upto, r % 32) - pair.units) * c.Hkv + pair.g * pair.units;
    mine = pair.units > 0 && pair.start / per != (pair.start + pair.units - 1) / per;
  } else {
    const int64_t next = ((int64_t)blockIdx.x + 1) * per;
    mine = next < total;
    if (mine) {
      pair.open(c, P.n_req, Q, (int)next, lane);
      mine = pair.start < next && pair.start / per == (int)blockIdx.x;
    }
  }
  // Every CTA waits, also one with nothing to do: the end of this kernel stands for the end of the one before.  (What is read
  // up to here that one has read too, after all before it.)
  after_previous();
  if (!mine) return;
  const int64_t at = (int64_t)pair.r * c.Hq + pair.g * G;
  const int c0 = pair.start / per, n = (pair.start + pair.units - 1) / per - c0 + 1;
  // (the first CTA's share is the one at the end of its run)
  auto share = [&](int x) { return (int64_t)(2 * (c0 + x) + (x == 0 ? 1 : 0)) * G; };
  const int quads = G * D / 4, parts = M_THREADS / quads, part = threadIdx.x / quads, quad = threadIdx.x % quads;
  const int h = quad / (D / 4);
  const float4* o = reinterpret_cast<const float4*>(P.shares) + quad;
  float4 v[M_AHEAD];
#pragma unroll
  for (int u = 0; u < M_AHEAD; ++u) {
    const int x = part + u * parts;
    v[u] = part < parts && x < n ? __ldcg(o + share(x) * (D / 4)) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const float* stats = P.shares + share_stats(ctas, G, D);
  for (int w = threadIdx.x >> 5; w < G; w += M_THREADS / 32) {                   // a warp per head
    float top = -CUDART_INF_F, sum = 0.f;
    for (int x = lane; x < n; x += 32) {
      const float2 t = __ldcg(reinterpret_cast<const float2*>(stats + (share(x) + w) * 2));
      m_smem[x * G + w] = t.x;
      const float to = fmaxf(top, t.x);
      sum = fmaf(sum, top == to ? 1.f : exp2f(top - to), t.y * exp2f(t.x - to));
      top = to;
    }
    float all = top;
#pragma unroll
    for (int y = 16; y > 0; y >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, y));
    sum *= top == -CUDART_INF_F ? 1.f : exp2f(top - all);
#pragma unroll
    for (int y = 16; y > 0; y >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, y);
    for (int x = lane; x < n; x += 32) m_smem[x * G + w] = exp2f(m_smem[x * G + w] - all);
    if (lane == 0) { s_top[w] = all; s_sum[w] = sum; }
  }
  __syncthreads();
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float4& y, float f) {
    acc.x = fmaf(y.x, f, acc.x); acc.y = fmaf(y.y, f, acc.y); acc.z = fmaf(y.z, f, acc.z); acc.w = fmaf(y.w, f, acc.w);
  };
  if (part < parts) {
#pragma unroll
    for (int u = 0; u < M_AHEAD; ++u) {
      const int x = part + u * parts;
      if (x < n) add(v[u], m_smem[x * G + h]);
    }
#pragma unroll 4
    for (int x = part + M_AHEAD * parts; x < n; x += parts) add(__ldcg(o + share(x) * (D / 4)), m_smem[x * G + h]);
  }
  float4* sums = reinterpret_cast<float4*>(m_smem + (ctas * G + 3) / 4 * 4);
  sums[threadIdx.x] = acc;
  __syncthreads();
  if ((int)threadIdx.x >= quads) return;
  for (int y = 1; y < parts; ++y) add(sums[y * quads + quad], 1.f);
  const float inv = 1.f / s_sum[h];
  T* to = (T*)c.out + at * D + 4 * quad;
  if constexpr (C::F32) *reinterpret_cast<float4*>(to) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  else *reinterpret_cast<uint2*>(to) = make_uint2(bf16_pair(acc.x * inv, acc.y * inv), bf16_pair(acc.z * inv, acc.w * inv));
  if (c.lse && quad % (D / 4) == 0) c.lse[at + h] = (s_top[h] + log2f(s_sum[h])) * kLn2;
}

template <typename T, int D, int GROUP, bool kTwo, int W, int ST>
cudaError_t run_units(const cake_ctx* ctx, const RowsParams& P, cudaStream_t st) {
  using M = RowsSmem<T, D, GROUP, kTwo, W, ST>;
  static_assert(M::BYTES <= 227 * 1024, "a CTA has 227 KB of shared memory");
  const auto kernel = attend_units<T, D, GROUP, kTwo, W, ST>;
  static PerDeviceOnce once;
  if (once.need(ctx->device)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)M::BYTES);
    if (e != cudaSuccess) return e;
    once.mark(ctx->device);
  }
  const cudaError_t e = launch_early(kernel, (unsigned)ctx->n_sm, W * 32, M::BYTES, 1, st, P);
  if (e != cudaSuccess) return e;
  const bool by_pair = (int64_t)P.n_req * P.c.Hkv < ctx->n_sm;
  const size_t smem = ((size_t)ctx->n_sm * (P.c.Hq / P.c.Hkv) + 3) / 4 * 16 + M_THREADS * 16;
  return launch_early(merge_shares<T, D, GROUP>, (unsigned)(by_pair ? P.n_req * P.c.Hkv : ctx->n_sm), M_THREADS, smem, 1, st, P, ctx->n_sm,
                      by_pair);
}

template <typename T, int D, int GROUP>
cudaError_t run_rows(const cake_ctx* ctx, const RowsParams& P, cudaStream_t st) {
  // Warps and stages as shared memory and registers hold them: bf16 rows 4 x 3 stages of 8 to 16 KB (3 x 4: 1 to 17 % slower, all but
  // one request of 2048 rows; 6 x 2: 32 ragged requests 2 % faster and 14 % with 64 channels, one KV head per query head 7 % and 6 %, but
  // 256 requests of 350 rows and one of 2048, 128 channels, 3 % slower), fp32 rows 3 x 2 of up to 32 KB (2 x 3: 3 to 43 % slower),
  // 4-bit rows of 128 channels 8 x 3 of 5 to 6 KB (12 x 2: one request of 144000 rows 5 % faster, 32 ragged ones as fast, one of 4096
  // rows and 256 of 560 4 % and eight heads on one 14 % slower; 16 x 2, with 128 registers a thread, 8 % slower), of 64 channels 12 x 2
  // (8 x 3: 6 % slower).
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int W = !GROUP ? (F32 ? 3 : 4) : F32 || D == 128 ? 8 : 12, ST = (GROUP ? D == 128 && !F32 : !F32) ? 3 : 2;
  return P.c.Hq / P.c.Hkv <= 4 ? run_units<T, D, GROUP, true, W, ST>(ctx, P, st) : run_units<T, D, GROUP, false, W, ST>(ctx, P, st);
}
template <typename T>
cudaError_t run_typed(const cake_ctx* ctx, const RowsParams& P, cudaStream_t st) {
  const bool wide = ctx->cfg.head_dim == 128;
  switch (P.c.group) {
    case 0: return wide ? run_rows<T, 128, 0>(ctx, P, st) : run_rows<T, 64, 0>(ctx, P, st);
    case 32: return wide ? run_rows<T, 128, 32>(ctx, P, st) : run_rows<T, 64, 32>(ctx, P, st);
    case 64: return wide ? run_rows<T, 128, 64>(ctx, P, st) : run_rows<T, 64, 64>(ctx, P, st);
    default: return run_rows<T, 128, 128>(ctx, P, st);
  }
}

}  // namespace

int64_t rows_workspace(const cake_ctx* ctx) {
  const int64_t G = ctx->cfg.n_q_heads / ctx->cfg.n_kv_heads;
  return (int64_t)ctx->n_sm * 2 * G * (ctx->cfg.head_dim + 2) * (int64_t)sizeof(float);
}

int32_t launch_rows(const cake_ctx* ctx, int32_t n_req, const CacheParams& c, void* workspace, cudaStream_t st) {
  RowsParams P;
  P.c = c;
  P.shares = (float*)workspace;
  P.status = ctx->d_status;
  P.limit = ctx->wait_limit_cycles > 0 ? ctx->wait_limit_cycles : kSpinLimit;
  P.n_req = n_req;
  return cuda_status(ctx->cfg.dtype == CAKE_DTYPE_FP32 ? run_typed<float>(ctx, P, st) : run_typed<__nv_bfloat16>(ctx, P, st));
}

}  // namespace cake
