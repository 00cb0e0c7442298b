// Attention of one new token per request over its cached rows, bf16 queries: the rows in bf16 or in 4 bits.
#include "cache_mma.cuh"

namespace cake {
namespace {

// ------------------------------------------------------------------ bf16 and 4-bit rows on the tensor cores
// Work.  The (request, KV head) pairs of the layer are cut into units of 32 rows (the tail's rows behind the packed ones; 8 rows
// a unit in the 4-bit kernel, whose stages are smaller), and every CTA of one per SM takes the same number of consecutive
// units, whatever pairs they belong to: the device works evenly on ragged batches, and on one long request.  Lengths lie on
// the device, so each CTA adds up the units of all requests for itself.  Inside a CTA the warps take the units in turn, each
// with copies of its own units in flight (cp.async) and its own running softmax; they meet only where a pair ends.  A pair that
// lies in one CTA is finished there; of the others a CTA leaves its share in the workspace (at most one share at either end
// of its run), and merge_shares, which is already resident when the last CTA ends, puts them together.
//
// Products (mma m16n8k16).  S^T[key][col] = K Q^T and O^T[channel][col] = V^T P^T with the query heads as the 8 columns.  With
// up to four heads the columns 4 to 7 hold the same heads once more, for the second term of what is held in two bf16 terms
// (kTwo): weights, and in the 4-bit kernel queries times scales, are then exact to 2^-16.  With more heads the 4-bit kernel
// multiplies twice and the weights of the bf16 kernel are rounded to bf16.
//
// 4-bit rows.  A code c becomes the bf16 16 + c by one shift and one logical operation per pair (the mantissa's upper four
// bits); scales and zeros are never applied to a row but to the other operand: q_c s_c for the keys, p_j s_j for the values, and
//     q.k = sum_c (q_c s_c)(16 + code) + sum_c q_c (z_c - 16 s_c) ,   p.v = sum_j (p_j s_j)(16 + code) + sum_j p_j (z_j - 16 s_j) .
// Channels and keys are taken in whatever order the words bring them, the same one in both operands; a value tile's 16
// channels come from one group of 32, which has one scale per row.
constexpr float kRefSlack = 8.f;                 // powers of two a maximum may lie above the reference before all is rescaled

template <int D, int GROUP> struct RowsCfg {
  static constexpr bool INT4 = GROUP != 0;
  static constexpr int UNIT = 32, TAIL = INT4 ? 8 : 32;                          // rows of a unit
  static constexpr int NG = INT4 ? D / GROUP : 1;                                // channel groups of a row
  static constexpr int K_BYTES = INT4 ? UNIT * D / 2 : UNIT * D * 2;
  static constexpr int VS_BYTES = INT4 ? UNIT * NG * 4 : 0, KS_BYTES = INT4 ? D * 4 : 0;
  static constexpr int STAGE = 2 * (K_BYTES + VS_BYTES + KS_BYTES);
  static_assert(!INT4 || TAIL * D * 4 <= STAGE, "tail rows fit a stage");
};

struct RowsParams {
  CacheParams c;
  float* shares;                                 // [CTA][2][G][D], then [CTA][2][G][2] (reference, sum)
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
  x.n = max((int64_t)0, (c.row_off[block + 1] - x.first) / c.Hkv);
  x.kgroup = c.group_off ? c.group_off[block] : 0;
  x.tail = c.tail_cap ? (int32_t)max((int64_t)0, min((int64_t)c.tail_len[r], c.tail_cap)) : 0;
  return x;
}
template <int UNIT, int TAIL>
__device__ __forceinline__ int units_of(const Lengths& x) { return (int)((x.n + UNIT - 1) / UNIT) + (x.tail + TAIL - 1) / TAIL; }

// Sum of v over the block; every thread gets it.
__device__ __forceinline__ int block_sum(int v, int* buf) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0;
  for (int i = 0; i < (int)(blockDim.x >> 5); ++i) v += buf[i];
  return v;
}
// (Units are counted in 32 bits: 2^31 of them are 4 TB of 4-bit rows.)
__device__ __forceinline__ int per_cta(int units, int ctas) { return max(1, (units + ctas - 1) / ctas); }

// A place in the sequence of units: moves forward only.
template <int D, int GROUP>
struct Cursor {
  using C = RowsCfg<D, GROUP>;
  int r, g;
  int start, units;                              // first unit of the pair, and how many it has
  Lengths len;
  __device__ __forceinline__ void open(const CacheParams& c, int req, int first_unit) {
    r = req; g = 0; start = first_unit;
    len = lengths_of(c, r);
    units = units_of<C::UNIT, C::TAIL>(len);
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

__device__ __forceinline__ float ex2a(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <int D, int GROUP, bool kTwo, int W, int ST>
struct RowsSmem {
  using C = RowsCfg<D, GROUP>;
  static constexpr int HEADS = kTwo ? 4 : 8, PK = 36;                            // floats of a head's weights of a unit (padded)
  static constexpr size_t RING = (size_t)W * ST * C::STAGE, WEIGHTS = (size_t)W * HEADS * PK * 4, OUT = (size_t)W * HEADS * D * 4,
                          ZERO = (size_t)W * HEADS * C::NG * 4, STATS = (size_t)W * HEADS * 8;
  static constexpr size_t BYTES = RING + WEIGHTS + OUT + ZERO + STATS + 512;
};

// A warp's running softmax: reference and (this lane's part of the) sum of the two heads of its columns 2 j, 2 j + 1, outputs
// as the products leave them, and for 4-bit rows the sums of weights times zeros of the head of column lane / 4.
template <int D, int NG>
struct Running {
  float ref[2], sum[2], o[D / 16][4], z[NG];
  __device__ __forceinline__ void clear() {
    ref[0] = ref[1] = -CUDART_INF_F;
    sum[0] = sum[1] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
#pragma unroll
    for (int i = 0; i < NG; ++i) z[i] = 0.f;
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
      const int key = 16 * m + (lane >> 2) + 8 * (e >> 1);
      s[m][e] = key < valid ? s[m][e] * scale2 : -CUDART_INF_F;
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
    for (int i = 0; i < NG; ++i) R.z[i] *= col & 1 ? b : a;
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

// (16 + code) of the nibbles i and i + 4 of a word, as bf16.
template <int I> __device__ __forceinline__ uint32_t codes(uint32_t w) {
  const uint32_t x = I == 0 ? w << 3 : w >> (4 * I - 3 > 0 ? 4 * I - 3 : 0);
  return (x & 0x00780078u) | 0x41804180u;
}

// 32 rows in 4 bits.  qf: queries of the head of column lane / 4, channels of quarter lane % 4 of a row.
template <int D, int GROUP, bool kTwo, int PK>
__device__ __forceinline__ void int4_unit(Running<D, D / GROUP>& R, const float (&qf)[D / 4], const uint8_t* st, int valid, float scale2, float* sp,
                                          int lane) {
  using C = RowsCfg<D, GROUP>;
  constexpr int NG = C::NG, WORDS = D / 32;        // words of a quarter of a row
  const int n = lane >> 2, j = lane & 3;
  const bool second = n >= 4;
  const uint8_t *kc = st, *vc = st + C::K_BYTES;
  const float *ks = (const float*)(st + 2 * C::K_BYTES), *kz = ks + D, *vs = kz + D, *vz = vs + C::UNIT * NG;
  // --- keys: the queries times the scales of the unit's group, and the part that the zeros give
  uint32_t b[D / 16][2], b2[kTwo ? 1 : D / 16][2];
  float2 bias = make_float2(0.f, 0.f);
#pragma unroll
  for (int w = 0; w < WORDS; ++w) {
    float x[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int c = j * (D / 16) + 2 * w + u, at = ((c & ~7) | ((c ^ (c >> 3)) & 7)) * 4;      // 16-byte piece, see load_int4
      const float4 sc = *reinterpret_cast<const float4*>(ks + at), ze = *reinterpret_cast<const float4*>(kz + at);
      const float* q = qf + 8 * w + 4 * u;
      x[4 * u] = q[0] * sc.x; x[4 * u + 1] = q[1] * sc.y; x[4 * u + 2] = q[2] * sc.z; x[4 * u + 3] = q[3] * sc.w;
      bias.x = fmaf(q[0], fmaf(-16.f, sc.x, ze.x), bias.x);
      bias.y = fmaf(q[1], fmaf(-16.f, sc.y, ze.y), bias.y);
      bias.x = fmaf(q[2], fmaf(-16.f, sc.z, ze.z), bias.x);
      bias.y = fmaf(q[3], fmaf(-16.f, sc.w, ze.w), bias.y);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {                  // channels i and i + 4 of the word
      const float lo = bf16_floor(x[i]), hi = bf16_floor(x[i + 4]);
      if constexpr (kTwo) {
        b[2 * w + i / 2][i & 1] = bf16_pair(second ? x[i] - lo : lo, second ? x[i + 4] - hi : hi);
      } else {
        b[2 * w + i / 2][i & 1] = bf16_pair(lo, hi);
        b2[2 * w + i / 2][i & 1] = bf16_pair(x[i] - lo, x[i + 4] - hi);
      }
    }
  }
  float bi = bias.x + bias.y;
  bi += __shfl_xor_sync(0xffffffffu, bi, 1);
  bi += __shfl_xor_sync(0xffffffffu, bi, 2);
  const int c0 = kTwo ? (2 * j) & 3 : 2 * j;
  const float bias0 = __shfl_sync(0xffffffffu, bi, 4 * c0), bias1 = __shfl_sync(0xffffffffu, bi, 4 * c0 + 4);
  float s[2][4];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    s[m][0] = s[m][1] = s[m][2] = s[m][3] = 0.f;
    uint32_t a[WORDS], c[WORDS];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int row = 16 * m + n + 8 * half;
      uint32_t* to = half ? c : a;
      if constexpr (D == 128) {
        const uint4 v = *reinterpret_cast<const uint4*>(kc + row * 64 + ((j ^ ((row >> 1) & 3)) << 4));
        to[0] = v.x; to[1] = v.y; to[2] = v.z; to[3] = v.w;
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(kc + row * 32 + j * 8);
        to[0] = v.x; to[1] = v.y;
      }
    }
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      const uint32_t a0 = codes<0>(a[w]), a1 = codes<0>(c[w]), a2 = codes<1>(a[w]), a3 = codes<1>(c[w]);
      const uint32_t d0 = codes<2>(a[w]), d1 = codes<2>(c[w]), d2 = codes<3>(a[w]), d3 = codes<3>(c[w]);
      mma16816(s[m], a0, a1, a2, a3, b[2 * w][0], b[2 * w][1]);
      mma16816(s[m], d0, d1, d2, d3, b[2 * w + 1][0], b[2 * w + 1][1]);
      if constexpr (!kTwo) {
        mma16816(s[m], a0, a1, a2, a3, b2[2 * w][0], b2[2 * w][1]);
        mma16816(s[m], d0, d1, d2, d3, b2[2 * w + 1][0], b2[2 * w + 1][1]);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (kTwo) s[m][e] += __shfl_xor_sync(0xffffffffu, s[m][e], 2);             // both terms
      s[m][e] += e & 1 ? bias1 : bias0;
    }
  }
  weigh<D, NG, kTwo, 2, PK>(R, s, valid, scale2, sp, lane);
  // --- values: keys j, j + 4, j + 8, j + 12 of 16
  const float* p = sp + (kTwo ? n & 3 : n) * PK;
#pragma unroll
  for (int kstep = 0; kstep < 2; ++kstep) {
    float x[NG][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 16 * kstep + j + 4 * i;
      const float w = p[row];
      float sc[NG], ze[NG];
      if constexpr (NG == 4) {
        const float4 u = *reinterpret_cast<const float4*>(vs + row * 4), v = *reinterpret_cast<const float4*>(vz + row * 4);
        sc[0] = u.x; sc[1] = u.y; sc[2] = u.z; sc[3] = u.w;
        ze[0] = v.x; ze[1] = v.y; ze[2] = v.z; ze[3] = v.w;
      } else if constexpr (NG == 2) {
        const float2 u = *reinterpret_cast<const float2*>(vs + row * 2), v = *reinterpret_cast<const float2*>(vz + row * 2);
        sc[0] = u.x; sc[1] = u.y;
        ze[0] = v.x; ze[1] = v.y;
      } else {
        sc[0] = vs[row];
        ze[0] = vz[row];
      }
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        x[g][i] = w * sc[g];
        R.z[g] = fmaf(w, fmaf(-16.f, sc[g], ze[g]), R.z[g]);
      }
    }
    uint32_t bb[NG][2], bl[kTwo ? 1 : NG][2];
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float lo = bf16_floor(x[g][2 * u]), hi = bf16_floor(x[g][2 * u + 1]);
        if constexpr (kTwo) {
          bb[g][u] = bf16_pair(second ? x[g][2 * u] - lo : lo, second ? x[g][2 * u + 1] - hi : hi);
        } else {
          bb[g][u] = bf16_pair(lo, hi);
          bl[g][u] = bf16_pair(x[g][2 * u] - lo, x[g][2 * u + 1] - hi);
        }
      }
#pragma unroll
    for (int blk = 0; blk < D / 32; ++blk) {         // 32 channels: two bytes of this lane's per row
      uint32_t h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = 16 * kstep + j + 4 * i, piece = D == 128 ? blk ^ ((row >> 1) & 3) : blk;
        h[i] = *reinterpret_cast<const uint16_t*>(vc + row * (D / 2) + piece * 16 + 2 * n);
      }
      const uint32_t w0 = __byte_perm(h[0], h[1], 0x5410), w1 = __byte_perm(h[2], h[3], 0x5410);
      constexpr int per = NG > 0 ? (D / 32) / NG : 1;
      const int g = blk / per;
      const uint32_t x0 = codes<0>(w0), x1 = codes<1>(w0), x2 = codes<0>(w1), x3 = codes<1>(w1);
      const uint32_t y0 = codes<2>(w0), y1 = codes<3>(w0), y2 = codes<2>(w1), y3 = codes<3>(w1);
      mma16816(R.o[2 * blk], x0, x1, x2, x3, bb[g][0], bb[g][1]);
      mma16816(R.o[2 * blk + 1], y0, y1, y2, y3, bb[g][0], bb[g][1]);
      if constexpr (!kTwo) {
        mma16816(R.o[2 * blk], x0, x1, x2, x3, bl[g][0], bl[g][1]);
        mma16816(R.o[2 * blk + 1], y0, y1, y2, y3, bl[g][0], bl[g][1]);
      }
    }
  }
  __syncwarp();
}

// Copies of `rows` bf16 rows (those from `valid` on read as zeros) into shared memory, 16-byte piece c of a row at c ^ (row % 8).
template <int D>
__device__ __forceinline__ void load_dense(uint32_t dst, const __nv_bfloat16* src, int rows, int valid, int lane) {
  constexpr int CH = D / 8;
#pragma unroll 8
  for (int i = lane; i < rows * CH; i += 32) {
    const int r = i / CH, c = i % CH;
    copy_async16(dst + (uint32_t)(r * D * 2 + ((c ^ (r & 7)) << 4)), src + (r < valid ? (int64_t)r * D + c * 8 : 0), r < valid);
  }
}
// Copies of a unit of 4-bit rows: codes (128 channels: piece c of a row at c ^ (row / 2 % 4), so that neither the keys' 16-byte
// nor the values' 2-byte reads meet bank conflicts), the keys' scales and zeros of their group (piece c at c ^ (c / 8) within eight
// pieces, for the same reason), the values' scales and zeros.
template <int D, int GROUP>
__device__ __forceinline__ void load_int4(uint8_t* st, const CacheParams& c, int64_t row, int64_t kgroup, int valid, int lane) {
  using C = RowsCfg<D, GROUP>;
  constexpr int NG = C::NG, CH = D / 32;
  const uint32_t at = smem_addr(st);
  const uint8_t *k = (const uint8_t*)c.k + row * (D / 2), *v = (const uint8_t*)c.v + row * (D / 2);
#pragma unroll
  for (int i = lane; i < C::UNIT * CH; i += 32) {
    const int r = i / CH, p = i % CH;
    const uint32_t to = at + (uint32_t)(r * (D / 2) + ((D == 128 ? p ^ ((r >> 1) & 3) : p) << 4));
    const bool in = r < valid;
    copy_async16(to, k + (in ? i * 16 : 0), in);
    copy_async16(to + C::K_BYTES, v + (in ? i * 16 : 0), in);
  }
  const uint32_t ks = at + 2 * C::K_BYTES, vs = ks + 2 * C::KS_BYTES;
  if (lane < D / 4) {
    const int p = (lane & ~7) | ((lane ^ (lane >> 3)) & 7);
    copy_async16(ks + p * 16, c.k_scale + kgroup * D + lane * 4, true);
    copy_async16(ks + C::KS_BYTES + p * 16, c.k_zero + kgroup * D + lane * 4, true);
  }
  if constexpr (NG == 4) {                           // a row's scales start on a 16-byte boundary
    const bool in = lane < valid;
    const int64_t o = in ? (row + lane) * 4 : 0;
    copy_async16(vs + lane * 16, c.v_scale + o, in);
    copy_async16(vs + C::VS_BYTES + lane * 16, c.v_zero + o, in);
  } else {
#pragma unroll
    for (int i = lane; i < C::UNIT * NG; i += 32) {
      const bool in = i / NG < valid;
      const int64_t o = in ? row * NG + i : 0;
      copy_async4z(vs + i * 4, c.v_scale + o, in);
      copy_async4z(vs + C::VS_BYTES + i * 4, c.v_zero + o, in);
    }
  }
}

template <int D, int GROUP, bool kTwo, int W, int ST>
__global__ void __launch_bounds__(W * 32, 1) attend_units(const RowsParams P) {
  using C = RowsCfg<D, GROUP>;
  using M = RowsSmem<D, GROUP, kTwo, W, ST>;
  constexpr int HEADS = M::HEADS, NG = C::NG, PK = M::PK;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* ring = smem_raw;
  float* weights = (float*)(smem_raw + M::RING);
  float* m_out = (float*)(smem_raw + M::RING + M::WEIGHTS);
  float* m_zero = (float*)(smem_raw + M::RING + M::WEIGHTS + M::OUT);
  float2* m_stat = (float2*)(smem_raw + M::RING + M::WEIGHTS + M::OUT + M::ZERO);
  int* scratch = (int*)(smem_raw + M::BYTES - 512);
  const CacheParams& c = P.c;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, G = c.Hq / c.Hkv;
  // merge_shares may take its places now; it waits for the end of this kernel before it reads anything of it
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // --- this CTA's units, and the pair of the first
  int mine = 0;
  for (int r = threadIdx.x; r < P.n_req; r += W * 32) mine += units_of<C::UNIT, C::TAIL>(lengths_of(c, r));
  const int total = block_sum(mine, scratch) * c.Hkv, per = per_cta(total, gridDim.x);
  const int u0 = (int)min((int64_t)total, (int64_t)blockIdx.x * per), u1 = min(u0 + per, total);
  if (u0 >= u1) return;
  if (warp == 0) {
    int before = 0;
    for (int base = 0; base < P.n_req; base += 32) {
      const int v = base + lane < P.n_req ? units_of<C::UNIT, C::TAIL>(lengths_of(c, base + lane)) : 0;
      int inc = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += x;
      }
      const uint32_t found = __ballot_sync(0xffffffffu, (before + inc) * c.Hkv > u0);
      if (found) {
        if (lane == __ffs(found) - 1) { scratch[32] = base + lane; scratch[33] = (before + inc - v) * c.Hkv; }
        break;
      }
      before += __shfl_sync(0xffffffffu, inc, 31);
    }
  }
  __syncthreads();
  Cursor<D, GROUP> load, work;
  load.open(c, scratch[32], scratch[33]);
  load.seek(c, P.n_req, u0);
  work = load;

  uint8_t* my_ring = ring + (size_t)warp * ST * C::STAGE;
  auto issue = [&](int k) {                          // copies of this warp's k-th unit
    const int u = u0 + warp + k * W;
    if (u < u1) {
      load.seek(c, P.n_req, u);
      const int packed = (int)((load.len.n + C::UNIT - 1) / C::UNIT), at = u - load.start;
      uint8_t* st = my_ring + (size_t)(k % ST) * C::STAGE;
      if (at < packed) {
        const int valid = (int)min((int64_t)C::UNIT, load.len.n - (int64_t)at * C::UNIT);
        const int64_t row = load.len.first + load.g * load.len.n + (int64_t)at * C::UNIT;
        if constexpr (C::INT4) {
          load_int4<D, GROUP>(st, c, row, load.len.kgroup + load.g * ((load.len.n + GROUP - 1) / GROUP) + (int64_t)at * C::UNIT / GROUP,
                              valid, lane);
        } else {
          load_dense<D>(smem_addr(st), (const __nv_bfloat16*)c.k + row * D, C::UNIT, valid, lane);
          load_dense<D>(smem_addr(st) + C::K_BYTES, (const __nv_bfloat16*)c.v + row * D, C::UNIT, valid, lane);
        }
      } else {
        const int t0 = (at - packed) * C::TAIL, valid = min(C::TAIL, load.len.tail - t0);
        const int64_t row = ((int64_t)load.r * c.Hkv + load.g) * c.tail_cap + t0;
        load_dense<D>(smem_addr(st), (const __nv_bfloat16*)c.k_tail + row * D, C::TAIL, valid, lane);
        load_dense<D>(smem_addr(st) + C::TAIL * D * 2, (const __nv_bfloat16*)c.v_tail + row * D, C::TAIL, valid, lane);
      }
    }
    copy_commit();
  };
#pragma unroll
  for (int k = 0; k < ST - 1; ++k) issue(k);

  const int n = lane >> 2, j = lane & 3, head = kTwo ? n & 3 : n;
  float* sp = weights + warp * HEADS * PK;
  int k = 0;
  for (int u = u0; u < u1; ) {                   // pair by pair
    work.seek(c, P.n_req, u);
    const int end = min(work.start + work.units, u1), packed = (int)((work.len.n + C::UNIT - 1) / C::UNIT);
    Running<D, NG> R;
    R.clear();
    // the queries of this lane's column, as the products take them
    const __nv_bfloat16* q = (const __nv_bfloat16*)c.q + ((int64_t)work.r * c.Hq + work.g * G + head) * D;
    const bool live = head < G;
    uint32_t qd[D / 16][2];
    float qf[C::INT4 ? D / 4 : 1];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      qd[i][0] = live ? *reinterpret_cast<const uint32_t*>(q + 16 * i + 2 * j) : 0u;
      qd[i][1] = live ? *reinterpret_cast<const uint32_t*>(q + 16 * i + 2 * j + 8) : 0u;
    }
    if constexpr (C::INT4) {
#pragma unroll
      for (int i = 0; i < D / 4; i += 2) {
        const uint32_t w = live ? *reinterpret_cast<const uint32_t*>(q + j * (D / 4) + i) : 0u;
        qf[i] = __uint_as_float(w << 16);
        qf[i + 1] = __uint_as_float(w & 0xFFFF0000u);
      }
    }
    for (; u0 + warp + k * W < end; ++k) {
      issue(k + ST - 1);
      copy_wait<ST - 1>();
      __syncwarp();
      const int at = u0 + warp + k * W - work.start;
      uint8_t* st = my_ring + (size_t)(k % ST) * C::STAGE;
      if (at < packed) {
        const int valid = (int)min((int64_t)C::UNIT, work.len.n - (int64_t)at * C::UNIT);
        if constexpr (C::INT4) int4_unit<D, GROUP, kTwo, PK>(R, qf, st, valid, c.scale2, sp, lane);
        else dense_unit<D, NG, kTwo, 2, PK>(R, qd, smem_addr(st), smem_addr(st) + C::K_BYTES, valid, c.scale2, sp, lane);
      } else {
        const int valid = min(C::TAIL, work.len.tail - (at - packed) * C::TAIL);
        dense_unit<D, NG, kTwo, C::TAIL == 32 ? 2 : 1, PK>(R, qd, smem_addr(st), smem_addr(st) + C::TAIL * D * 2, valid, c.scale2, sp, lane);
      }
    }
    // --- the pair ends here (or this CTA's part of it): the warps' results together
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) {
      R.sum[0] += __shfl_xor_sync(0xffffffffu, R.sum[0], x);
      R.sum[1] += __shfl_xor_sync(0xffffffffu, R.sum[1], x);
    }
    if (n == 0 && (!kTwo || j < 2)) {
      m_stat[warp * HEADS + 2 * j] = make_float2(R.ref[0], R.sum[0]);
      m_stat[warp * HEADS + 2 * j + 1] = make_float2(R.ref[1], R.sum[1]);
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      // channels of the tile's rows lane / 4 and + 8
      const int ch0 = C::INT4 ? 32 * (i / 2) + 4 * n + 2 * (i & 1) : 16 * i + n, ch1 = C::INT4 ? ch0 + 1 : ch0 + 8;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = R.o[i][e];
        if (kTwo) x += __shfl_xor_sync(0xffffffffu, x, 2);
        if (!kTwo || j < 2) m_out[(warp * HEADS + 2 * j + (e & 1)) * D + (e >> 1 ? ch1 : ch0)] = x;
      }
    }
    if constexpr (C::INT4) {
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        float x = R.z[i];
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        if (j == 0 && (!kTwo || n < 4)) m_zero[(warp * HEADS + head) * NG + i] = x;
      }
    }
    __syncthreads();
    const bool whole = work.start >= u0 && work.start + work.units <= u1;
    const int64_t share = (int64_t)blockIdx.x * 2 + (work.start >= u0 ? 1 : 0);
    for (int i = threadIdx.x; i < G * D; i += W * 32) {
      const int h = i / D, ch = i % D;
      float top = -CUDART_INF_F, sum = 0.f, acc = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) top = fmaxf(top, m_stat[w * HEADS + h].x);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float2 t = m_stat[w * HEADS + h];
        if (t.y == 0.f) continue;                    // a warp without units of this pair
        const float f = exp2f(t.x - top);
        float x = m_out[(w * HEADS + h) * D + ch];
        if constexpr (C::INT4) x += m_zero[(w * HEADS + h) * NG + ch / GROUP];
        sum = fmaf(t.y, f, sum);
        acc = fmaf(x, f, acc);
      }
      if (whole) {
        const int64_t at = (int64_t)work.r * c.Hq + work.g * G + h;
        ((__nv_bfloat16*)c.out)[at * D + ch] = __float2bfloat16_rn(acc / sum);
        if (c.lse && ch == 0) c.lse[at] = (top + log2f(sum)) * kLn2;
      } else {
        P.shares[(share * G + h) * D + ch] = acc;
        if (ch == 0) {
          float* st = P.shares + share_stats(gridDim.x, G, D) + (share * G + h) * 2;
          st[0] = top;
          st[1] = sum;
        }
      }
    }
    __syncthreads();
    u = end;
  }
  copy_wait<0>();
}

// Pairs that lie in several CTAs, from the shares these left; and pairs without any row.
template <int D, int GROUP>
__global__ void __launch_bounds__(128) merge_shares(const RowsParams P, int ctas) {
  using C = RowsCfg<D, GROUP>;
  __shared__ int scratch[4];
  const CacheParams& c = P.c;
  const int g = blockIdx.x, r = blockIdx.y, G = c.Hq / c.Hkv;
  int all = 0, before = 0;
  for (int x = threadIdx.x; x < P.n_req; x += 128) {
    const int v = units_of<C::UNIT, C::TAIL>(lengths_of(c, x));
    all += v;
    before += x < r ? v : 0;
  }
  all = block_sum(all, scratch) * c.Hkv;
  before = block_sum(before, scratch) * c.Hkv;
  const int mine = units_of<C::UNIT, C::TAIL>(lengths_of(c, r)), start = before + g * mine, per = per_cta(all, ctas);
  // Every CTA waits, also one with nothing to do: the end of this kernel stands for the end of the one before.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t at = (int64_t)r * c.Hq + g * G;
  if (mine == 0) {
    for (int i = threadIdx.x; i < G * D; i += 128) ((__nv_bfloat16*)c.out)[at * D + i] = __float2bfloat16_rn(0.f);
    if (c.lse && (int)threadIdx.x < G) c.lse[at + threadIdx.x] = -CUDART_INF_F;
    return;
  }
  const int c0 = start / per, c1 = (start + mine - 1) / per;
  if (c0 == c1) return;
  const float* stats = P.shares + share_stats(ctas, G, D);
  for (int i = threadIdx.x; i < G * D / 4; i += 128) {
    const int h = i / (D / 4), ch = i % (D / 4) * 4;
    // (the first CTA's share is the one at the end of its run)
    auto share = [&](int x) { return (int64_t)(2 * x + (x == c0 ? 1 : 0)) * G + h; };
    float top = -CUDART_INF_F, sum = 0.f;
    for (int x = c0; x <= c1; ++x) top = fmaxf(top, __ldcg(stats + share(x) * 2));
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int x = c0; x <= c1; ++x) {
      const float2 t = __ldcg(reinterpret_cast<const float2*>(stats + share(x) * 2));
      const float4 o = __ldcg(reinterpret_cast<const float4*>(P.shares + share(x) * D + ch));
      const float f = exp2f(t.x - top);
      sum = fmaf(t.y, f, sum);
      acc.x = fmaf(o.x, f, acc.x); acc.y = fmaf(o.y, f, acc.y); acc.z = fmaf(o.z, f, acc.z); acc.w = fmaf(o.w, f, acc.w);
    }
    const float inv = 1.f / sum;
    uint2 w = make_uint2(bf16_pair(acc.x * inv, acc.y * inv), bf16_pair(acc.z * inv, acc.w * inv));
    *reinterpret_cast<uint2*>((__nv_bfloat16*)c.out + (at + h) * D + ch) = w;
    if (c.lse && ch == 0) c.lse[at + h] = (top + log2f(sum)) * kLn2;
  }
}

template <int D, int GROUP, bool kTwo, int W, int ST>
cudaError_t run_units(const cake_ctx* ctx, const RowsParams& P, cudaStream_t st) {
  using M = RowsSmem<D, GROUP, kTwo, W, ST>;
  static_assert(M::BYTES <= 227 * 1024, "a CTA has 227 KB of shared memory");
  const auto kernel = attend_units<D, GROUP, kTwo, W, ST>;
  static PerDeviceOnce once;
  if (once.need(ctx->device)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)M::BYTES);
    if (e != cudaSuccess) return e;
    once.mark(ctx->device);
  }
  kernel<<<(unsigned)ctx->n_sm, W * 32, M::BYTES, st>>>(P);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)P.c.Hkv, (unsigned)P.n_req, 1);
  cfg.blockDim = dim3(128, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, merge_shares<D, GROUP>, P, ctx->n_sm);
  count_launch(2);
  return e;
}

template <int D, int GROUP>
cudaError_t run_rows(const cake_ctx* ctx, const RowsParams& P, cudaStream_t st) {
  // Warps and stages as shared memory holds them: bf16 rows 4 x 3 stages of 8 to 16 KB, 4-bit rows 12 x 2 of 2 to 6 KB.
  constexpr int W = GROUP ? 12 : 4, ST = GROUP ? 2 : 3;
  return P.c.Hq / P.c.Hkv <= 4 ? run_units<D, GROUP, true, W, ST>(ctx, P, st) : run_units<D, GROUP, false, W, ST>(ctx, P, st);
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
  P.n_req = n_req;
  const bool wide = ctx->cfg.head_dim == 128;
  cudaError_t e;
  switch (c.group) {
    case 0: e = wide ? run_rows<128, 0>(ctx, P, st) : run_rows<64, 0>(ctx, P, st); break;
    case 32: e = wide ? run_rows<128, 32>(ctx, P, st) : run_rows<64, 32>(ctx, P, st); break;
    case 64: e = wide ? run_rows<128, 64>(ctx, P, st) : run_rows<64, 64>(ctx, P, st); break;
    default: e = run_rows<128, 128>(ctx, P, st); break;
  }
  return cuda_status(e);
}

}  // namespace cake
