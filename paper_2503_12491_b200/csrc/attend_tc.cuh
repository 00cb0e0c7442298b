// Tensor-memory access and operands of the prompt kernels.
#pragma once

#include "attend.cuh"
#include "tc_ptx.cuh"

namespace cake {

constexpr int TILE = 128;
constexpr int SLAB = TILE * 128;                 // bytes of 64 bf16 channels of a tile of 128 rows
constexpr float kRefSlack = 8.f;                 // powers of two that a row's maximum may lie above its reference
// Weights are 2^(s * scale - ref) in one rounding, and the reference is the rounded product of the largest s: a difference of up to half
// of a step of the reference, which cancels in output and log-sum-exp as long as it is a power of two that fp32 has.  From 2^30 on,
// where a step is 128, both terms are multiplied with this factor, which keeps the difference below 32.  (Other logits, a step of s
// away, stay at least 32 below the largest, weights of 2^-32 in place of less.)
__device__ __forceinline__ float coarse_factor(float ref) {
  const int k = max(0, (int)(__float_as_uint(ref) >> 23 & 255u) - (127 + 29));
  return __uint_as_float((uint32_t)(127 - k) << 23);
}
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2) {
  asm volatile("{\n.reg .pred e;\nelect.sync _|e, 0xffffffff;\n"
               "@e cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n}"
               ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
// D = A B + (kAcc ? D : 0) with A in tensor memory (16 bf16 of K per step: 8 columns) and B in shared memory, K rows of 64
// channels in the 128-byte swizzle: the operand's N runs along the row, and beyond 64 channels in the next slab
// (leading-dimension offset); 8 rows of K are 1024 bytes (stride offset).
__device__ __forceinline__ void umma_ts(uint32_t tmem_d, uint32_t tmem_a, uint32_t b_lo, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n.reg .pred p, e;\n.reg .b64 db;\nsetp.ne.b32 p, %4, 0;\nelect.sync _|e, 0xffffffff;\nmov.b64 db, {%2, %5};\n"
               "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n}"
               ::"r"(tmem_d), "r"(tmem_a), "r"(b_lo), "r"(idesc), "r"(acc), "r"(kDescHi) : "memory");
}
#define R32(r) "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), \
  "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), \
  "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
#define L32 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, " \
  "%28, %29, %30, %31}"
// 32 fp32 columns of this thread's TMEM lane (valid after tmem_wait_ld, which must come before any use).
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 " L32 ", [%32];" : R32(r) : "r"(addr));
}
#define RW32(r) "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), \
  "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), \
  "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
// The registers pass through the statement, so that none of their uses is scheduled before it.
__device__ __forceinline__ void tmem_wait_ld32(uint32_t* r) { asm volatile("tcgen05.wait::ld.sync.aligned;" : RW32(r) : : "memory"); }
__device__ __forceinline__ void pin32(uint32_t* r) { asm volatile("" : RW32(r)); }
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
               "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
               "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
               "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

// 2^x of two values on the FMA pipe, x <= 100: x = n + f with n an integer and |f| <= 1/2, 2^f by a polynomial of degree 5, times
// 2^n put together from its bits: zero from n = -127 down.  A NaN stays one.  The polynomial is 1 at f = 0 and has no error on
// average over f; among those it is the one with the least largest error, 1.2e-7 relative (1.8e-7 with the roundings of fp32), fitted
// with one coefficient after the other rounded to fp32.  (A free fit, 0.75e-7, has a first coefficient that rounds to 1 + 2^-23:
// every weight was 5e-8 too large.)
__device__ __forceinline__ f32x2 splat(float x) { return pack2(x, x); }
__device__ __forceinline__ void exp2_poly(f32x2 x, float& a, float& b) {
  float x0, x1;
  unpack2(x, x0, x1);
  x = pack2(max_or_nan(x0, -127.f), max_or_nan(x1, -127.f));
  const f32x2 r = add2(x, splat(12582912.f));                     // 1.5 * 2^23: the integer lands in the low bits
  const f32x2 f = fma2(add2(r, splat(-12582912.f)), splat(-1.f), x);
  f32x2 p = fma2(f, splat(1.3254279037937522e-3f), splat(9.668318554759026e-3f));
  p = fma2(p, f, splat(5.550743639469147e-2f));
  p = fma2(p, f, splat(2.4022312462329865e-1f));
  p = fma2(p, f, splat(6.931470036506653e-1f));
  p = fma2(p, f, splat(1.f));
  float r0, r1;
  unpack2(r, r0, r1);
  unpack2(mul2(p, pack2(__uint_as_float((__float_as_uint(r0) << 23) + 0x3F800000u),
                        __uint_as_float((__float_as_uint(r1) << 23) + 0x3F800000u))), a, b);
}

// This thread's key against 32 queries: the sum of its weights.  kEdge: queries before the key, or beyond the prompt, do not
// count (whatever their logits are).
template <bool kEdge, bool kPoly>
__device__ __forceinline__ void weigh32(const uint32_t (&r)[32], const float* nl, f32x2 sc, int first, int past, f32x2& acc0, f32x2& acc1) {
#pragma unroll
  for (int c = 0; c < 32; c += 8) {
    float e[8];
    const float4 n0 = *reinterpret_cast<const float4*>(nl + c), n1 = *reinterpret_cast<const float4*>(nl + c + 4);
    const float n[8] = {n0.x, n0.y, n0.z, n0.w, n1.x, n1.y, n1.z, n1.w};
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const f32x2 x = fma2(pack2(__uint_as_float(r[c + i]), __uint_as_float(r[c + i + 1])), sc, pack2(n[i], n[i + 1]));
      if (kPoly && i == 6) {                     // a quarter of the exponentials on the FMA pipe
        exp2_poly(x, e[i], e[i + 1]);
      } else {
        float a, b;
        unpack2(x, a, b);
        e[i] = ex2(a);
        e[i + 1] = ex2(b);
      }
    }
    if constexpr (kEdge) {
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = c + i >= first && c + i < past ? e[i] : 0.f;
    }
    acc0 = add2(acc0, pack2(e[0], e[1]));
    acc1 = add2(acc1, pack2(e[2], e[3]));
    acc0 = add2(acc0, pack2(e[4], e[5]));
    acc1 = add2(acc1, pack2(e[6], e[7]));
  }
}

}  // namespace cake
