// Warp-level pieces of the cached attention: asynchronous copies, matrix fragments.
#pragma once

#include "attend.cuh"

namespace cake {

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 (4) bytes, or zeros if n is 0: nothing is read then.  The immediate offsets spare an addition per access.
template <int TO = 0, int FROM = 0>
__device__ __forceinline__ void copy_async16n(uint32_t dst, const void* src, int n) {
  asm volatile("cp.async.cg.shared.global [%0 + %3], [%1 + %4], 16, %2;" ::"r"(dst), "l"(src), "r"(n), "n"(TO), "n"(FROM) : "memory");
}
template <int TO = 0, int FROM = 0>
__device__ __forceinline__ void copy_async4n(uint32_t dst, const void* src, int n) {
  asm volatile("cp.async.ca.shared.global [%0 + %3], [%1 + %4], 4, %2;" ::"r"(dst), "l"(src), "r"(n), "n"(TO), "n"(FROM) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr) : "memory");
}
template <int OFF = 0> __device__ __forceinline__ void ld_shared(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4 + %5];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr), "n"(OFF) : "memory");
}
template <int OFF = 0> __device__ __forceinline__ void ld_shared(uint32_t (&r)[2], uint32_t addr) {
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2 + %3];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr), "n"(OFF) : "memory");
}
// Pairs of fp32 values.
template <int OFF = 0> __device__ __forceinline__ void ld_shared(unsigned long long (&r)[2], uint32_t addr) {
  asm volatile("ld.shared.v2.b64 {%0, %1}, [%2 + %3];" : "=l"(r[0]), "=l"(r[1]) : "r"(addr), "n"(OFF) : "memory");
}
template <int OFF = 0> __device__ __forceinline__ void ld_shared(unsigned long long (&r)[1], uint32_t addr) {
  asm volatile("ld.shared.b64 %0, [%1 + %2];" : "=l"(r[0]) : "r"(addr), "n"(OFF) : "memory");
}
template <int OFF = 0> __device__ __forceinline__ float ld_shared_f(uint32_t addr) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1 + %2];" : "=f"(v) : "r"(addr), "n"(OFF) : "memory");
  return v;
}
template <int OFF = 0> __device__ __forceinline__ uint32_t ld_shared_u16(uint32_t addr) {
  uint32_t v;
  asm volatile("{\n.reg .u16 t;\nld.shared.u16 t, [%1 + %2];\ncvt.u32.u16 %0, t;\n}" : "=r"(v) : "r"(addr), "n"(OFF) : "memory");
  return v;
}
// for_n<N>([&](auto i) { ... }): i is a constant in each of its N calls.
template <int I> struct Const { static constexpr int value = I; __host__ __device__ constexpr operator int() const { return I; } };
template <int N, int I = 0, typename F>
__device__ __forceinline__ void for_n(F&& f) {
  if constexpr (I < N) {
    f(Const<I>{});
    for_n<N, I + 1>(f);
  }
}
// c[16 x 8] += a[16 x 16] b[16 x 8].  Lane 4 i + j holds of a the rows i, i + 8 and columns 2 j, 2 j + 1 and those + 8; of b the
// same columns as rows, and column i; of c the rows i, i + 8 and columns 2 j, 2 j + 1.
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float bf16_floor(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }

}  // namespace cake
