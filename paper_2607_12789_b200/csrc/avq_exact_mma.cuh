// Exact attention: warp-level matrix products and what feeds them (not part of the ABI).
#pragma once

#include <cuda_fp16.h>

#include "avq_exact.cuh"
#include "avq_tc_common.cuh"

namespace avq {
namespace exact {

// 16-byte chunks of a row are stored at chunk ^ swizzle(row): eight neighbouring rows' chunks of one column, and four rows'
// two apart, lie in different banks.
__device__ __forceinline__ uint32_t swizzle(int r) { return ((r & 1) << 2) | (r & 2) | ((r >> 2) & 1); }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {   // from zero
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {   // from zero
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {   // an 8 x 8 matrix of 16-bit values, a pair per lane
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
  return v;
}
template <int N> __device__ __forceinline__ void lds_words(uint32_t (&w)[N], uint32_t at) {   // N = 2 or 4
  if constexpr (N == 4) {
    const uint4 v = lds128(at);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  } else {
    const uint2 v = lds64(at);
    w[0] = v.x; w[1] = v.y;
  }
}
// 128 + c of the codes at bits 4 i of both halves
__device__ __forceinline__ uint32_t codes_at(uint32_t w, int i) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(w >> (4 * i)), "r"(0x000f000fu), "r"(0x43004300u));   // (a & b) | c
  return r;
}
// c - 8 of such a pair, exactly
__device__ __forceinline__ uint32_t centred(uint32_t pair) {
  uint32_t r;
  asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(pair), "r"(0xc308c308u));   // - 136
  return r;
}
// c - 8 of the codes at bits 4 (i - i % 2) of both halves, 16 (c - 8) of those at bits 4 i (odd i), as halves, exactly
__device__ __forceinline__ uint32_t centred_codes(uint32_t w, int i) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(w >> (8 * (i >> 1))), "r"((i & 1) ? 0x00f000f0u : 0x000f000fu), "r"(0x64006400u));
  asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(r) : "r"((i & 1) ? 0x64806480u : 0x64086408u));   // 1024 and the middle
  return r;
}
// c 2^-24 of the codes at bits 4 (i - i % 2) of both halves, c 2^-20 of those at bits 4 i (odd i)
__device__ __forceinline__ uint32_t subnormal_codes(uint32_t w, int i) { return (w >> (8 * (i >> 1))) & ((i & 1) ? 0x00f000f0u : 0x000f000fu); }
__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float tf32_high(float x) { return __uint_as_float(__float_as_uint(x) & 0xffffe000u); }
// The low part of a value with the high part h, for an operand whose last 13 bits the tensor cores do not read: rounded to
// the bits that they do.  An infinity is its own high part; its low part is a number far above those of finite values, not a
// NaN.  (The product of an infinity and a low part of zero is NaN all the same, and that of the number and a factor above 340
// is an infinity of the other sign, perhaps: logits that are NaN are taken again from the operands themselves.)
__device__ __forceinline__ uint32_t tf32_low(float x, float h) { return __float_as_uint(fminf(x - h, 1e36f)) + 0x1000u; }
// The same of a weight, never zero beside a high part, so that an infinite value times it is that infinity and no NaN: 2^-30 of
// it at least, and 2^-126, which is the smallest that a weight is (smaller ones are zero).
__device__ __forceinline__ uint32_t tf32_low_weight(float p, float h) {
  return __float_as_uint(fmaxf(fmaxf(p - h, h * 9.3132257e-10f), fminf(p, 1.17549435e-38f))) + 0x1000u;
}
__device__ __forceinline__ float low_f(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high_f(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }
// Three bfloat16 parts of a pair of float32 values, which add up to them exactly (but for values near the smallest).
__device__ __forceinline__ void three_parts(float x, float y, uint32_t (&p)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    p[i] = pack_bf16(x, y);
    x -= low_f(p[i]);
    y -= high_f(p[i]);
  }
}
__device__ __forceinline__ void three_f16_parts(float x, float y, uint32_t (&p)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    p[i] = pack_f16(x, y);
    x -= __half2float(__ushort_as_half((unsigned short)p[i]));
    y -= __half2float(__ushort_as_half((unsigned short)(p[i] >> 16)));
  }
}


}  // namespace exact
}  // namespace avq
