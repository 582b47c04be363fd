// The 4-bit form of K and V rows: what the kernels that write and read it share.
//
// Sixteen neighbouring columns of a row share a scale s, an 8-bit number of 1 sign, 4 exponent and 3 mantissa bits (e4m3, never negative); a value is
// code * s * 2^e with whole codes from -7 to 7 and e the pool's.  Code and scale have 3 and 4 significant bits, their product 7: it is a bf16 and an
// fp16 number exactly, so what attention multiplies is what the cache stands for, not a rounding of it.  Whole-number codes and not 4-bit
// floating-point ones: of sixteen normally distributed values they keep 21.3 dB instead of 20.4.
//
// A page of one head is one block: codes of K [64][d / 2], codes of V, scales of K [64][d / 16], scales of V (9216 bytes for d = 128), so one copy
// without a tensor map brings it.  A 4-byte word holds eight columns' codes + 8: even columns in the low half's four fields, odd ones in the high half's,
// so that a shift and a mask give a pair of neighbours in two 16-bit halves.
#pragma once
#include <cuda_fp16.h>

#include "paged.h"

namespace heatkv {

__host__ __device__ constexpr int block4_bytes(int d) { return PAGE * (d + d / 8); }

template <int D>
struct Block4 {
  static constexpr int ROW = D / 2, SCALES = D / 16;             // bytes of a row's codes and scales
  static constexpr int K = 0, V = PAGE * ROW, KS = 2 * PAGE * ROW, VS = KS + PAGE * SCALES, BYTES = VS + PAGE * SCALES;
  static_assert(BYTES == block4_bytes(D), "blocks are dense");
};

// Constants that take the fields of a word to values, two fields at a time, in fp16: the bits of 1024 with a field c at the mantissa's low end are
// the number 1024 + c, with the field four bits up 1024 + 16 c, so one multiply-add each gives (c - 8) s'.  s' = s / 256: then s' is the
// scale's byte, shifted by 7, and every product here is exact (1032 s' and 72 s' have 11 and 8 significant bits, nothing exceeds 1806, the
// smallest step is 2^-21).
struct Steps4 {
  __half2 lo, hi, lo8, hi8;                                      // s', s' / 16, -1032 s', -72 s'
  // two scale bytes, in bits 0..7 and 16..23
  __device__ __forceinline__ explicit Steps4(uint32_t bytes) {
    const uint32_t s = bytes << 7;
    lo = *reinterpret_cast<const __half2*>(&s);
    hi = __hmul2(lo, __float2half2_rn(1.f / 16.f));
    lo8 = __hmul2(lo, __float2half2_rn(-1032.f));
    hi8 = __hmul2(lo, __float2half2_rn(-72.f));
  }
};
__device__ __forceinline__ uint32_t fields_lo(uint32_t x) {      // (x & 0x000f000f) | 0x64006400
  uint32_t r;
  asm("lop3.b32 %0, %1, 0x000f000f, 0x64006400, 0xea;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t fields_hi(uint32_t x) {
  uint32_t r;
  asm("lop3.b32 %0, %1, 0x00f000f0, 0x64006400, 0xea;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t as_word(__half2 x) { return *reinterpret_cast<uint32_t*>(&x); }
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<__half2*>(&x); }
// the pairs of fields 0..3 of a word's halves
__device__ __forceinline__ void values4(uint32_t w, const Steps4& s, uint32_t (&out)[4]) {
  const uint32_t up = w >> 8;
  out[0] = as_word(__hfma2(as_half2(fields_lo(w)), s.lo, s.lo8));
  out[1] = as_word(__hfma2(as_half2(fields_hi(w)), s.hi, s.hi8));
  out[2] = as_word(__hfma2(as_half2(fields_lo(up)), s.lo, s.lo8));
  out[3] = as_word(__hfma2(as_half2(fields_hi(up)), s.hi, s.hi8));
}
// The same with every second pair 16 times as large, which who takes them puts right elsewhere: 16 (c - 8) s' = (1024 + 16 c) s' - 1152 s', exact like the
// others, and a constant fewer for every scale.
struct Steps4Uneven {
  __half2 s, lo8, hi8;                                           // s', -1032 s', -1152 s'
  __device__ __forceinline__ explicit Steps4Uneven(uint32_t bytes) {
    s = as_half2(bytes << 7);
    lo8 = __hmul2(s, __float2half2_rn(-1032.f));
    hi8 = __hmul2(s, __float2half2_rn(-1152.f));
  }
};
__device__ __forceinline__ void values4(uint32_t w, const Steps4Uneven& s, uint32_t (&out)[4]) {
  const uint32_t up = w >> 8;
  out[0] = as_word(__hfma2(as_half2(fields_lo(w)), s.s, s.lo8));
  out[1] = as_word(__hfma2(as_half2(fields_hi(w)), s.s, s.hi8));
  out[2] = as_word(__hfma2(as_half2(fields_lo(up)), s.s, s.lo8));
  out[3] = as_word(__hfma2(as_half2(fields_hi(up)), s.s, s.hi8));
}
// The same in bf16: 128 + c is a number of 8 bits, of a half's fields one at a time, and (c - 8) s' with s' = s / 256 is exact as 136 s' = 17 * 8 s' has 8
// bits.  The scale's byte, shifted by 4, is s' 2^-112.
struct Steps4Bf16 {
  __nv_bfloat162 s, s8;                                          // s', -136 s'
  __device__ __forceinline__ explicit Steps4Bf16(uint32_t bytes) {
    const uint32_t x = bytes << 4;
    s = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&x), __float2bfloat162_rn(5.192296858534828e33f));      // 2^112
    s8 = __hmul2(s, __float2bfloat162_rn(-136.f));
  }
};
__device__ __forceinline__ void values4(uint32_t w, const Steps4Bf16& s, uint32_t (&out)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t x;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(x) : "r"(w >> (4 * i)));
    const __nv_bfloat162 y = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&x), s.s, s.s8);
    out[i] = *reinterpret_cast<const uint32_t*>(&y);
  }
}
// A copy of contiguous bytes (a multiple of 16) from global to shared memory, counted by a barrier there.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
constexpr float VALUES4_UNIT = 256.f;                            // what values4's numbers are to be multiplied by

}  // namespace heatkv
