// Rows of the quantised paged cache: dh whole numbers x in [-127, 127] and an exponent e, of
// one token and key head; values x 2^e.
//   e = min { e >= -126 : max |y| <= 127 2^e },  x = rint(y 2^-e)
// x has 7 bits, so that x 2^e is a bf16 number.  PQ_NAN stands for a row that is not finite, or
// reaches past 127 2^PQ_TOP: all of its values are NaN.
#pragma once

#include "common.cuh"

namespace pf {

constexpr int PQ_NAN = -128, PQ_LOW = -126, PQ_TOP = 104;

// The exponent of a row whose largest absolute value is m.  The mantissa decides whether 2^6 of
// m's own power of two are enough: up to 127 / 64.
__device__ __forceinline__ int pq_exp(float m) {
  const int u = __float_as_int(m);
  const int e = (u >> 23) - 127 - 6 + ((u & 0x7fffff) > 0x7e0000 ? 1 : 0);
  return e > PQ_TOP ? PQ_NAN : e < PQ_LOW ? PQ_LOW : e;
}
// 2^-e (PQ_NAN: 0)
__device__ __forceinline__ float pq_inverse(int e) {
  return e == PQ_NAN ? 0.f : __int_as_float((127 - e) << 23);
}

// 2^e.  Of PQ_NAN the bits of -inf come out: with pq_shift's +inf its values below are NaN.
__device__ __forceinline__ float pq_scale(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ float pq_shift(float f) { return -8388736.f * f; }  // 2^23 + 128

// Four whole numbers (a word's bytes, lowest first) as bf16 values: byte + 128 as the low bits
// of 2^23, (2^23 + byte + 128) 2^e - (2^23 + 128) 2^e in one exact FMA, upper halves.
__device__ __forceinline__ uint2 pq_values(uint32_t w, float2 f, float2 b) {
  w ^= 0x80808080u;
  auto at = [&](uint32_t sel) { return __uint_as_float(__byte_perm(w, 0x4b000000u, sel)); };
  const float2 lo = __ffma2_rn(make_float2(at(0x7440), at(0x7441)), f, b);
  const float2 hi = __ffma2_rn(make_float2(at(0x7442), at(0x7443)), f, b);
  return make_uint2(__byte_perm(__float_as_uint(lo.x), __float_as_uint(lo.y), 0x7632),
                    __byte_perm(__float_as_uint(hi.x), __float_as_uint(hi.y), 0x7632));
}

// The same times 2^-7 (PQ_DOWN), as fast as it goes: a byte + 128 with zeros above it is, as a
// bf16's bits, so many times 2^-133, whether below 2^-126 or in the binade above, and one FMA
// takes it to (byte + 128) 2^(e - 7) - 128 2^(e - 7).  The factor, 2^(126 + e), is a bf16 up to
// e = 1 (rows up to 254); 5 instructions for four values where pq_values takes 9.
constexpr int PQ_DOWN = 7;
__device__ __forceinline__ bool pq_small(int e) { return e <= 1; }
__device__ __forceinline__ uint32_t pq_factor(int e) {  // twice (PQ_NAN: NaN)
  return __byte_perm(e == PQ_NAN ? 0x7fff : (uint32_t)(e + 253) << 7, 0, 0x1010);
}
__device__ __forceinline__ uint32_t pq_offset(int e) { return __byte_perm((uint32_t)(e + 383) << 7, 0, 0x1010); }
__device__ __forceinline__ uint32_t pq_pair(uint32_t w, uint32_t sel, uint32_t f, uint32_t c) {
  uint32_t r;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(__byte_perm(w, 0, sel)), "r"(f), "r"(c));
  return r;
}
__device__ __forceinline__ uint32_t pq_twice(int e) {  // 2^e, twice (PQ_NAN: any number)
  return __byte_perm((uint32_t)(max(e, -PQ_DOWN) + 127) << 7, 0, 0x1010);
}
__device__ __forceinline__ uint2 pq_times(uint2 v, uint32_t f) {
  asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(v.x) : "r"(f));
  asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(v.y) : "r"(f));
  return v;
}
// bytes 0, 1 and 2, 3 of w ^ 0x80808080, and (pq_down_cols) bytes 0, 2 and 1, 3
__device__ __forceinline__ uint2 pq_down(uint32_t w, uint32_t f, uint32_t c) {
  w ^= 0x80808080u;
  return make_uint2(pq_pair(w, 0x4140, f, c), pq_pair(w, 0x4342, f, c));
}
__device__ __forceinline__ uint2 pq_down_cols(uint32_t w, uint32_t f, uint32_t c) {
  w ^= 0x80808080u;
  return make_uint2(pq_pair(w, 0x4240, f, c), pq_pair(w, 0x4341, f, c));
}

}  // namespace pf
