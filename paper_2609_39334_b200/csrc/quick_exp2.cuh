// Packed fp32 pairs, and 2^(l c) of two logits at a time in fp32 with a proven bound.
#pragma once
#include "common.cuh"

namespace ss {

typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unpack2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 both(float a) { return pack2(a, a); }

// Terms relative to a power of two 2^e0 (a whole number).
// l * c = n + f with |f| <= 1/2: n from a sum whose low bits are the integer, f exactly by an FMA with the high part of c (one
// rounding to 2^-26) and one with the low part; 2^f by a polynomial of degree 6 (minimax of the relative error on |f| <=
// 0.5002, coefficients rounded: 1.6e-8); n into the exponent by an integer addition.  A term is within 1.21e-7: 1.6e-8, 2.1e-8
// from f, 2.4e-8 from the polynomial's inner roundings and 6e-8 from its last one.  Eight terms added pairwise (three roundings,
// 1.79e-7) that go to fp64 from there are within 3.2e-7 of the exact sum.  Terms below 2^(e0 - 124) count as that.
struct QuickBase {
  float low, shift;
};
__device__ __forceinline__ QuickBase quick_base(float e0, float c_hi) { return QuickBase{(e0 - 124.f) / c_hi, 12582912.f - e0}; }   // 1.5 * 2^23
__device__ __forceinline__ f32x2 quick_pair(float l0, float l1, const QuickBase& q, float c_hi, float c_lo) {
  const f32x2 l = pack2(fmaxf(l0, q.low), fmaxf(l1, q.low)), c = both(c_hi);
  const f32x2 nb = fma2(l, c, both(q.shift));                  // bits: 0x4b400000 + (n - e0)
  f32x2 f = fma2(l, c, fma2(nb, both(-1.f), both(q.shift)));
  f = fma2(l, both(c_lo), f);
  f32x2 p = fma2(f, both(0.00015353319759014994f), both(0.0013398926239460707f));
  p = fma2(p, f, both(0.009618437848985195f));
  p = fma2(p, f, both(0.055503323674201965f));
  p = fma2(p, f, both(0.24022647738456726f));
  p = fma2(p, f, both(0.6931471824645996f));
  p = fma2(p, f, both(1.f));
  float p0, p1, n0, n1;
  unpack2(p, p0, p1);
  unpack2(nb, n0, n1);
  return pack2(__int_as_float(__float_as_int(p0) + (__float_as_int(n0) << 23)), __int_as_float(__float_as_int(p1) + (__float_as_int(n1) << 23)));
}

}  // namespace ss
