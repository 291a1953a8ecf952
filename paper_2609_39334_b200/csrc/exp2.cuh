// Powers of two for the softmax loops: the special-function unit, and a polynomial for the FMA pipe beside it.
#pragma once
#include <stdint.h>

namespace ss {
namespace umma {

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unpack2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ float clamped(float x, float least) { // to [least, 127], NaN remains
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(least));
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(127.f));
  return x;
}
// 2^x of two values on the FMA pipe: n = the nearest integer to x, 2^(x - n) by a polynomial of degree 5 (its largest relative error on
// [-1/2, 1/2] made smallest: 2.3e-7 with fp32's roundings, as the special-function unit's), n added to the exponent.  What lies outside
// [least, 127] counts as the end of it; a NaN or more than 2^126 comes out as that or as more than 2^126.  least >= -127, whose power comes
// out as 2^-149.
__device__ __forceinline__ void exp2_pair(float& a, float& b, float least) {
  const float kRound = 12582912.0f;                              // 1.5 * 2^23
  const f32x2 x = pack2(clamped(a, least), clamped(b, least)), t = add2(x, pack2(kRound, kRound)), n = add2(t, pack2(-kRound, -kRound));
  const f32x2 f = fma2(n, pack2(-1.f, -1.f), x);
  f32x2 p = pack2(0.0013276473619043827f, 0.0013276473619043827f);
  p = fma2(p, f, pack2(0.009675541892647743f, 0.009675541892647743f));
  p = fma2(p, f, pack2(0.05550713092088699f, 0.05550713092088699f));
  p = fma2(p, f, pack2(0.24022120237350464f, 0.24022120237350464f));
  p = fma2(p, f, pack2(0.6931469440460205f, 0.6931469440460205f));
  p = fma2(p, f, pack2(1.0000001192092896f, 1.0000001192092896f));
  float t0, t1, p0, p1;
  unpack2(t, t0, t1);
  unpack2(p, p0, p1);
  a = __uint_as_float((__float_as_uint(t0) << 23) + __float_as_uint(p0));
  b = __uint_as_float((__float_as_uint(t1) << 23) + __float_as_uint(p1));
}

}  // namespace umma
}  // namespace ss
