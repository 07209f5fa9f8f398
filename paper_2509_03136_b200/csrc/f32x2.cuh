// Packed pairs of 32-bit floats and powers of two of them, on the special-function unit or on the FMA pipe (accumulate.cu,
// attend_many.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace gvote {

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Packed pairs of 32-bit floats.
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ float2 unpack2(uint64_t d) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(d));
  return f;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// 2^x for a pair, x <= 127, without the special-function unit: x = i + f with i the nearest integer (read off the low bits
// of x + 1.5 * 2^23 + 127, which are i + 127), 2^f by the polynomial of degree 5 with the smallest largest relative error
// on [-1/2, 1/2] (Remez exchange; 1.5e-7 with the coefficients as they are rounded here, 2.1e-7 in 32 bits).  x is taken to
// -127 at least, where the power that i gives is zero: what lies below 2^-126.5 is zero, -inf too; a NaN stays one.
__device__ __forceinline__ uint64_t exp2_poly2(uint64_t x2) {
  float2 x = unpack2(x2);
  x2 = pack2(max_nan(x.x, -127.f), max_nan(x.y, -127.f));
  const uint64_t r2 = add2(x2, pack2(12583039.f, 12583039.f));
  const uint64_t i2 = add2(r2, pack2(-12583039.f, -12583039.f));
  const uint64_t f2 = fma2(i2, pack2(-1.f, -1.f), x2);
  uint64_t p = pack2(1.3276472e-3f, 1.3276472e-3f);
  p = fma2(p, f2, pack2(9.6755410e-3f, 9.6755410e-3f));
  p = fma2(p, f2, pack2(5.5507131e-2f, 5.5507131e-2f));
  p = fma2(p, f2, pack2(2.4022120e-1f, 2.4022120e-1f));
  p = fma2(p, f2, pack2(6.9314694e-1f, 6.9314694e-1f));
  p = fma2(p, f2, pack2(1.0000001f, 1.0000001f));
  const float2 r = unpack2(r2);
  return mul2(p, pack2(__uint_as_float(__float_as_uint(r.x) << 23), __uint_as_float(__float_as_uint(r.y) << 23)));
}
// Of every eight consecutive pairs j, kShare spread evenly go to the FMA pipe.
template <int kShare>
__device__ __forceinline__ uint64_t exp2_pair(int j, uint64_t x2) {
  if (((j + 1) * kShare) / 8 != (j * kShare) / 8) return exp2_poly2(x2);
  const float2 x = unpack2(x2);
  return pack2(exp2_fast(x.x), exp2_fast(x.y));
}

}  // namespace gvote
