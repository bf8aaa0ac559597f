// Values in 8 bits with a scale: what the kernels that make them share.
#pragma once

#include "rows.cuh"

namespace xconv {

constexpr float Q_LEAST = 7.888609052210118e-31f;          // 2^-100

// The largest magnitude, NaN above all.
__device__ __forceinline__ float most_of(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float magnitude(const float (&y)[8]) {
  float m[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) m[e] = most_of(fabsf(y[e]), fabsf(y[e + 4]));
  return most_of(most_of(m[0], m[1]), most_of(m[2], m[3]));
}
__device__ __forceinline__ float reciprocal(float a) {
  float r;
  asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(a));
  return r;
}
// rstd as a power of two and a factor between 1 and 2.  Values are u = h (power w) until the row's or the group's largest magnitude is known, so that nothing is rounded but the product
// h w (of 16-bit activations and weights it mostly is exact); the factor goes into the scale alone.  (Of NaN the power is infinity, which makes the scale NaN.)
struct Root { float power, factor; };
__device__ __forceinline__ Root root_of(float rstd) {
  const uint32_t b = __float_as_uint(rstd);
  return {__uint_as_float(b & 0x7f800000u), __uint_as_float((b & 0x007fffffu) | 0x3f800000u)};
}
// The scale of values u up to a, the nearest float but one (NaN where a is not finite), and what they are multiplied by, M / a, as a sum of two floats: with the second one the product is rounded
// once, so that a value between two codes, at the same distance from both, is still there when it is rounded to 8 bits, and goes to the even one.  (By one float some 3 of
// 10^5 values of 16-bit activations and weights went to the odd code.)
struct Scale { float scale, inv, low; };
__device__ __forceinline__ Scale q_scale(float a, const Root& root, int q) {
  const float M = q == XCONV_Q_E4M3 ? 448.f : 127.f, most = most_of(a * root.factor, Q_LEAST), from = most_of(a, Q_LEAST * reciprocal(root.factor)), r = reciprocal(from), inv = M * r;
  return {fmaf(most, q == XCONV_Q_E4M3 ? 1.f / 448.f : 1.f / 127.f, 0.f * most), inv, fmaf(-inv, from, M) * r};
}
// Two values at a time: an instruction for both.
__device__ __forceinline__ float2 q_of(float u0, float u1, const Scale& f) {
  float2 v;
  asm("{.reg .b64 u, i, l, v;\n\tmov.b64 u, {%2, %3};\n\tmov.b64 i, {%4, %4};\n\tmov.b64 l, {%5, %5};\n\tmul.rn.f32x2 v, u, l;\n\tfma.rn.f32x2 v, u, i, v;\n\tmov.b64 {%0, %1}, v;}"
      : "=f"(v.x), "=f"(v.y) : "f"(u0), "f"(u1), "f"(f.inv), "f"(f.low));
  return v;
}
__device__ __forceinline__ uint32_t e4m3x2(float2 v) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(v.y), "f"(v.x));
  return r;
}
// The nearest whole numbers of two values, at most 127 (and a little) in magnitude, in the low bytes: added to 3 * 2^22, where a float's last place is one.
__device__ __forceinline__ uint32_t int8x2(float2 v) { return __byte_perm(__float_as_uint(v.x + 12582912.f), __float_as_uint(v.y + 12582912.f), 0x0040); }
// (over the threads of a row, as row_sum)
__device__ __forceinline__ float row_most(float v, int group, float* buf) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < group) v = most_of(v, __shfl_xor_sync(0xffffffffu, v, o));
  if (group <= 32) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = lane < (group >> 5) ? buf[lane] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = most_of(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

}  // namespace xconv
