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
// The scale of values up to a, and what they are multiplied by: the nearest floats but one, by a reciprocal within an ulp.  (NaN where a is not finite.)
struct Scale { float scale, inv; };
__device__ __forceinline__ Scale q_scale(float a, int q) {
  const float M = q == XCONV_Q_E4M3 ? 448.f : 127.f, least = a < Q_LEAST ? Q_LEAST : a;
  float r;
  asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(least));
  return {fmaf(least, q == XCONV_Q_E4M3 ? 1.f / 448.f : 1.f / 127.f, 0.f * least), M * r};
}
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// The nearest whole number of y * inv, at most 127 (and a little) in magnitude, in the low byte: added to 3 * 2^22, where a float's last place is one.
__device__ __forceinline__ uint32_t int8(float y, float inv) { return __float_as_uint(fmaf(y, inv, 12582912.f)); }
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
