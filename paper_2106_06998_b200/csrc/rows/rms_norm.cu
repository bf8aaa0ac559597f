// RMS norm with the residual's addition and dropout in front of it, and 8-bit outputs.
//
//   h = drop(x) + residual,  rstd = 1 / sqrt(sum h^2 / C + eps),  y = h rstd w
//
// Memory bounds it: x and the residual are read once, h and y written once.  A row lies in the registers of `group` threads, V octets each; h stays in float for y (it
// is rounded once, where it is written).
#include "rows.cuh"

#include <algorithm>

namespace xconv {

namespace {

struct RmsArgs {
  const void *X, *R;
  Weight w;
  void *H, *Y;
  float *scales, *rstd;
  long rows, sx, sr, sh, sy;
  int C, octets, group;
  int q, q_group, q_groups;        // 8 bits: the type, values of a scale (0: the row), scales of a row
  float eps, inv_c;
  Drop drop;
};

// ---- 8 bits

constexpr float Q_LEAST = 7.888609052210118e-31f;          // 2^-100

__device__ __forceinline__ float q_largest(int q) { return q == XCONV_Q_E4M3 ? 448.f : 127.f; }
__device__ __forceinline__ uint32_t magnitude(const float (&y)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(y[e]) & 0x7fffffffu);
  return m;
}
// The scale of values up to `most` (as bits: infinities and NaN stay what they are).
__device__ __forceinline__ float q_scale(uint32_t most, int q) {
  const float a = __uint_as_float(most);
  return (a < Q_LEAST ? Q_LEAST : a) / q_largest(q);
}
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t int8(float v) { return (uint32_t)max(-127, min(127, __float2int_rn(v))) & 0xffu; }
template <bool VEC>
__device__ __forceinline__ void store8q(unsigned char* row, int c, int C, const float (&y)[8], float inv, int q) {
  uint32_t b[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float *v = y + 4 * i;
    b[i] = q == XCONV_Q_E4M3 ? e4m3x2(v[0] * inv, v[1] * inv) | e4m3x2(v[2] * inv, v[3] * inv) << 16
                             : int8(v[0] * inv) | int8(v[1] * inv) << 8 | int8(v[2] * inv) << 16 | int8(v[3] * inv) << 24;
  }
  if (VEC) {
    *reinterpret_cast<uint2*>(row + c) = make_uint2(b[0], b[1]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < C) row[c + e] = (unsigned char)(b[e / 4] >> (8 * (e % 4)));
  }
}

// ---- the kernel.  V octets a thread; V = 0: rows of any length, read again for every step.

template <typename T, int V, bool VEC>
__global__ void __launch_bounds__(1024) rms_forward_kernel(const RmsArgs a) {
  __shared__ float sums[2][32];
  __shared__ uint32_t most[2][32];
  const int group = a.group, lane = group <= 32 ? threadIdx.x & (group - 1) : threadIdx.x;
  const int groups = group <= 32 ? blockDim.x / group : 1, own = group <= 32 ? threadIdx.x / group : 0;
  const uint2 key = a.drop.on ? a.drop.key() : make_uint2(0u, 0u);
  const int steps = V ? V : (a.octets + group - 1) / group;
  int turn = 0;
  for (long row0 = (long)blockIdx.x * groups; row0 < a.rows; row0 += (long)gridDim.x * groups, turn ^= 1) {
    const long row = row0 + own;
    const bool in = row < a.rows;
    const T *x = static_cast<const T*>(a.X) + row * a.sx, *r = static_cast<const T*>(a.R) + row * a.sr;
    const unsigned long long block = (unsigned long long)a.drop.mask_row(row) * a.octets;
    const auto sum_of = [&](int k, float (&h)[8]) {
      if (!in || k >= a.octets) {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = 0.f;
        return;
      }
      load8<T, VEC>(x, 8 * k, a.C, h);
      float f[8];
      if (a.R) load8<T, VEC>(r, 8 * k, a.C, f);
      if (a.drop.on) drop8(a.drop, key, block + k, h);
      if (a.R)
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] += f[e];
    };
    float held[V ? V : 1][8], ss = 0.f;
#pragma unroll
    for (int v = 0; v < steps; ++v) {
      const int k = lane + v * group;
      float (&h)[8] = held[V ? v : 0];
      sum_of(k, h);
      if (a.H && in && k < a.octets) store8<T, VEC>(static_cast<T*>(a.H) + row * a.sh, 8 * k, a.C, h);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(h[e], h[e], ss);
    }
    ss = row_sum(ss, group, sums[turn]);
    const float rstd = rsqrtf(fmaf(ss, a.inv_c, a.eps));
    if (in && lane == 0 && a.rstd) a.rstd[row] = rstd;
    const auto normed = [&](int v, float (&y)[8]) {
      const int k = lane + v * group;
      if (!V) sum_of(k, held[0]);
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = 0.f;
      if (k < a.octets) a.w.load<T, VEC>(8 * k, a.C, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = held[V ? v : 0][e] * rstd * w[e];
    };
    float y[8];
    if (!a.q) {
#pragma unroll
      for (int v = 0; v < steps; ++v) {
        normed(v, y);
        const int k = lane + v * group;
        if (in && k < a.octets) store8<T, VEC>(static_cast<T*>(a.Y) + row * a.sy, 8 * k, a.C, y);
      }
      continue;
    }
    uint32_t m = 0;
    if (!a.q_group) {
#pragma unroll
      for (int v = 0; v < steps; ++v) {
        normed(v, y);
        m = max(m, magnitude(y));
        if (V)
#pragma unroll
          for (int e = 0; e < 8; ++e) held[V ? v : 0][e] = y[e];
      }
      m = row_max(m, group, most[turn]);
    }
#pragma unroll
    for (int v = 0; v < steps; ++v) {
      const int k = lane + v * group;
      if (V && !a.q_group) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = held[V ? v : 0][e];
      } else {
        normed(v, y);
      }
      if (a.q_group) {                                       // (a scale's octets are neighbours in a warp)
        m = magnitude(y);
        for (int o = a.q_group >> 4; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      }
      const float scale = q_scale(m, a.q);
      if (!in || k >= a.octets) continue;
      const bool first = a.q_group ? (8 * k) % a.q_group == 0 : k == 0;
      if (first) a.scales[row * a.q_groups + (a.q_group ? 8 * k / a.q_group : 0)] = scale;
      store8q<VEC>(static_cast<unsigned char*>(a.Y) + row * a.sy, 8 * k, a.C, y, 1.f / scale, a.q);
    }
  }
}

}  // namespace

cudaError_t launch_rms_forward(const xconv_rows_desc* d, const void* X, const void* residual, const void* weight, void* H, void* Y, float* scales, float* rstd,
                               cudaStream_t st) {
  RmsArgs a = {};
  a.X = X; a.R = residual; a.w = {weight, d->param_dtype == XCONV_F32}; a.H = H; a.Y = Y; a.scales = scales; a.rstd = rstd;
  a.rows = d->rows; a.sx = d->x_stride; a.sr = d->r_stride; a.sh = d->h_stride; a.sy = d->y_stride;
  a.C = d->C; a.octets = (d->C + 7) / 8; a.eps = d->eps; a.inv_c = 1.f / (float)d->C;
  a.q = d->q_type; a.q_group = d->q_group < d->C ? d->q_group : 0; a.q_groups = a.q_group ? (d->C + a.q_group - 1) / a.q_group : 1;
  a.drop = drop_of(d);
  const int n = d->dtype == XCONV_F32 ? 4 : 8;             // values of 16 bytes
  const bool vec = d->C % (a.q ? 8 : n) == 0 && at(X, 16) && at(residual, 16) && at(weight, 16) && at(H, 16) && at(Y, a.q ? 8 : 16) && d->x_stride % n == 0 &&
                   (!residual || d->r_stride % n == 0) && (!H || d->h_stride % n == 0) && d->y_stride % (a.q ? 8 : n) == 0;
  int V = 1;
  if (a.octets <= 32) a.group = pow2_from(a.octets);
  else if (a.octets <= 1024) a.group = (a.octets + 31) / 32 * 32;
  else { a.group = 1024; V = 0; }
  const int threads = a.group <= 32 ? 128 : a.group;
  const long groups = a.group <= 32 ? threads / a.group : 1;
  const long blocks = std::min((d->rows + groups - 1) / groups, (long)ROWS_SMS * (2048 / threads));
  return with_type(d->dtype, [&](auto t) {
    using T = decltype(t);
    const auto kernel = vec ? (V ? rms_forward_kernel<T, 1, true> : rms_forward_kernel<T, 0, true>) : (V ? rms_forward_kernel<T, 1, false> : rms_forward_kernel<T, 0, false>);
    kernel<<<(unsigned)blocks, threads, 0, st>>>(a);
    return cudaGetLastError();
  });
}

}  // namespace xconv
