// Dropout whose mask is drawn from a seed, with a residual's addition, and values back from 8 bits.
//
//   y = residual + (dropped ? 0 : x / (1 - p)),    x = q scale
//
// Memory bounds both; a thread takes an octet, whose mask is one Philox block.
#include "rows.cuh"

#include <algorithm>

namespace xconv {

namespace {

struct DropArgs {
  const void *X, *R;
  void* Y;
  long rows, sx, sr, sy, units;
  int C, octets;
  Drop drop;
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dropout_kernel(const DropArgs a) {
  const uint2 key = a.drop.on ? a.drop.key() : make_uint2(0u, 0u);
  for (long u = (long)blockIdx.x * 256 + threadIdx.x; u < a.units; u += (long)gridDim.x * 256) {
    const long row = u / a.octets;
    const int k = (int)(u - row * a.octets);
    float f[8], r[8];
    load8<T, VEC>(static_cast<const T*>(a.X) + row * a.sx, 8 * k, a.C, f);
    if (a.R) load8<T, VEC>(static_cast<const T*>(a.R) + row * a.sr, 8 * k, a.C, r);
    if (a.drop.on) drop8(a.drop, key, (unsigned long long)a.drop.mask_row(row) * a.octets + k, f);
    if (a.R)
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] += r[e];
    store8<T, VEC>(static_cast<T*>(a.Y) + row * a.sy, 8 * k, a.C, f);
  }
}

struct DequantArgs {
  const unsigned char* Q;
  const float* scales;
  void* X;
  long sq, sx, units;
  int C, octets, q, q_group, q_groups;
};

__device__ __forceinline__ float2 from_e4m3x2(uint32_t u) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)u));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dequantize_kernel(const DequantArgs a) {
  for (long u = (long)blockIdx.x * 256 + threadIdx.x; u < a.units; u += (long)gridDim.x * 256) {
    const long row = u / a.octets;
    const int k = (int)(u - row * a.octets);
    const unsigned char* q = a.Q + row * a.sq + 8 * k;
    uint32_t b[2] = {0u, 0u};
    if (VEC) {
      const uint2 t = *reinterpret_cast<const uint2*>(q);
      b[0] = t.x; b[1] = t.y;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (8 * k + e < a.C) b[e / 4] |= (uint32_t)q[e] << (8 * (e % 4));
    }
    const float scale = __ldg(a.scales + row * a.q_groups + (a.q_group ? 8 * k / a.q_group : 0));
    float f[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (a.q == XCONV_Q_E4M3) {
        const float2 lo = from_e4m3x2(b[i] & 0xffffu), hi = from_e4m3x2(b[i] >> 16);
        f[4 * i] = lo.x; f[4 * i + 1] = lo.y; f[4 * i + 2] = hi.x; f[4 * i + 3] = hi.y;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[4 * i + e] = (float)(int)(signed char)(b[i] >> (8 * e));
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= scale;
    store8<T, VEC>(static_cast<T*>(a.X) + row * a.sx, 8 * k, a.C, f);
  }
}

inline unsigned blocks_of(long units) { return (unsigned)std::min((units + 255) / 256, 1L << 30); }

}  // namespace

cudaError_t launch_dropout(const xconv_rows_desc* d, const void* X, const void* residual, void* Y, cudaStream_t st) {
  DropArgs a = {};
  a.X = X; a.R = residual; a.Y = Y;
  a.rows = d->rows; a.sx = d->x_stride; a.sr = d->r_stride; a.sy = d->y_stride;
  a.C = d->C; a.octets = (d->C + 7) / 8; a.units = d->rows * a.octets;
  a.drop = drop_of(d);
  const int n = d->dtype == XCONV_F32 ? 4 : 8;
  const bool vec = d->C % n == 0 && at(X, 16) && at(residual, 16) && at(Y, 16) && d->x_stride % n == 0 && (!residual || d->r_stride % n == 0) && d->y_stride % n == 0;
  return with_type(d->dtype, [&](auto t) {
    using T = decltype(t);
    const auto kernel = vec ? dropout_kernel<T, true> : dropout_kernel<T, false>;
    kernel<<<blocks_of(a.units), 256, 0, st>>>(a);
    return cudaGetLastError();
  });
}

cudaError_t launch_dequantize(const xconv_rows_desc* d, const void* Q, const float* scales, void* X, cudaStream_t st) {
  DequantArgs a = {};
  a.Q = static_cast<const unsigned char*>(Q); a.scales = scales; a.X = X;
  a.sq = d->y_stride; a.sx = d->x_stride;
  a.C = d->C; a.octets = (d->C + 7) / 8; a.units = d->rows * a.octets;
  a.q = d->q_type; a.q_group = d->q_group < d->C ? d->q_group : 0; a.q_groups = a.q_group ? (d->C + a.q_group - 1) / a.q_group : 1;
  const bool vec = d->C % 8 == 0 && at(Q, 8) && at(X, 16) && d->y_stride % 8 == 0 && d->x_stride % (d->dtype == XCONV_F32 ? 4 : 8) == 0;
  return with_type(d->dtype, [&](auto t) {
    using T = decltype(t);
    const auto kernel = vec ? dequantize_kernel<T, true> : dequantize_kernel<T, false>;
    kernel<<<blocks_of(a.units), 256, 0, st>>>(a);
    return cudaGetLastError();
  });
}

}  // namespace xconv
