// Dropout whose mask is drawn from a seed, with a residual's addition, and values back from 8 bits.
//
//   y = residual + (dropped ? 0 : x / (1 - p)),    x = q scale
//
// Memory bounds both; a thread takes an octet, whose mask is one Philox block.
#include "rows.cuh"

namespace xconv {

namespace {

// Octets by number: a thread takes EACH of them, 256 apart, and reads all before it works on any.  FLAT: the rows lie behind one another in all tensors and are whole octets, which
// then are one long row.
struct Units {
  long count;
  int octets, C;
  Divisor by;                      // octets, of numbers below 2^31
};
template <bool FLAT>
struct Unit {
  long u, row;
  int k, C;
  bool in;
  __device__ __forceinline__ Unit(const Units& a, long u) : u(u), row(0), k(0), C(FLAT ? 8 : a.C), in(u < a.count) {
    if (FLAT) return;
    row = a.count <= (1L << 31) ? (long)a.by((uint32_t)u) : u / a.octets;
    k = (int)(u - row * a.octets);
  }
  template <typename T> __device__ __forceinline__ T* at(const Rows& t) const {
    return const_cast<T*>(FLAT ? reinterpret_cast<const T*>(t.p) + 8 * u : row_of<T>(t, row));
  }
};

struct DropArgs {
  Rows X, R, Y;
  Units units;
  Drop drop;
};

template <typename T, bool VEC, bool FLAT, int DROP, int EACH>
__global__ void __launch_bounds__(256) dropout_kernel(const DropArgs a) {
  const uint2 key = a.drop.key<DROP>();
  const long first = (long)blockIdx.x * (256 * EACH) + threadIdx.x;
  Fetched<T, VEC> fx[EACH], fr[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const Unit<FLAT> n(a.units, first + 256 * i);
    fetch8<T, VEC>(a.X, n.template at<T>(a.X), n.row, 8 * n.k, n.C, n.in, fx[i]);
    if (a.R.p) fetch8<T, VEC>(a.R, n.template at<T>(a.R), n.row, 8 * n.k, n.C, n.in, fr[i]);
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const Unit<FLAT> n(a.units, first + 256 * i);
    float f[8], r[8];
    values_of<T, VEC, false>(fx[i], 8 * n.k, n.C, n.in, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = 0.f;
    if (a.R.p) values_of<T, VEC, false>(fr[i], 8 * n.k, n.C, n.in, r);
    if (DROP) {
      bool gone[8];
      mask8(a.drop, key, FLAT ? (unsigned long long)n.u : a.drop.first_block(n.row, a.units.octets) + n.k, gone);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = gone[e] ? r[e] : fmaf(f[e], a.drop.scale, r[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] += r[e];
    }
    store8<T, VEC>(n.template at<T>(a.Y), 8 * n.k, n.C, n.in, f);
  }
}

struct DequantArgs {
  Rows Q, X;
  const float* scales;
  Units units;
  int q, shift, q_groups;          // values of a scale: 2^shift, or (0) a row
};

__device__ __forceinline__ float2 from_e4m3x2(uint32_t u) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)u));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

template <typename T, bool VEC, bool FLAT, int EACH>
__global__ void __launch_bounds__(256) dequantize_kernel(const DequantArgs a) {
  typedef unsigned char byte;
  const long first = (long)blockIdx.x * (256 * EACH) + threadIdx.x;
  Fetched<byte, VEC> fq[EACH];
  float scale[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const Unit<FLAT> n(a.units, first + 256 * i);
    fetch8<byte, VEC>(a.Q, n.template at<byte>(a.Q), n.row, 8 * n.k, n.C, n.in, fq[i]);
    scale[i] = n.in ? __ldg(a.scales + (FLAT ? 8 * n.u >> a.shift : n.row * a.q_groups + (a.shift ? 8 * n.k >> a.shift : 0))) : 0.f;
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const Unit<FLAT> n(a.units, first + 256 * i);
    uint32_t b[2];
    words_of<byte, VEC>(fq[i], b);
    float f[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (a.q == XCONV_Q_E4M3) {
        const float2 lo = from_e4m3x2(b[h] & 0xffffu), hi = from_e4m3x2(b[h] >> 16);
        f[4 * h] = lo.x; f[4 * h + 1] = lo.y; f[4 * h + 2] = hi.x; f[4 * h + 3] = hi.y;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[4 * h + e] = (float)(int)(signed char)(b[h] >> (8 * e));
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= scale[i];
    store8<T, VEC>(n.template at<T>(a.X), 8 * n.k, n.C, n.in, f);
  }
}

inline Units units_of(const xconv_rows_desc* d) {
  Units u = {};
  u.octets = (d->C + 7) / 8; u.count = d->rows * u.octets; u.C = d->C; u.by = divisor((uint32_t)u.octets);
  return u;
}
inline unsigned blocks_of(long units, int each) { return (unsigned)((units + 256L * each - 1) / (256L * each)); }

}  // namespace

cudaError_t launch_dropout(const xconv_rows_desc* d, const void* X, const void* residual, void* Y, cudaStream_t st) {
  DropArgs a = {};
  const size_t es = d->dtype == XCONV_F32 ? 4 : 2;
  a.X = rows_of(X, d->rows, d->C, d->x_stride, es); a.R = rows_of(residual, d->rows, d->C, d->r_stride, es); a.Y = rows_of(Y, d->rows, d->C, d->y_stride, es);
  a.drop = drop_of(d);
  const bool vec = d->C % (16 / es) == 0 && whole(a.X, 16) && whole(a.R, 16) && whole(a.Y, 16);
  const bool dense = d->x_stride == d->C && (!residual || d->r_stride == d->C) && d->y_stride == d->C;
  const bool flat = vec && dense && d->C % 8 == 0 && (!a.drop.how || d->rows_per_mask == 1);
  a.units = units_of(d);
  return with_type(d->dtype, [&](auto t) {
    using T = decltype(t);
    const auto kernel = with_kinds(vec, a.drop.how, [&](auto v, auto how) -> void (*)(const DropArgs) {
      if constexpr (!decltype(v)::value) return dropout_kernel<T, false, false, decltype(how)::value, 1>;
      else return flat ? dropout_kernel<T, true, true, decltype(how)::value, 2> : dropout_kernel<T, true, false, decltype(how)::value, 2>;
    });
    kernel<<<blocks_of(a.units.count, vec ? 2 : 1), 256, 0, st>>>(a);
    return cudaGetLastError();
  });
}

cudaError_t launch_dequantize(const xconv_rows_desc* d, const void* Q, const float* scales, void* X, cudaStream_t st) {
  DequantArgs a = {};
  const size_t es = d->dtype == XCONV_F32 ? 4 : 2;
  a.Q = rows_of(Q, d->rows, d->C, d->y_stride, 1); a.X = rows_of(X, d->rows, d->C, d->x_stride, es);
  a.scales = scales; a.q = d->q_type;
  const int group = d->q_group < d->C ? d->q_group : 0;
  while (group && (1 << a.shift) < group) ++a.shift;
  a.q_groups = group ? (d->C + group - 1) / group : 1;
  const bool vec = d->C % 8 == 0 && whole(a.Q, 8) && whole(a.X, 16);
  const bool flat = vec && group && d->C % group == 0 && d->x_stride == d->C && d->y_stride == d->C;
  a.units = units_of(d);
  return with_type(d->dtype, [&](auto t) {
    using T = decltype(t);
    if (flat) dequantize_kernel<T, true, true, 4><<<blocks_of(a.units.count, 4), 256, 0, st>>>(a);
    else if (vec) dequantize_kernel<T, true, false, 4><<<blocks_of(a.units.count, 4), 256, 0, st>>>(a);
    else dequantize_kernel<T, false, false, 1><<<blocks_of(a.units.count, 1), 256, 0, st>>>(a);
    return cudaGetLastError();
  });
}

}  // namespace xconv
