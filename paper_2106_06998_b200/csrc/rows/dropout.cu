// Dropout whose mask is drawn from a seed, with a residual's addition, and values back from 8 bits.
//
//   y = residual + (dropped ? 0 : x / (1 - p)),    x = q scale
//
// Memory bounds both, or, of 16-bit values, the ten rounds and the choice of what they leave (24 and some 50 cycles of an SM for the octets of a warp, against 66 of memory for three
// tensors); a thread takes octets, whose masks are one Philox block each.
//
// Measured (B200, copy rate 6.57 TB/s; replayed from a graph): 512 x 256 x 28 x 28 bf16 with a residual, 617 MB, 100 us = 6.2 TB/s (108 in a long loop, at lower clocks); 8192 x 4096 floats
// 60 us, as a copy; gradients of 16 M bf16 values 18 us (floor 10.2); rows at any alignment: 164948 x 97 bf16 23 us (floor 14.6), by octets cut out in registers 37, whole
// channels of 47250 x 97 float16 4.5 us (floor 2.8), 10.7; back from int8, 8192 x 4096 into bf16 18.2 us (floor 15.3).
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
  pdl_wait();
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

// Dense rows that do not begin on 16-byte boundaries: whatever the rows, in pieces of 16 bytes.  A block draws the mask of its pieces' rows into shared memory, a byte an octet, and
// every piece picks its bits from the up to three octets that it meets.  Rows that share a mask row find it drawn once a block.
constexpr int LOOSE_EACH = 4, LOOSE_PIECES = 256 * LOOSE_EACH, LOOSE_BYTES = 24 * 1024;

struct LooseArgs {
  const void *X, *R;
  void* Y;
  long values;
  int C, octets, shared;           // shared: mask rows have several rows
  Divisor by;                      // C
  Drop drop;
};

template <typename T, int DROP>
__global__ void __launch_bounds__(256, 4) dropout_loose_kernel(const LooseArgs a) {
  extern __shared__ unsigned char masks[];
  constexpr int PER = 16 / sizeof(T);
  pdl_wait();
  const long first = (long)blockIdx.x * (LOOSE_PIECES * PER);                   // the block's first value
  const int here = (int)min((long)(LOOSE_PIECES * PER), a.values - first);
  const auto load = [&](const void* from, int i, uint4& u) {
    const int at = i * PER;
    u = make_uint4(0u, 0u, 0u, 0u);
    if (at + PER <= here) {
      u = *reinterpret_cast<const uint4*>(static_cast<const T*>(from) + first + at);
    } else {
      uint32_t* w = &u.x;
#pragma unroll
      for (int e = 0; e < PER; ++e)
        if (at + e < here) {
          if constexpr (sizeof(T) == 4) w[e] = static_cast<const uint32_t*>(from)[first + at + e];
          else w[e / 2] |= (uint32_t)static_cast<const unsigned short*>(from)[first + at + e] << (16 * (e % 2));
        }
    }
  };
  uint4 x[LOOSE_EACH];
#pragma unroll
  for (int i = 0; i < LOOSE_EACH; ++i) load(a.X, threadIdx.x + 256 * i, x[i]);
  long row0 = 0;
  int col0 = 0, rows = 0, origin = 0;                        // of the block's first value; rows behind its row; the byte of its row's first octet (before the masks, if these begin within the row)
  if (DROP) {
    const uint2 key = a.drop.key<DROP>();
    row0 = first / a.C;
    col0 = (int)(first - row0 * a.C);
    rows = (int)(((long)col0 + here - 1) / a.C);
    const uint32_t m0 = a.drop.per((uint32_t)row0), m1 = a.drop.per((uint32_t)(row0 + rows));
    // from the octet of the first value to that of the last; of shared mask rows all octets
    const unsigned long long begin = (unsigned long long)m0 * (uint32_t)a.octets + (a.shared ? 0 : col0 / 8);
    const int last = (int)(((long)col0 + here - 1) - (long)rows * a.C) / 8;
    const int count = (int)((unsigned long long)m1 * (uint32_t)a.octets + (a.shared ? a.octets - 1 : last) + 1 - begin);
    origin = a.shared ? 0 : -(col0 / 8);
    int k = (a.shared ? 0 : col0 / 8) + (int)threadIdx.x;
    k %= a.octets;
    const int step = 256 % a.octets;
    for (int i = threadIdx.x; i < count; i += 256) {
      const uint32_t b = mask_bits(a.drop, key, begin + i);
      masks[i] = (unsigned char)(8 * k + 8 <= a.C ? b : b & ((1u << (a.C - 8 * k)) - 1u));
      k += step;
      if (k >= a.octets) k -= a.octets;
    }
    if (threadIdx.x < 2) masks[count + threadIdx.x] = 0;                         // (what the last pieces ask for)
    __syncthreads();
  }
  uint4 r[LOOSE_EACH];
  if (a.R)
#pragma unroll
    for (int i = 0; i < LOOSE_EACH; ++i) load(a.R, threadIdx.x + 256 * i, r[i]);
#pragma unroll
  for (int i = 0; i < LOOSE_EACH; ++i) {
    const int at = (threadIdx.x + 256 * i) * PER;
    if (at >= here) continue;
    float f[PER], g[PER];
    const auto floats = [](const uint4& u, float (&v)[PER]) {
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(w[e]);
      } else {
        floats_of<T>(w, v);
      }
    };
    floats(x[i], f);
#pragma unroll
    for (int e = 0; e < PER; ++e) g[e] = 0.f;
    if (a.R) floats(r[i], g);
    if (DROP) {
      const uint32_t n = (uint32_t)col0 + (uint32_t)at, row = a.by(n);
      const int c = (int)(n - row * (uint32_t)a.C), k = c >> 3;
      const auto byte_of = [&](uint32_t r) { return (a.shared ? (int)(a.drop.per((uint32_t)row0 + r) - a.drop.per((uint32_t)row0)) : (int)r) * a.octets + origin; };
      // the octet of the first value, the one behind it, and the one behind that
      const int b = byte_of(row) + k, here0 = min(8, a.C - 8 * k) - (c & 7);
      const bool more = k + 1 < a.octets;
      const int next = a.shared && k + 2 >= a.octets ? byte_of(min(row + 1, (uint32_t)rows)) : b + (more ? 2 : 1);
      uint32_t bits = (uint32_t)masks[b] >> (c & 7);
      if (more) {
        bits |= (uint32_t)masks[b + 1] << here0;
        bits |= (uint32_t)masks[next] << min(here0 + min(8, a.C - 8 * k - 8), 31);
      } else {
        bits |= (uint32_t)masks[next] << here0;
      }
#pragma unroll
      for (int e = 0; e < PER; ++e) f[e] = bits >> e & 1 ? g[e] : fmaf(f[e], a.drop.scale, g[e]);
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e) f[e] += g[e];
    }
    uint32_t w[4];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(f[e]);
    } else {
      words_for<T>(f, w);
    }
    T* to = static_cast<T*>(a.Y) + first + at;
    if (at + PER <= here) {
      *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e)
        if (at + e < here) to[e] = from_f<T>(f[e]);
    }
  }
}

struct DequantArgs {
  Rows Q, X;
  const float* scales;
  Units units;
  int shift, q_groups;             // values of a scale: 2^shift, or (0) a row
};

__device__ __forceinline__ float2 from_e4m3x2(uint32_t u) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)u));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

template <int Q>
__device__ __forceinline__ void codes_of(uint32_t lo, uint32_t hi, float (&f)[8]) {
  const uint32_t b[2] = {lo, hi};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (Q == XCONV_Q_E4M3) {
      const float2 x = from_e4m3x2(b[h] & 0xffffu), y = from_e4m3x2(b[h] >> 16);
      f[4 * h] = x.x; f[4 * h + 1] = x.y; f[4 * h + 2] = y.x; f[4 * h + 3] = y.y;
    } else {
      // (a byte moved up by 128 as the last one of 2^23 and so much: a conversion would take the unit that makes a quarter as many)
#pragma unroll
      for (int e = 0; e < 4; ++e) f[4 * h + e] = __uint_as_float(__byte_perm(b[h] ^ 0x80808080u, 0x4b000000u, 0x7650 + e)) - 8388736.f;
    }
  }
}

// Octets a thread of aligned rows: two (32 x 4096 e4m3 into bf16 1.5 us, 8192 x 4096 17.7, into floats 36.5, 131072 x 64 int8 into bf16 6.0) or four (1.9, 18.0, 38.0, 5.9).
constexpr int DEQUANTIZE_EACH = 2;

template <typename T, bool VEC, bool FLAT, int Q, int EACH>
__global__ void __launch_bounds__(256) dequantize_kernel(const DequantArgs a) {
  typedef unsigned char byte;
  pdl_wait();
  const long first = (long)blockIdx.x * (256 * EACH) + threadIdx.x;
  Fetched<byte, VEC> fq[EACH];
  float scale[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const Unit<FLAT> n(a.units, first + 256 * i);
    fetch8<byte, VEC>(a.Q, n.template at<byte>(a.Q), n.row, 8 * n.k, n.C, n.in, fq[i]);
    scale[i] = n.in ? a.scales[FLAT ? 8 * n.u >> a.shift : n.row * a.q_groups + (a.shift ? 8 * n.k >> a.shift : 0)] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const Unit<FLAT> n(a.units, first + 256 * i);
    uint32_t b[2];
    words_of<byte, VEC>(fq[i], b);
    float f[8];
    codes_of<Q>(b[0], b[1], f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= scale[i];
    store8<T, VEC>(n.template at<T>(a.X), 8 * n.k, n.C, n.in, f);
  }
}

// Dense rows that do not begin on boundaries, whatever the rows, in pieces of eight values, which meet up to three scales; these lie in the order of the values.
struct LooseDequantArgs {
  const unsigned char* Q;
  void* X;
  const float* scales;
  long values, count;              // count: scales
  int C, group, q_groups;          // group: values of a scale (C: the row)
  Divisor by;                      // C
};
template <typename T, int Q>
__global__ void __launch_bounds__(256) dequantize_loose_kernel(const LooseDequantArgs a) {
  pdl_wait();
  const long first = (long)blockIdx.x * (LOOSE_PIECES * 8);
  const int here = (int)min((long)(LOOSE_PIECES * 8), a.values - first);
  const long row0 = first / a.C;
  const int col0 = (int)(first - row0 * a.C);
  uint2 q[LOOSE_EACH];
#pragma unroll
  for (int i = 0; i < LOOSE_EACH; ++i) {
    const int at = (threadIdx.x + 256 * i) * 8;
    q[i] = make_uint2(0u, 0u);
    if (at + 8 <= here) {
      q[i] = *reinterpret_cast<const uint2*>(a.Q + first + at);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < here) (e < 4 ? q[i].x : q[i].y) |= (uint32_t)a.Q[first + at + e] << (8 * (e % 4));
    }
  }
#pragma unroll
  for (int i = 0; i < LOOSE_EACH; ++i) {
    const int at = (threadIdx.x + 256 * i) * 8;
    if (at >= here) continue;
    const uint32_t n = (uint32_t)col0 + (uint32_t)at, row = a.by(n);
    const int c = (int)(n - row * (uint32_t)a.C), g = a.q_groups == 1 ? 0 : c / a.group;
    // the values of the first scale, and of the first two
    const int one = min((g + 1) * a.group, a.C) - c, two = one + (c + one < a.C ? min(a.group, a.C - c - one) : a.group);
    const long s = (row0 + row) * a.q_groups + g;
    const float s0 = a.scales[s], s1 = a.scales[min(s + 1, a.count - 1)], s2 = a.scales[min(s + 2, a.count - 1)];
    float f[8];
    codes_of<Q>(q[i].x, q[i].y, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= e < one ? s0 : e < two ? s1 : s2;
    uint32_t w[Octet<T>::WORDS];
    words_for<T>(f, w);
    T* to = static_cast<T*>(a.X) + first + at;
    if (at + 8 <= here) {
#pragma unroll
      for (int k = 0; k < Octet<T>::WORDS; k += 4) reinterpret_cast<uint4*>(to)[k / 4] = make_uint4(w[k], w[k + 1], w[k + 2], w[k + 3]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < here) to[e] = from_f<T>(f[e]);
    }
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
  if (!vec && dense && d->C >= 8 && at(X, 16) && at(residual, 16) && at(Y, 16)) {
    LooseArgs l = {};
    l.X = X; l.R = residual; l.Y = Y; l.values = d->rows * d->C; l.C = d->C; l.octets = (d->C + 7) / 8; l.by = divisor((uint32_t)d->C); l.drop = a.drop;
    const long values = LOOSE_PIECES * 16 / (long)es;
    l.shared = a.drop.how && d->rows_per_mask > 1;
    // bytes of a block's masks, at most
    const long rows = values / d->C + 2, bytes = l.shared ? (rows / d->rows_per_mask + 2) * l.octets + 2 : values / 8 + 2 * rows + 4;
    if (!a.drop.how || bytes <= LOOSE_BYTES)
      return with_type(d->dtype, [&](auto t) {
        using T = decltype(t);
        const auto kernel = a.drop.how == DROP_NONE ? dropout_loose_kernel<T, DROP_NONE> : a.drop.how == DROP_HOST ? dropout_loose_kernel<T, DROP_HOST> : dropout_loose_kernel<T, DROP_DEVICE>;
        return launch_pdl(kernel, dim3((unsigned)((l.values + values - 1) / values)), dim3(256), a.drop.how ? (size_t)bytes : 0, st, l);
      });
  }
  const bool flat = vec && dense && d->C % 8 == 0 && (!a.drop.how || d->rows_per_mask == 1);
  a.units = units_of(d);
  return with_type(d->dtype, [&](auto t) {
    using T = decltype(t);
    // Octets a thread: 64 bytes of a tensor, where there are enough for all SMs (512 x 256 x 28 x 28 bf16 100 us, with half as many 103, with one octet 116).
    constexpr int MOST = sizeof(T) == 2 ? 4 : 2;
    const int each = vec && a.units.count >= 2L * ROWS_SMS * 2048 ? MOST : 1;
    const auto kernel = with_kinds(vec, a.drop.how, [&](auto v, auto how) -> void (*)(const DropArgs) {
      constexpr int HOW = decltype(how)::value;
      if constexpr (!decltype(v)::value) return dropout_kernel<T, false, false, HOW, 1>;
      else if (each == 1) return flat ? dropout_kernel<T, true, true, HOW, 1> : dropout_kernel<T, true, false, HOW, 1>;
      else return flat ? dropout_kernel<T, true, true, HOW, MOST> : dropout_kernel<T, true, false, HOW, MOST>;
    });
    return launch_pdl(kernel, dim3(blocks_of(a.units.count, each)), dim3(256), 0, st, a);
  });
}

cudaError_t launch_dequantize(const xconv_rows_desc* d, const void* Q, const float* scales, void* X, cudaStream_t st) {
  DequantArgs a = {};
  const size_t es = d->dtype == XCONV_F32 ? 4 : 2;
  a.Q = rows_of(Q, d->rows, d->C, d->y_stride, 1); a.X = rows_of(X, d->rows, d->C, d->x_stride, es);
  a.scales = scales; 
  const int group = d->q_group < d->C ? d->q_group : 0;
  while (group && (1 << a.shift) < group) ++a.shift;
  a.q_groups = group ? (d->C + group - 1) / group : 1;
  const bool vec = d->C % 8 == 0 && whole(a.Q, 8) && whole(a.X, 16);
  const bool dense = d->x_stride == d->C && d->y_stride == d->C;
  if (!vec && dense && d->C >= 8 && at(Q, 8) && at(X, 16)) {
    LooseDequantArgs l = {};
    l.Q = static_cast<const unsigned char*>(Q); l.X = X; l.scales = scales; l.values = d->rows * d->C; l.C = d->C;
    l.group = group ? group : d->C; l.q_groups = a.q_groups; l.count = d->rows * a.q_groups; l.by = divisor((uint32_t)d->C);
    return with_type(d->dtype, [&](auto t) {
      using T = decltype(t);
      return launch_pdl(d->q_type == XCONV_Q_E4M3 ? dequantize_loose_kernel<T, XCONV_Q_E4M3> : dequantize_loose_kernel<T, XCONV_Q_INT8>, dim3((unsigned)((l.values + LOOSE_PIECES * 8 - 1) / (LOOSE_PIECES * 8))), dim3(256), 0, st, l);
    });
  }
  const bool flat = vec && dense && group && d->C % group == 0;
  a.units = units_of(d);
  return with_type(d->dtype, [&](auto t) {
    using T = decltype(t);
    const auto pick = [&](auto q) {
      constexpr int Q = decltype(q)::value;
      return flat ? dequantize_kernel<T, true, true, Q, DEQUANTIZE_EACH> : vec ? dequantize_kernel<T, true, false, Q, DEQUANTIZE_EACH> : dequantize_kernel<T, false, false, Q, 1>;
    };
    const auto kernel = d->q_type == XCONV_Q_E4M3 ? pick(std::integral_constant<int, XCONV_Q_E4M3>()) : pick(std::integral_constant<int, XCONV_Q_INT8>());
    return launch_pdl(kernel, dim3(blocks_of(a.units.count, vec ? DEQUANTIZE_EACH : 1)), dim3(256), 0, st, a);
  });
}

}  // namespace xconv
