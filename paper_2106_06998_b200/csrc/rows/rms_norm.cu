// RMS norm with the residual's addition and dropout in front of it, and 8-bit outputs.
//
//   h = drop(x) + residual,  rstd = 1 / sqrt(sum h^2 / C + eps),  y = h rstd w
//
// Memory bounds it: x and the residual are read once, h and y written once.  A row lies in the registers of `group` threads, V octets each; h stays in float for y (it
// is rounded once, where it is written).  Blocks go from row to row, and a row's loads are under way while the one before is summed and written; nothing is staged.
//
// Measured (B200, copy rate 6.57 TB/s; replayed from a graph, with a residual): 8192 x 4096 bf16, 268 MB, 44.5 us = 6.0 TB/s; 8192 x 4096 floats 85.6 us = 6.3 TB/s; 125000 x 128 bf16
// 23.0 us; with dropout 8192 x 4096 bf16 53.3 us (a Philox block costs 24 cycles of an SM for 32 octets, and 122 registers hold half the threads); into e4m3 with a scale
// for 128 values, 235 MB, 8192 x 4096 bf16 47 us (issue slots 75 %); one row 2.5 us, a launch.  Rows that do not begin on 16-byte boundaries: rms_staged.cu.
#include "eight_bits.cuh"
#include "rms.h"

namespace xconv {

namespace {

struct RmsArgs {
  Rows X, R, H, Y;
  Weight w;
  float *scales, *rstd;
  long rows;
  int C, octets, group;
  int q, q_group, q_shift, q_groups;       // 8 bits: the type, values of a scale (2^q_shift, or 0: the row), scales of a row
  float eps, inv_c;
  Drop drop;
};

template <bool VEC>
__device__ __forceinline__ void store8q(unsigned char* row, int c, int C, bool in, const float (&u)[8], const Scale& f, int q) {
  uint32_t b[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 v = q_of(u[4 * i], u[4 * i + 1], f), w = q_of(u[4 * i + 2], u[4 * i + 3], f);
    b[i] = q == XCONV_Q_E4M3 ? e4m3x2(v) | e4m3x2(w) << 16 : __byte_perm(int8x2(v), int8x2(w), 0x5410);
  }
  store8<unsigned char, VEC>(row, c, C, in, b);
}
// The largest magnitude of the `width` values of which this lane and its neighbours hold an octet each.
__device__ __forceinline__ float group_most(float m, int width) {
  for (int o = width >> 4; o > 0; o >>= 1) m = most_of(m, __shfl_xor_sync(0xffffffffu, m, o));
  return m;
}
// The octet of h from what was fetched of x and r, and which of x's values are dropped, by bits.
template <typename T, bool VEC, int DROP>
__device__ __forceinline__ void sum_of(const RmsArgs& a, uint32_t dropped, const Fetched<T, VEC>& fx, const Fetched<T, VEC>& fr, int k, bool in, float (&h)[8]) {
  values_of<T, VEC>(fx, 8 * k, a.C, in, h);
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = 0.f;
  if (a.R.p) values_of<T, VEC>(fr, 8 * k, a.C, in, f);
  if (DROP) {
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = dropped & 1u << e ? f[e] : fmaf(h[e], a.drop.scale, f[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] += f[e];
  }
}

// ---- rows in registers, V octets a thread; the next row is fetched while this one is worked on

// (Two octets into 8 bits: 64 registers, at which an SM holds 1024 threads; with the 69 that the compiler would take 8192 x 4096 bf16 takes 50.1 us, not 47.1.)
template <typename T, int V, bool VEC, bool Q, int DROP>
__global__ void __launch_bounds__(512, Q && VEC && V == 2 && sizeof(T) == 2 && DROP == DROP_NONE ? 2 : 0) rms_forward_kernel(const RmsArgs a) {
  __shared__ float sums[2][32];
  __shared__ float most[2][32];
  typedef std::conditional_t<Q, unsigned char, T> Y;
  const int group = a.group, lane = group <= 32 ? threadIdx.x & (group - 1) : threadIdx.x;
  const int groups = group <= 32 ? blockDim.x / group : 1, own = group <= 32 ? threadIdx.x / group : 0;
  pdl_wait();
  const uint2 key = a.drop.key<DROP>();
  const long step = (long)gridDim.x * groups;
  long row = (long)blockIdx.x * groups + own;
  Walk<T> x(a.X, row, step), r(a.R, row, step), hs(a.H, row, step);
  Walk<Y> ys(a.Y, row, step);
  Fetched<T, VEC> fx[V], fr[V];
  const auto fetch = [&](long next) {
    const bool in = next < a.rows;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int k = lane + v * group;
      fetch8<T, VEC>(a.X, x.row, next, 8 * k, a.C, in && k < a.octets, fx[v]);
      if (a.R.p) fetch8<T, VEC>(a.R, r.row, next, 8 * k, a.C, in && k < a.octets, fr[v]);
    }
    x.next(); r.next();
  };
  // (the next row's mask, too: there are loads to wait for meanwhile)
  uint32_t dropped[V];
  const auto draw = [&](long next) {
    if (!DROP) return;
    const unsigned long long block = a.drop.first_block(next, a.octets);
#pragma unroll
    for (int v = 0; v < V; ++v) dropped[v] = mask_bits(a.drop, key, block + lane + v * group);
  };
#pragma unroll
  for (int v = 0; v < V; ++v) dropped[v] = 0;
  fetch(row);
  draw(row);
  float w[8];
  if (V == 1) a.w.load<T, VEC>(8 * min(lane, a.octets - 1), a.C, w);
  int turn = 0;
  for (long row0 = (long)blockIdx.x * groups; row0 < a.rows; row0 += step, row += step, turn ^= 1, hs.next(), ys.next()) {
    const bool in = row < a.rows;
    float h[V][8], ss = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int k = lane + v * group;
      sum_of<T, VEC, DROP>(a, dropped[v], fx[v], fr[v], k, in && k < a.octets, h[v]);
    }
    fetch(row + step);
    draw(row + step);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int k = lane + v * group;
      if (a.H.p) store8<T, VEC>(hs.out(), 8 * k, a.C, in && k < a.octets, h[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(h[v][e], h[v][e], ss);
    }
    ss = row_sum(ss, group, sums[turn]);
    const float rstd = rsqrtf(fmaf(ss, a.inv_c, a.eps));
    if (in && lane == 0 && a.rstd) a.rstd[row] = rstd;
    const Root root = root_of(rstd);
    const float by = Q ? root.power : rstd;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int k = lane + v * group;
      if (V > 1) a.w.load<T, VEC>(8 * min(k, a.octets - 1), a.C, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[v][e] *= by * w[e];
      if constexpr (!Q) store8<T, VEC>(ys.out(), 8 * k, a.C, in && k < a.octets, h[v]);
    }
    if constexpr (Q) {
      float m[V];
#pragma unroll
      for (int v = 0; v < V; ++v) m[v] = magnitude(h[v]);
      if (a.q_group) {
#pragma unroll
        for (int v = 0; v < V; ++v) m[v] = group_most(m[v], a.q_group);
      } else {
#pragma unroll
        for (int v = 1; v < V; ++v) m[0] = most_of(m[0], m[v]);
        m[0] = row_most(m[0], group, most[turn]);
#pragma unroll
        for (int v = 1; v < V; ++v) m[v] = m[0];
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int k = lane + v * group;
        const bool here = in && k < a.octets;
        const Scale f = q_scale(m[v], root, a.q);
        if (here && (a.q_group ? (8 * k & (a.q_group - 1)) == 0 : k == 0)) a.scales[row * a.q_groups + (a.q_group ? 8 * k >> a.q_shift : 0)] = f.scale;
        store8q<VEC>(ys.out(), 8 * k, a.C, here, h[v], f, a.q);
      }
    }
  }
}

// ---- rows of any length, a block each, read again for every step

template <typename T, bool VEC, bool Q, int DROP>
__global__ void __launch_bounds__(1024) rms_forward_wide_kernel(const RmsArgs a) {
  __shared__ float sums[2][32];
  __shared__ float most[2][32];
  pdl_wait();
  const uint2 key = a.drop.key<DROP>();
  const int steps = (a.octets + 1023) / 1024;
  int turn = 0;
  for (long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const T *x = row_of<T>(a.X, row), *r = row_of<T>(a.R, row);
    const unsigned long long block = DROP ? a.drop.first_block(row, a.octets) : 0;
    // f(k) with the octet k of h in y, for all octets of this thread; the next one is fetched meanwhile, where the registers hold it (4096 x 16392 bf16 into e4m3 202 us, else 224; of
    // unaligned rows 525 and 456).
    float y[8];
    const auto over = [&](auto&& f) {
      Fetched<T, VEC> fx, fr;
      const auto fetch = [&](int k) {
        fetch8<T, VEC>(a.X, x, row, 8 * k, a.C, k < a.octets, fx);
        if (a.R.p) fetch8<T, VEC>(a.R, r, row, 8 * k, a.C, k < a.octets, fr);
      };
      constexpr bool AHEAD = VEC && (sizeof(T) == 2 || DROP == DROP_NONE);
      if (AHEAD) fetch(threadIdx.x);
      for (int v = 0; v < steps; ++v) {
        const int k = threadIdx.x + v * 1024;
        if (!AHEAD) fetch(k);
        sum_of<T, VEC, DROP>(a, DROP ? mask_bits(a.drop, key, block + k) : 0, fx, fr, k, k < a.octets, y);
        if (AHEAD) fetch(k + 1024);
        f(k);
      }
    };
    float ss = 0.f;
    over([&](int k) {
      if (a.H.p) store8<T, VEC>(const_cast<T*>(row_of<T>(a.H, row)), 8 * k, a.C, k < a.octets, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(y[e], y[e], ss);
    });
    ss = row_sum(ss, 1024, sums[turn]);
    const float rstd = rsqrtf(fmaf(ss, a.inv_c, a.eps));
    if (threadIdx.x == 0 && a.rstd) a.rstd[row] = rstd;
    const Root root = root_of(rstd);
    const float by = Q ? root.power : rstd;
    const auto weigh = [&](int k) {
      float w[8];
      a.w.load<T, VEC>(8 * min(k, a.octets - 1), a.C, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] *= by * w[e];
    };
    float m = 0.f;
    if (Q && !a.q_group) {
      over([&](int k) {
        weigh(k);
        m = most_of(m, magnitude(y));
      });
      m = row_most(m, 1024, most[turn]);
    }
    over([&](int k) {
      const bool here = k < a.octets;
      weigh(k);
      if (!Q) {
        store8<T, VEC>(const_cast<T*>(row_of<T>(a.Y, row)), 8 * k, a.C, here, y);
        return;
      }
      if (a.q_group) m = group_most(magnitude(y), a.q_group);
      const Scale f = q_scale(m, root, a.q);
      if (here && (a.q_group ? (8 * k & (a.q_group - 1)) == 0 : k == 0)) a.scales[row * a.q_groups + (a.q_group ? 8 * k >> a.q_shift : 0)] = f.scale;
      store8q<VEC>(const_cast<unsigned char*>(row_of<unsigned char>(a.Y, row)), 8 * k, a.C, here, y, f, a.q);
    });
  }
}

}  // namespace

cudaError_t launch_rms_forward(const xconv_rows_desc* d, const void* X, const void* residual, const void* weight, void* H, void* Y, float* scales, float* rstd,
                               cudaStream_t st) {
  RmsArgs a = {};
  const size_t es = d->dtype == XCONV_F32 ? 4 : 2, ys = d->q_type ? 1 : es;
  a.X = rows_of(X, d->rows, d->C, d->x_stride, es); a.R = rows_of(residual, d->rows, d->C, d->r_stride, es);
  a.H = rows_of(H, d->rows, d->C, d->h_stride, es); a.Y = rows_of(Y, d->rows, d->C, d->y_stride, ys);
  a.w = {weight, d->param_dtype == XCONV_F32}; a.scales = scales; a.rstd = rstd;
  a.rows = d->rows; a.C = d->C; a.octets = (d->C + 7) / 8; a.eps = d->eps; a.inv_c = 1.f / (float)d->C;
  a.q = d->q_type; a.q_group = d->q_group < d->C ? d->q_group : 0; a.q_groups = a.q_group ? (d->C + a.q_group - 1) / a.q_group : 1;
  while (a.q_group >> a.q_shift > 1) ++a.q_shift;
  a.drop = drop_of(d);
  const bool vec = d->C % (a.q ? 8 : 16 / es) == 0 && whole(a.X, 16) && whole(a.R, 16) && whole(a.H, 16) && whole(a.Y, a.q ? 8 : 16) && at(weight, 16);
  cudaError_t e;
  if (!vec && rms_staged_forward(d, X, residual, weight, H, Y, scales, rstd, st, &e)) return e;
  const Team p = team_of(a.octets, !vec || (a.q && es == 4), vec && es == 2);
  a.group = p.group;
  return with_type(d->dtype, [&](auto t) {
    using T = decltype(t);
    const auto pick = [&](auto v, auto dropped) -> void (*)(const RmsArgs) {
      constexpr bool VEC = decltype(v)::value;
      constexpr int DROP = decltype(dropped)::value;
      if (p.V == 0) return a.q ? rms_forward_wide_kernel<T, VEC, true, DROP> : rms_forward_wide_kernel<T, VEC, false, DROP>;
      if constexpr (VEC && sizeof(T) == 2)
        if (p.V == 4) return a.q ? rms_forward_kernel<T, 4, VEC, true, DROP> : rms_forward_kernel<T, 4, VEC, false, DROP>;
      if (a.q) return p.V == 1 ? rms_forward_kernel<T, 1, VEC, true, DROP> : rms_forward_kernel<T, 2, VEC, true, DROP>;
      return p.V == 1 ? rms_forward_kernel<T, 1, VEC, false, DROP> : rms_forward_kernel<T, 2, VEC, false, DROP>;
    };
    const auto kernel = with_kinds(vec, a.drop.how, pick);
    // As many blocks as the SMs hold, or several times as many: the later ones' rows begin as the first ones' end, at different times, which serves where memory alone bounds them (four
    // times: 125000 x 128 floats 42.0 us, once 48.1; twice: 8192 x 4096 bf16 44.1 us, once 46.9) and costs where threads have much to set up for little (8192 x 4096 bf16 with dropout: four times
    // 55.2 us, once 53.2; of 125000 x 128 bf16 four times would be 22.2 us, once is 23.2).
    const int waves = es == 4 ? 4 : a.drop.how == DROP_NONE && p.group > 32 ? 2 : 1;
    const long blocks = std::min((d->rows + p.groups - 1) / p.groups, (long)ROWS_SMS * waves * resident_blocks(kernel, p.threads, 0));
    return launch_pdl(kernel, dim3((unsigned)blocks), dim3(p.threads), 0, st, a);
  });
}

}  // namespace xconv
