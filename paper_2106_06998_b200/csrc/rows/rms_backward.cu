// Gradients of the RMS norm, of the residual's addition and of the dropout in front of it.
//
//   xh = h rstd,  g = dy w,  dr = dh + rstd (g - xh sum(g xh) / C),  dx = drop'(dr),  dw = sum over rows of dy xh
//
// Memory bounds it: dy, h (and dh) are read once, dr (and dx) written once.  The threads of a block keep the same columns from row to row and carry dw in registers; blocks
// leave a partial sum a column each, which a second kernel adds in fixed order (no atomics: the same bits every time).
#include "rows.cuh"

#include <algorithm>

namespace xconv {

namespace {

struct RmsBackArgs {
  const void *dY, *H, *dH;
  const float* rstd;
  Weight w;
  void *dX, *dR;
  float* part;
  long rows, sy, sh, sdh, sx, sr;
  int C, octets, group;
  float inv_c;
  Drop drop;
};

// V octets a thread; V = 0: rows of any length, read again for the second step; dw is then another kernel's.
template <typename T, int V, bool VEC>
__global__ void __launch_bounds__(1024) rms_backward_kernel(const RmsBackArgs a) {
  extern __shared__ float cols[];                            // C floats a warp, or a block of several
  __shared__ float sums[2][32];
  const int group = a.group, lane = group <= 32 ? threadIdx.x & (group - 1) : threadIdx.x;
  const int groups = group <= 32 ? blockDim.x / group : 1, own = group <= 32 ? threadIdx.x / group : 0;
  const uint2 key = a.drop.on ? a.drop.key() : make_uint2(0u, 0u);
  const int steps = V ? V : (a.octets + group - 1) / group;
  constexpr int HELD = V ? V : 1;
  float dw[HELD][8];
#pragma unroll
  for (int v = 0; v < HELD; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[v][e] = 0.f;
  int turn = 0;
  for (long row0 = (long)blockIdx.x * groups; row0 < a.rows; row0 += (long)gridDim.x * groups, turn ^= 1) {
    const long row = row0 + own;
    const bool in = row < a.rows;
    const float rstd = in ? __ldg(a.rstd + row) : 0.f;
    float xh[HELD][8], g[HELD][8], s = 0.f;
    const auto read = [&](int k, float (&x)[8], float (&y)[8]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = y[e] = 0.f;
      if (!in || k >= a.octets) return;
      load8<T, VEC>(static_cast<const T*>(a.H) + row * a.sh, 8 * k, a.C, x);
      load8<T, VEC>(static_cast<const T*>(a.dY) + row * a.sy, 8 * k, a.C, y);
    };
    const auto weigh = [&](int k, float (&x)[8], float (&y)[8], float (&d)[8]) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = 0.f;
      if (k < a.octets) a.w.load<T, VEC>(8 * k, a.C, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] *= rstd;
        d[e] = fmaf(y[e], x[e], d[e]);
        y[e] *= w[e];
      }
    };
#pragma unroll
    for (int v = 0; v < steps; ++v) {
      const int i = V ? v : 0, k = lane + v * group;
      read(k, xh[i], g[i]);
      weigh(k, xh[i], g[i], dw[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(g[i][e], xh[i][e], s);
    }
    const float mean = row_sum(s, group, sums[turn]) * a.inv_c;
    const unsigned long long block = (unsigned long long)a.drop.mask_row(row) * a.octets;
#pragma unroll
    for (int v = 0; v < steps; ++v) {
      const int i = V ? v : 0, k = lane + v * group;
      if (!in || k >= a.octets) continue;
      if (!V) {
        read(k, xh[0], g[0]);
        weigh(k, xh[0], g[0], dw[0]);
      }
      float d[8];
      if (a.dH) {
        load8<T, VEC>(static_cast<const T*>(a.dH) + row * a.sdh, 8 * k, a.C, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = fmaf(rstd, fmaf(-xh[i][e], mean, g[i][e]), d[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = rstd * fmaf(-xh[i][e], mean, g[i][e]);
      }
      if (a.dR) store8<T, VEC>(static_cast<T*>(a.dR) + row * a.sr, 8 * k, a.C, d);
      if (a.dX) {
        if (a.drop.on) drop8(a.drop, key, block + k, d);
        store8<T, VEC>(static_cast<T*>(a.dX) + row * a.sx, 8 * k, a.C, d);
      }
    }
  }
  if constexpr (V > 0) {
    if (!a.part) return;
    // The groups of a warp by shuffles, the warps side by side in shared memory, then column by column in order.
    for (int o = group; o < 32; o <<= 1)
#pragma unroll
      for (int v = 0; v < HELD; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[v][e] += __shfl_xor_sync(0xffffffffu, dw[v][e], o);
    if (group > 32) {
#pragma unroll
      for (int v = 0; v < HELD; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = 8 * (lane + v * group) + e;
          if (c < a.C) a.part[(size_t)blockIdx.x * a.C + c] = dw[v][e];
        }
      return;
    }
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) < group)
#pragma unroll
      for (int v = 0; v < HELD; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = 8 * (lane + v * group) + e;
          if (c < a.C) cols[warp * a.C + c] = dw[v][e];
        }
    __syncthreads();
    for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
      float t = cols[c];
      for (int i = 1; i < warps; ++i) t += cols[i * a.C + c];
      a.part[(size_t)blockIdx.x * a.C + c] = t;
    }
  }
}

// dw of rows that no block holds: a thread a column, a block a run of rows.
template <typename T>
__global__ void __launch_bounds__(256) rms_columns_kernel(const RmsBackArgs a, long rows_per) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.C) return;
  const long r0 = (long)blockIdx.y * rows_per, r1 = min(a.rows, r0 + rows_per);
  float dw = 0.f;
#pragma unroll 4
  for (long row = r0; row < r1; ++row)
    dw = fmaf(to_f(static_cast<const T*>(a.dY)[row * a.sy + c]), to_f(static_cast<const T*>(a.H)[row * a.sh + c]) * __ldg(a.rstd + row), dw);
  a.part[(size_t)blockIdx.y * a.C + c] = dw;
}

// Columns' sums over the parts, 32 columns a block: each of its warps adds every 32nd part, then the warps' sums are added in order.  (No parts: zeros.)
__global__ void __launch_bounds__(1024) rms_sums_kernel(const float* part, int parts, int C, float* dweight) {
  __shared__ float sums[32][33];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long c = (long)blockIdx.x * 32 + lane;
  float own[4] = {0.f, 0.f, 0.f, 0.f};
  if (c < C) sum_splits<32, 4, 4>(part + c, (size_t)C, warp, parts, own);
  sums[warp][lane] = (own[0] + own[1]) + (own[2] + own[3]);
  __syncthreads();
  float s = sums[lane][warp];                                // (column `warp` of the block's 32)
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  const long col = (long)blockIdx.x * 32 + warp;
  if (lane == 0 && col < C) dweight[col] = s;
}

// Rows that a block of rms_columns_kernel adds, at least, and partial sums at most.
constexpr long WIDE_ROWS = 64, WIDE_PARTS = 512;

struct Plan { int V, group, threads; long blocks, parts; };
Plan plan_of(const xconv_rows_desc* d) {
  Plan p = {};
  const long octets = (d->C + 7) / 8;
  p.V = 1;
  if (octets <= 32) p.group = pow2_from(octets);
  else if (octets <= 1024) p.group = (int)((octets + 31) / 32 * 32);
  else { p.group = 1024; p.V = 0; }
  p.threads = p.group <= 32 ? 128 : p.group;
  const long groups = p.group <= 32 ? p.threads / p.group : 1;
  p.blocks = std::min((d->rows + groups - 1) / groups, (long)ROWS_SMS * std::max(1, 1024 / p.threads));
  p.parts = p.V ? p.blocks : std::min((d->rows + WIDE_ROWS - 1) / WIDE_ROWS, WIDE_PARTS);
  return p;
}

}  // namespace

size_t rms_backward_part_bytes(const xconv_rows_desc* d) { return (size_t)plan_of(d).parts * (size_t)d->C * sizeof(float); }

cudaError_t launch_rms_backward(const xconv_rows_desc* d, const void* dY, const void* H, const float* rstd, const void* weight, const void* dH, void* dX, void* dR,
                                float* dweight, float* part, cudaStream_t st, int* launches) {
  const Plan p = plan_of(d);
  RmsBackArgs a = {};
  a.dY = dY; a.H = H; a.dH = dH; a.rstd = rstd; a.w = {weight, d->param_dtype == XCONV_F32}; a.dX = dX; a.dR = dR; a.part = part;
  a.rows = d->rows; a.sy = d->y_stride; a.sh = d->h_stride; a.sdh = d->dh_stride; a.sx = d->x_stride; a.sr = d->r_stride;
  a.C = d->C; a.octets = (d->C + 7) / 8; a.group = p.group; a.inv_c = 1.f / (float)d->C;
  a.drop = drop_of(d);
  const int n = d->dtype == XCONV_F32 ? 4 : 8;
  const bool vec = d->C % n == 0 && at(dY, 16) && at(H, 16) && at(dH, 16) && at(weight, 16) && at(dX, 16) && at(dR, 16) && d->y_stride % n == 0 && d->h_stride % n == 0 &&
                   (!dH || d->dh_stride % n == 0) && (!dX || d->x_stride % n == 0) && (!dR || d->r_stride % n == 0);
  if (d->rows > 0) {
    const cudaError_t e = with_type(d->dtype, [&](auto t) {
      using T = decltype(t);
      if (p.V || dX || dR) {
        const auto kernel = vec ? (p.V ? rms_backward_kernel<T, 1, true> : rms_backward_kernel<T, 0, true>) : (p.V ? rms_backward_kernel<T, 1, false> : rms_backward_kernel<T, 0, false>);
        const size_t smem = p.V && part && p.group <= 32 ? (size_t)(p.threads / 32) * d->C * sizeof(float) : 0;
        kernel<<<(unsigned)p.blocks, p.threads, smem, st>>>(a);
        ++*launches;
      }
      if (!p.V && part) {
        rms_columns_kernel<T><<<dim3((unsigned)((d->C + 255) / 256), (unsigned)p.parts), 256, 0, st>>>(a, (d->rows + p.parts - 1) / p.parts);
        ++*launches;
      }
      return cudaGetLastError();
    });
    if (e != cudaSuccess) return e;
  }
  if (!dweight) return cudaSuccess;
  ++*launches;
  return launch_pdl(rms_sums_kernel, dim3((unsigned)((d->C + 31) / 32)), dim3(1024), 0, st, (const float*)part, (int)p.parts, (int)d->C, dweight);
}

}  // namespace xconv
