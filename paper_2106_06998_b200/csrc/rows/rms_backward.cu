// Gradients of the RMS norm, of the residual's addition and of the dropout in front of it.
//
//   xh = h rstd,  g = dy w,  dr = dh + rstd (g - xh sum(g xh) / C),  dx = drop'(dr),  dw = sum over rows of dy xh
//
// Memory bounds it: dy, h (and dh) are read once, dr (and dx) written once.  The threads of a block keep the same columns from row to row and carry dw in registers; blocks
// leave a partial sum a column each, which a second kernel adds in fixed order (no atomics: the same bits every time).
//
// Measured (B200, copy rate 6.57 TB/s; replayed from a graph, with dh): 8192 x 4096 bf16, 268 MB, 47.0 us = 5.7 TB/s, of which the columns' sums 3; 8192 x 4096 floats 87.7 us
// = 6.1 TB/s; 131072 x 128 bf16 26 us, with one octet a thread 30.  Registers (126 a thread) hold 512 threads an SM, whose loads for the next row are on their way during a sum.
// One cluster of eight blocks that adds its own sums (a launch less) was slower wherever rows take more than two rounds (1568 x 96 floats 7.0 us, 4.2 by two kernels).
#include "rms.h"
#include "rows.cuh"

namespace xconv {

namespace {

struct RmsBackArgs {
  Rows dY, H, dH, dX, dR;
  const float* rstd;
  Weight w;
  float* part;
  long rows;
  int C, octets, group;
  float inv_c;
  Drop drop;
};

// xh and g of an octet from what was fetched of h and dy, and its part of dw.
template <typename T, bool VEC>
__device__ __forceinline__ void weigh(const RmsBackArgs& a, const Fetched<T, VEC>& fh, const Fetched<T, VEC>& fy, int k, bool in, float rstd,
                                      const float (&w)[8], float (&xh)[8], float (&g)[8], float (&dw)[8]) {
  values_of<T, VEC>(fh, 8 * k, a.C, in, xh);
  values_of<T, VEC>(fy, 8 * k, a.C, in, g);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    xh[e] *= rstd;
    dw[e] = fmaf(g[e], xh[e], dw[e]);
    g[e] *= w[e];
  }
}
// dr, and dx, of an octet.
template <typename T, bool VEC, int DROP>
__device__ __forceinline__ void write_out(const RmsBackArgs& a, uint2 key, unsigned long long block, T* dR, T* dX, const Fetched<T, VEC>& fd, int k, bool in, float rstd, float mean,
                                          const float (&xh)[8], const float (&g)[8]) {
  float d[8];
  if (a.dH.p) {
    values_of<T, VEC>(fd, 8 * k, a.C, in, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = fmaf(rstd, fmaf(-xh[e], mean, g[e]), d[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = rstd * fmaf(-xh[e], mean, g[e]);
  }
  if (a.dR.p) store8<T, VEC>(dR, 8 * k, a.C, in, d);
  if (a.dX.p) {
    if (DROP) {
      bool gone[8];
      mask8(a.drop, key, block + k, gone);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = gone[e] ? 0.f : d[e] * a.drop.scale;
    }
    store8<T, VEC>(dX, 8 * k, a.C, in, d);
  }
}

// ---- rows in registers, V octets a thread; the next row is fetched while this one is worked on

template <typename T, int V, bool VEC, int DROP>
__global__ void __launch_bounds__(512) rms_backward_kernel(const RmsBackArgs a) {
  extern __shared__ __align__(16) float cols[];                            // C floats a warp, in a block of several groups
  __shared__ float sums[2][32];
  const int group = a.group, lane = group <= 32 ? threadIdx.x & (group - 1) : threadIdx.x;
  const int groups = group <= 32 ? blockDim.x / group : 1, own = group <= 32 ? threadIdx.x / group : 0;
  pdl_wait();
  const uint2 key = a.drop.key<DROP>();
  const long step = (long)gridDim.x * groups;
  long row = (long)blockIdx.x * groups + own;
  Walk<T> hs(a.H, row, step), dy(a.dY, row, step), dh(a.dH, row, step), dr(a.dR, row, step), dx(a.dX, row, step);
  Fetched<T, VEC> fh[V], fy[V], fd[V];
  float next_rstd = 0.f;
  const auto fetch = [&](long next) {
    const bool in = next < a.rows;
    next_rstd = in ? a.rstd[next] : 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int k = lane + v * group;
      fetch8<T, VEC>(a.H, hs.row, next, 8 * k, a.C, in && k < a.octets, fh[v]);
      fetch8<T, VEC>(a.dY, dy.row, next, 8 * k, a.C, in && k < a.octets, fy[v]);
      if (a.dH.p) fetch8<T, VEC>(a.dH, dh.row, next, 8 * k, a.C, in && k < a.octets, fd[v]);
    }
    hs.next(); dy.next(); dh.next();
  };
  fetch(row);
  float dw[V][8], w[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[v][e] = 0.f;
    a.w.load<T, VEC>(8 * min(lane + v * group, a.octets - 1), a.C, w[v]);
  }
  int turn = 0;
  for (long row0 = (long)blockIdx.x * groups; row0 < a.rows; row0 += step, row += step, turn ^= 1, dr.next(), dx.next()) {
    const bool in = row < a.rows;
    const float rstd = next_rstd;
    float xh[V][8], g[V][8], s = 0.f;
    Fetched<T, VEC> d[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int k = lane + v * group;
      weigh<T, VEC>(a, fh[v], fy[v], k, in && k < a.octets, rstd, w[v], xh[v], g[v], dw[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(g[v][e], xh[v][e], s);
      d[v] = fd[v];
    }
    fetch(row + step);
    const float mean = row_sum(s, group, sums[turn]) * a.inv_c;
    const unsigned long long block = DROP ? a.drop.first_block(row, a.octets) : 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int k = lane + v * group;
      write_out<T, VEC, DROP>(a, key, block, dr.out(), dx.out(), d[v], k, in && k < a.octets, rstd, mean, xh[v], g[v]);
    }
  }
  pdl_trigger();
  if (!a.part) return;
  // The groups of a warp by shuffles, the warps side by side in shared memory, then column by column in order.
  for (int o = group; o < 32; o <<= 1)
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) dw[v][e] += __shfl_xor_sync(0xffffffffu, dw[v][e], o);
  const bool several = group <= 32;
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  float* to = several ? cols + warp * a.C : a.part + (size_t)blockIdx.x * a.C;
  if ((threadIdx.x & 31) < group)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = 8 * (lane + v * group);
      if (VEC && a.C % 4 == 0) {
#pragma unroll
        for (int e = 0; e < 8; e += 4)
          if (c + e < a.C) *reinterpret_cast<float4*>(to + c + e) = make_float4(dw[v][e], dw[v][e + 1], dw[v][e + 2], dw[v][e + 3]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < a.C) to[c + e] = dw[v][e];
      }
    }
  if (!several) return;
  __syncthreads();
  for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
    float t = cols[c];
    for (int i = 1; i < warps; ++i) t += cols[i * a.C + c];
    a.part[(size_t)blockIdx.x * a.C + c] = t;
  }
}

// ---- 16-bit rows that take four octets a thread: of what a thread keeps only h, dy and dh stay in its registers, as they came; xh and g are made twice, the weight and dw lie in shared
// memory, every thread's own in a place of their own, and the next row's octets are fetched one by one as this row's are written.  4096 x 12288 bf16 with dh 97 us = 4.2 TB/s (floor 61),
// with dropout 127; all in registers of which most then lie in local memory 209, with 32 registers a thread 780; rows read again for the second step 199.

constexpr int LONG_V = 4, LONG_SMEM = 512 * LONG_V * 2 * 8 * 4;

template <typename T, int DROP>
__global__ void __launch_bounds__(512, 1) rms_backward_long_kernel(const RmsBackArgs a) {
  extern __shared__ __align__(16) float cols[];
  __shared__ float sums[2][32];
  float4* const own = reinterpret_cast<float4*>(cols) + threadIdx.x;
  const int group = blockDim.x;
  const auto lay = [&](int v, const float (&f)[8]) {                          // v: the octet, or LONG_V and more: of dw
    own[2 * v * group] = make_float4(f[0], f[1], f[2], f[3]);
    own[(2 * v + 1) * group] = make_float4(f[4], f[5], f[6], f[7]);
  };
  const auto take = [&](int v, float (&f)[8]) {
    const float4 x = own[2 * v * group], y = own[(2 * v + 1) * group];
    f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w; f[4] = y.x; f[5] = y.y; f[6] = y.z; f[7] = y.w;
  };
  pdl_wait();
  const uint2 key = a.drop.key<DROP>();
  Fetched<T, true> fh[LONG_V], fy[LONG_V], fd[LONG_V];
  const auto fetch = [&](long row, int v) {
    const int k = threadIdx.x + v * group;
    const bool in = row < a.rows && k < a.octets;
    fetch8<T, true>(a.H, row_of<T>(a.H, row), row, 8 * k, a.C, in, fh[v]);
    fetch8<T, true>(a.dY, row_of<T>(a.dY, row), row, 8 * k, a.C, in, fy[v]);
    if (a.dH.p) fetch8<T, true>(a.dH, row_of<T>(a.dH, row), row, 8 * k, a.C, in, fd[v]);
  };
  float w[8], dw[8], xh[8], g[8];
  float next_rstd = a.rstd[blockIdx.x];
#pragma unroll
  for (int v = 0; v < LONG_V; ++v) {
    fetch(blockIdx.x, v);
    a.w.load<T, true>(8 * min((int)threadIdx.x + v * group, a.octets - 1), a.C, w);
    lay(v, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[e] = 0.f;
    lay(LONG_V + v, dw);
  }
  int turn = 0;
  for (long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const float rstd = next_rstd;
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < LONG_V; ++v) {
      const int k = threadIdx.x + v * group;
      take(v, w);
      take(LONG_V + v, dw);
      weigh<T, true>(a, fh[v], fy[v], k, k < a.octets, rstd, w, xh, g, dw);
      lay(LONG_V + v, dw);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(g[e], xh[e], s);
    }
    const long next = row + gridDim.x;
    if (next < a.rows) next_rstd = a.rstd[next];
    const float mean = row_sum(s, group, sums[turn]) * a.inv_c;
    const unsigned long long block = DROP ? a.drop.first_block(row, a.octets) : 0;
#pragma unroll
    for (int v = 0; v < LONG_V; ++v) {
      const int k = threadIdx.x + v * group;
      take(v, w);
      weigh<T, true>(a, fh[v], fy[v], k, k < a.octets, rstd, w, xh, g, dw);     // (this dw is not kept)
      const Fetched<T, true> d = fd[v];
      fetch(next, v);
      write_out<T, true, DROP>(a, key, block, const_cast<T*>(row_of<T>(a.dR, row)), const_cast<T*>(row_of<T>(a.dX, row)), d, k, k < a.octets, rstd, mean, xh, g);
    }
  }
  pdl_trigger();
  if (!a.part) return;
#pragma unroll
  for (int v = 0; v < LONG_V; ++v) {
    const int c = 8 * (threadIdx.x + v * group);
    take(LONG_V + v, dw);
    float* const to = a.part + (size_t)blockIdx.x * a.C + c;
    if (c < a.C) {
      reinterpret_cast<float4*>(to)[0] = make_float4(dw[0], dw[1], dw[2], dw[3]);
      reinterpret_cast<float4*>(to)[1] = make_float4(dw[4], dw[5], dw[6], dw[7]);
    }
  }
}

// ---- rows of any length, a block each, read again for the second step; dw is another kernel's

template <typename T, bool VEC, int DROP>
__global__ void __launch_bounds__(1024) rms_backward_wide_kernel(const RmsBackArgs a) {
  __shared__ float sums[2][32];
  pdl_wait();
  const uint2 key = a.drop.key<DROP>();
  const int steps = (a.octets + 1023) / 1024;
  int turn = 0;
  for (long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const float rstd = a.rstd[row];
    float xh[8], g[8], unused[8], s = 0.f;
    const auto read = [&](int k) {
      Fetched<T, VEC> fh, fy;
      fetch8<T, VEC>(a.H, row_of<T>(a.H, row), row, 8 * k, a.C, k < a.octets, fh);
      fetch8<T, VEC>(a.dY, row_of<T>(a.dY, row), row, 8 * k, a.C, k < a.octets, fy);
      float w[8];
      a.w.load<T, VEC>(8 * min(k, a.octets - 1), a.C, w);
      weigh<T, VEC>(a, fh, fy, k, k < a.octets, rstd, w, xh, g, unused);
    };
    for (int v = 0; v < steps; ++v) {
      read(threadIdx.x + v * 1024);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(g[e], xh[e], s);
    }
    const float mean = row_sum(s, 1024, sums[turn]) * a.inv_c;
    const unsigned long long block = DROP ? a.drop.first_block(row, a.octets) : 0;
    for (int v = 0; v < steps; ++v) {
      const int k = threadIdx.x + v * 1024;
      read(k);
      Fetched<T, VEC> fd;
      if (a.dH.p) fetch8<T, VEC>(a.dH, row_of<T>(a.dH, row), row, 8 * k, a.C, k < a.octets, fd);
      write_out<T, VEC, DROP>(a, key, block, const_cast<T*>(row_of<T>(a.dR, row)), const_cast<T*>(row_of<T>(a.dX, row)), fd, k, k < a.octets, rstd, mean, xh, g);
    }
  }
}

// dw of rows that no block holds: a thread a column, a block a run of rows.
template <typename T>
__global__ void __launch_bounds__(256) rms_columns_kernel(const RmsBackArgs a, long rows_per) {
  pdl_wait();
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.C) return;
  const long r0 = (long)blockIdx.y * rows_per, r1 = min(a.rows, r0 + rows_per);
  float dw = 0.f;
#pragma unroll 4
  for (long row = r0; row < r1; ++row)
    dw = fmaf(to_f(row_of<T>(a.dY, row)[c]), to_f(row_of<T>(a.H, row)[c]) * a.rstd[row], dw);
  a.part[(size_t)blockIdx.y * a.C + c] = dw;
}

// Columns' sums over the parts: 16 columns a block (VEC: four a thread), of which every thread adds every GROUPS-th part -- all loads in flight at once up to 640 parts, or 320 one column a thread: this
// kernel is a chain of waits for L2 -- then the threads' sums are added in order.  (No parts: zeros.)
template <bool VEC>
__global__ void __launch_bounds__(256) rms_sums_kernel(const float* part, int parts, int C, float* dweight) {
  constexpr int EACH = VEC ? 4 : 1, LANES = 16 / EACH, GROUPS = 256 / LANES, DEEP = VEC ? 10 : 20;
  __shared__ float sums[GROUPS][17];
  const int lane = threadIdx.x % LANES, g = threadIdx.x / LANES, c = blockIdx.x * 16 + lane * EACH;
  float own[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) own[e] = 0.f;
  pdl_wait();
  if (c < C)
    for (int first = g; first < parts; first += GROUPS * DEEP) {
      float v[DEEP][EACH];
#pragma unroll
      for (int i = 0; i < DEEP; ++i) {
        const int n = first + i * GROUPS;
        const float* at = part + (size_t)n * C + c;
        if constexpr (VEC) {
          const float4 t = n < parts ? __ldcg(reinterpret_cast<const float4*>(at)) : make_float4(0.f, 0.f, 0.f, 0.f);
          v[i][0] = t.x; v[i][1] = t.y; v[i][2] = t.z; v[i][3] = t.w;
        } else {
          v[i][0] = n < parts ? __ldcg(at) : 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < DEEP; ++i)
#pragma unroll
        for (int e = 0; e < EACH; ++e) own[e] += v[i][e];
    }
#pragma unroll
  for (int e = 0; e < EACH; ++e) sums[g][lane * EACH + e] = own[e];
  __syncthreads();
  // 16 threads a column
  const int col = threadIdx.x >> 4, t = threadIdx.x & 15;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < GROUPS / 16; ++i) s += sums[t + 16 * i][col];
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (t == 0 && blockIdx.x * 16 + col < C) dweight[blockIdx.x * 16 + col] = s;
}

// Rows that a block of rms_columns_kernel adds, at least, and partial sums at most.
constexpr long WIDE_ROWS = 64, WIDE_PARTS = 512;

struct Plan { Team team; long blocks, parts; };
Plan plan_of(const xconv_rows_desc* d, bool vec) {
  Plan p = {};
  p.team = team_of((d->C + 7) / 8, d->dtype == XCONV_F32 || !vec, vec && d->dtype != XCONV_F32);
  // (at most: 1024 threads of an SM)
  p.blocks = std::min((d->rows + p.team.groups - 1) / p.team.groups, (long)ROWS_SMS * std::max(1, 1024 / p.team.threads));
  p.parts = p.team.V ? p.blocks : std::min((d->rows + WIDE_ROWS - 1) / WIDE_ROWS, WIDE_PARTS);
  return p;
}

}  // namespace

size_t rms_backward_part_bytes(const xconv_rows_desc* d) { return (size_t)std::max({plan_of(d, true).parts, plan_of(d, false).parts, rms_staged_backward_parts(d)}) * (size_t)d->C * sizeof(float); }

cudaError_t launch_rms_backward(const xconv_rows_desc* d, const void* dY, const void* H, const float* rstd, const void* weight, const void* dH, void* dX, void* dR,
                                float* dweight, float* part, cudaStream_t st, int* launches) {
  RmsBackArgs a = {};
  const size_t es = d->dtype == XCONV_F32 ? 4 : 2;
  a.dY = rows_of(dY, d->rows, d->C, d->y_stride, es); a.H = rows_of(H, d->rows, d->C, d->h_stride, es); a.dH = rows_of(dH, d->rows, d->C, d->dh_stride, es);
  a.dX = rows_of(dX, d->rows, d->C, d->x_stride, es); a.dR = rows_of(dR, d->rows, d->C, d->r_stride, es);
  a.rstd = rstd; a.w = {weight, d->param_dtype == XCONV_F32}; a.part = part;
  a.rows = d->rows; a.C = d->C; a.octets = (d->C + 7) / 8; a.inv_c = 1.f / (float)d->C;
  a.drop = drop_of(d);
  const bool vec = d->C % (16 / es) == 0 && whole(a.dY, 16) && whole(a.H, 16) && whole(a.dH, 16) && whole(a.dX, 16) && whole(a.dR, 16) && at(weight, 16);
  const Plan p = plan_of(d, vec);
  a.group = p.team.group;
  long parts = p.parts;
  if (d->rows > 0) {
    cudaError_t e;
    if (!vec && rms_staged_backward(d, dY, H, rstd, weight, dH, dX, dR, part, &parts, st, &e)) ++*launches;
    else e = with_type(d->dtype, [&](auto t) {
      using T = decltype(t);
      const int V = p.team.V;
      cudaError_t e = cudaSuccess;
      if (V || dX || dR) {
        const auto pick = [&](auto v, auto dropped) -> void (*)(const RmsBackArgs) {
          constexpr bool VEC = decltype(v)::value;
          constexpr int DROP = decltype(dropped)::value;
          if constexpr (VEC && sizeof(T) == 2)
            if (V == LONG_V) return rms_backward_long_kernel<T, DROP>;
          return V == 0 ? rms_backward_wide_kernel<T, VEC, DROP> : V == 1 ? rms_backward_kernel<T, 1, VEC, DROP> : rms_backward_kernel<T, 2, VEC, DROP>;
        };
        const auto kernel = with_kinds(vec, a.dX.p ? a.drop.how : DROP_NONE, pick);
        const size_t smem = V == LONG_V ? (size_t)p.team.threads * LONG_V * 2 * 8 * sizeof(float) : V && part && p.team.group <= 32 ? (size_t)(p.team.threads / 32) * d->C * sizeof(float) : 0;
        if (V == LONG_V) {
          e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LONG_SMEM);
          if (e != cudaSuccess) return e;
        }
        const long blocks = std::min(p.blocks, (long)ROWS_SMS * resident_blocks(kernel, p.team.threads, (int)smem));
        if (V) parts = blocks;
        e = launch_pdl(kernel, dim3((unsigned)blocks), dim3(p.team.threads), smem, st, a);
        ++*launches;
      }
      if (e == cudaSuccess && !V && part) {
        e = launch_pdl(rms_columns_kernel<T>, dim3((unsigned)((d->C + 255) / 256), (unsigned)p.parts), dim3(256), 0, st, a, (d->rows + p.parts - 1) / p.parts);
        ++*launches;
      }
      return e;
    });
    if (e != cudaSuccess) return e;
  }
  if (!dweight) return cudaSuccess;
  ++*launches;
  return launch_pdl(d->C % 4 == 0 ? rms_sums_kernel<true> : rms_sums_kernel<false>, dim3((unsigned)((d->C + 15) / 16)), dim3(256), 0, st, (const float*)part, (int)parts, (int)d->C, dweight);
}

}  // namespace xconv
