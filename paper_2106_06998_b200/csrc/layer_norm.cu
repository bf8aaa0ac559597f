// Layer norm over the channels of channels-last tensors: rows of C values (a pixel's channels, a token), forward and backward.
//
//   forward    y = (x - mean) rstd w + b,  mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps)
//   backward   with xh = (x - mean) rstd and g = dy w:
//              dx = rstd (g - sum g / C - xh sum (g xh) / C),  dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Memory bounds both: every input is read once and every output written once.  A row lies in the registers of `group` threads (up to 512 of them), so
// that the variance is the sum of squares about the mean that is known by then, not a difference of two large sums; all sums are float.  Backward, the threads of
// a block keep the same columns from row to row and carry the sums of dw and db in registers; blocks leave one partial sum a column each, which a second kernel
// adds in fixed order (no atomics: the same bits every time).
//
// Rows that are not aligned to 16 bytes are read element by element; rows that do not fit the registers of a block are read again for every sum.
#include "layer_norm.h"

#include <algorithm>
#include <type_traits>

#include "common.cuh"

namespace xconv {

namespace {

constexpr int NORM_SMS = 148;
constexpr int NORM_THREADS = 512;            // of a block whose threads hold the row

template <typename T> constexpr int vec_of() { return 16 / (int)sizeof(T); }

// VEC neighbouring elements as floats.
template <typename T, int VEC>
__device__ __forceinline__ void load_elems(const T* p, float (&f)[VEC]) {
  if constexpr (VEC == 1) {
    f[0] = to_f(*p);
  } else if constexpr (sizeof(T) == 4) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
  } else {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, bf16>::value) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        f[2 * i] = t.x; f[2 * i + 1] = t.y;
      }
    }
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_elems(T* p, const float (&f)[VEC]) {
  if constexpr (VEC == 1) {
    *p = from_f<T>(f[0]);
  } else if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, bf16>::value) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
      } else {
        const __half2 v = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
      }
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// VEC parameters (weight, bias): VEC elements of the activations are up to 32 bytes of them.
template <typename P, int VEC>
__device__ __forceinline__ void load_params(const P* p, float (&f)[VEC]) {
  if constexpr (VEC == 8 && sizeof(P) == 4) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
    load_elems<P, VEC>(p, f);
  }
}

// Sums over the `group` threads of a row, the same in each of them: within a warp by shuffles, across warps through shared memory (a buffer of
// blockDim.x / 32 entries that no one else uses before the next barrier but one).  All threads of the block take part.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], int group, float (*buf)[N]) {
  const int width = min(group, 32);
  for (int o = width >> 1; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if (group <= 32) return;
  const int warp = threadIdx.x >> 5, per = group >> 5;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) buf[warp][i] = v[i];
  __syncthreads();
  // (each warp adds the `per` sums by shuffles too: 32 of them at most)
  const int lane = threadIdx.x & 31, first = warp / per * per;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lane < per ? buf[first + lane][i] : 0.f;
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

struct NormArgs {
  const void *X, *dY, *weight, *bias;
  void *Y, *dX;
  float *mean, *rstd;              // (read by the backward pass)
  float* part;
  long rows, sx, sy, sdx;          // row strides in elements
  int C, group, shift;             // group = 2^shift threads a row
  float eps, inv_c;
};

template <typename T, typename P, int VEC, int V, int ROWS>
__global__ void __launch_bounds__(NORM_THREADS) norm_forward_kernel(const NormArgs a) {
  __shared__ float sums[2 * ROWS][32][1];
  const int group = a.group, lane = threadIdx.x & (group - 1);
  const long row0 = ((long)blockIdx.x * (blockDim.x >> a.shift) + (threadIdx.x >> a.shift)) * ROWS;
  const T* X = static_cast<const T*>(a.X);
  float x[ROWS][V][VEC];
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (lane + v * group) * VEC;
      if (c < a.C && row0 + r < a.rows) load_elems<T, VEC>(X + (row0 + r) * a.sx + c, x[r][v]);
      else
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[r][v][e] = 0.f;
    }
  float mean[ROWS], rstd[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    float s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < VEC; ++e) s[0] += x[r][v][e];
    group_sum<1>(s, group, sums[2 * r]);
    mean[r] = s[0] * a.inv_c;
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    float s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v)
      if ((lane + v * group) * VEC < a.C)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          x[r][v][e] -= mean[r];
          s[0] = fmaf(x[r][v][e], x[r][v][e], s[0]);
        }
    group_sum<1>(s, group, sums[2 * r + 1]);
    rstd[r] = 1.f / sqrtf(fmaf(s[0], a.inv_c, a.eps));
    if (lane == 0 && row0 + r < a.rows && a.mean) { a.mean[row0 + r] = mean[r]; a.rstd[row0 + r] = rstd[r]; }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (lane + v * group) * VEC;
    if (c >= a.C) continue;
    float w[VEC], b[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) { w[e] = 1.f; b[e] = 0.f; }
    if (a.weight) load_params<P, VEC>(static_cast<const P*>(a.weight) + c, w);
    if (a.bias) load_params<P, VEC>(static_cast<const P*>(a.bias) + c, b);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (row0 + r >= a.rows) continue;
      float y[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) y[e] = fmaf(x[r][v][e] * rstd[r], w[e], b[e]);
      store_elems<T, VEC>(static_cast<T*>(a.Y) + (row0 + r) * a.sy + c, y);
    }
  }
}

// Rows from blockIdx.x * groups on, every gridDim.x * groups-th: a thread has the same columns in all of them.
template <typename T, typename P, int VEC, int V>
__global__ void __launch_bounds__(NORM_THREADS) norm_backward_kernel(const NormArgs a) {
  extern __shared__ float cols[];                          // [2][C], for the sums over the block's groups
  __shared__ float sums[2][32][2];
  const int group = a.group, lane = threadIdx.x & (group - 1), groups = blockDim.x >> a.shift;
  const T *X = static_cast<const T*>(a.X), *dY = static_cast<const T*>(a.dY);
  float dw[V][VEC], db[V][VEC], w[V][VEC];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (lane + v * group) * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) { dw[v][e] = db[v][e] = 0.f; w[v][e] = 1.f; }
    if (a.weight && c < a.C) load_params<P, VEC>(static_cast<const P*>(a.weight) + c, w[v]);
  }
  int turn = 0;
  for (long base = (long)blockIdx.x * groups; base < a.rows; base += (long)gridDim.x * groups, turn ^= 1) {
    const long row = base + (threadIdx.x >> a.shift);
    const bool in = row < a.rows;
    float x[V][VEC], dy[V][VEC];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (lane + v * group) * VEC;
      if (in && c < a.C) {
        load_elems<T, VEC>(X + row * a.sx + c, x[v]);
        load_elems<T, VEC>(dY + row * a.sy + c, dy[v]);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[v][e] = dy[v][e] = 0.f;
      }
    }
    const float mean = in ? __ldg(a.mean + row) : 0.f, rstd = in ? __ldg(a.rstd + row) : 0.f;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!in || (lane + v * group) * VEC >= a.C) continue;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        x[v][e] = (x[v][e] - mean) * rstd;
        dw[v][e] = fmaf(dy[v][e], x[v][e], dw[v][e]);
        db[v][e] += dy[v][e];
        dy[v][e] *= w[v][e];
        s[0] += dy[v][e];
        s[1] = fmaf(dy[v][e], x[v][e], s[1]);
      }
    }
    group_sum<2>(s, group, sums[turn]);
    const float m0 = s[0] * a.inv_c, m1 = s[1] * a.inv_c;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (lane + v * group) * VEC;
      if (!in || c >= a.C) continue;
#pragma unroll
      for (int e = 0; e < VEC; ++e) dy[v][e] = rstd * (dy[v][e] - m0 - x[v][e] * m1);
      store_elems<T, VEC>(static_cast<T*>(a.dX) + row * a.sdx + c, dy[v]);
    }
  }
  if (!a.part) return;
  // The groups of a warp add up by shuffles, the warps (or the groups of several warps) one behind the other.
  const int width = min(group, 32), team = threadIdx.x / max(group, 32), teams = blockDim.x / max(group, 32);
  for (int o = width; o < 32; o <<= 1)
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        dw[v][e] += __shfl_xor_sync(0xffffffffu, dw[v][e], o);
        db[v][e] += __shfl_xor_sync(0xffffffffu, db[v][e], o);
      }
  const bool first = (threadIdx.x & 31) < width;
  for (int t = 0; t < teams; ++t) {
    if (t == team && first)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (lane + v * group) * VEC;
        if (c >= a.C) continue;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          cols[c + e] = dw[v][e] + (t ? cols[c + e] : 0.f);
          cols[a.C + c + e] = db[v][e] + (t ? cols[a.C + c + e] : 0.f);
        }
      }
    __syncthreads();
  }
  for (int c = threadIdx.x; c < 2 * a.C; c += blockDim.x) a.part[(size_t)blockIdx.x * 2 * a.C + c] = cols[c];
}

// ---- rows of any length, read from memory (or L2) for every sum; a block takes a row

template <typename T, typename P>
__global__ void __launch_bounds__(1024) norm_forward_wide_kernel(const NormArgs a) {
  __shared__ float sums[2][32][1];
  for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.X) + row * a.sx;
    float s[1] = {0.f};
    for (int c = threadIdx.x; c < a.C; c += 1024) s[0] += to_f(x[c]);
    group_sum<1>(s, 1024, sums[0]);
    const float mean = s[0] * a.inv_c;
    s[0] = 0.f;
    for (int c = threadIdx.x; c < a.C; c += 1024) { const float d = to_f(x[c]) - mean; s[0] = fmaf(d, d, s[0]); }
    group_sum<1>(s, 1024, sums[1]);
    const float rstd = 1.f / sqrtf(fmaf(s[0], a.inv_c, a.eps));
    if (threadIdx.x == 0 && a.mean) { a.mean[row] = mean; a.rstd[row] = rstd; }
    for (int c = threadIdx.x; c < a.C; c += 1024) {
      const float w = a.weight ? to_f(static_cast<const P*>(a.weight)[c]) : 1.f, b = a.bias ? to_f(static_cast<const P*>(a.bias)[c]) : 0.f;
      static_cast<T*>(a.Y)[row * a.sy + c] = from_f<T>(fmaf((to_f(x[c]) - mean) * rstd, w, b));
    }
  }
}
template <typename T, typename P>
__global__ void __launch_bounds__(1024) norm_backward_wide_kernel(const NormArgs a) {
  __shared__ float sums[2][32][2];
  int turn = 0;
  for (long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const T *x = static_cast<const T*>(a.X) + row * a.sx, *dy = static_cast<const T*>(a.dY) + row * a.sy;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s[2] = {0.f, 0.f};
    for (int c = threadIdx.x; c < a.C; c += 1024) {
      const float g = to_f(dy[c]) * (a.weight ? to_f(static_cast<const P*>(a.weight)[c]) : 1.f);
      s[0] += g;
      s[1] = fmaf(g, (to_f(x[c]) - mean) * rstd, s[1]);
    }
    group_sum<2>(s, 1024, sums[turn]);
    const float m0 = s[0] * a.inv_c, m1 = s[1] * a.inv_c;
    for (int c = threadIdx.x; c < a.C; c += 1024) {
      const float g = to_f(dy[c]) * (a.weight ? to_f(static_cast<const P*>(a.weight)[c]) : 1.f);
      static_cast<T*>(a.dX)[row * a.sdx + c] = from_f<T>(rstd * (g - m0 - (to_f(x[c]) - mean) * rstd * m1));
    }
  }
}
// dweight and dbias of wide rows: a thread a column, a block a run of rows.
template <typename T>
__global__ void __launch_bounds__(256) norm_columns_wide_kernel(const NormArgs a, long rows_per) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.C) return;
  const long r0 = (long)blockIdx.y * rows_per, r1 = min(a.rows, r0 + rows_per);
  float dw = 0.f, db = 0.f;
#pragma unroll 4
  for (long row = r0; row < r1; ++row) {
    const float dy = to_f(static_cast<const T*>(a.dY)[row * a.sy + c]);
    dw = fmaf(dy, (to_f(static_cast<const T*>(a.X)[row * a.sx + c]) - __ldg(a.mean + row)) * __ldg(a.rstd + row), dw);
    db += dy;
  }
  a.part[(size_t)blockIdx.y * 2 * a.C + c] = dw;
  a.part[(size_t)blockIdx.y * 2 * a.C + a.C + c] = db;
}

// Columns' sums over the parts, 32 columns a block: each of its warps adds every 32nd part, then the warps' sums are added in order.
__global__ void __launch_bounds__(1024) norm_sums_kernel(const float* part, long parts, int C, float* dweight, float* dbias) {
  __shared__ float sums[32][33];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long c = (long)blockIdx.x * 32 + lane;
  float own[4];
  if (c < 2L * C) sum_splits<32, 4, 4>(part + c, 2 * (size_t)C, warp, (int)parts, own);
  else own[0] = own[1] = own[2] = own[3] = 0.f;
  sums[warp][lane] = (own[0] + own[1]) + (own[2] + own[3]);
  __syncthreads();
  float s = sums[lane][warp];                              // (column `warp` of the block's 32)
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  const long col = (long)blockIdx.x * 32 + warp;
  if (lane == 0 && col < 2L * C) {
    if (col < C) { if (dweight) dweight[col] = s; }
    else if (dbias) dbias[col - C] = s;
  }
}

inline int pow2_at_least(long n) { int p = 1; while (p < n) p *= 2; return p; }
inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// Vectors a thread for which there is a kernel: at least `v`, or 0.
int vectors(long v, bool forward, bool vec, int es) {
  if (v <= 4) return v <= 2 || forward || es == 4 || !vec ? (int)v : 0;      // (backward, 16-bit: five times 16 floats a thread fit, not 32)
  if (vec) return forward && v <= 8 ? 8 : 0;
  return v <= 8 ? (int)v : v <= 12 ? 12 : v <= 16 ? 16 : 0;
}
// Threads a row and vectors a thread: as few idle ones as possible, then rather many vectors a thread, but eight threads that read one line where the row has
// them.
void pick_group(long nv, bool forward, int es, NormPlan* p) {
  long best = -1;
  for (int g = 1; g <= NORM_THREADS; g *= 2) {
    const int v = vectors((nv + g - 1) / g, forward, p->vec, es);
    if (v == 0) continue;
    const long slots = (long)v * g;
    if (best < 0 || (g <= 8 ? slots <= best : slots < best)) { best = slots; p->group = g; p->V = v; }
  }
  p->wide = best < 0;
  if (p->wide) { p->V = 1; p->group = 1024; }
}

template <typename F>
bool vec_fits(const xconv_norm_desc* d, F&& strides_and_pointers) {
  const int vec = d->dtype == XCONV_F32 ? 4 : 8;
  return d->C % vec == 0 && strides_and_pointers(vec);
}

NormArgs args_of(const xconv_norm_desc* d, const NormPlan& p) {
  NormArgs a = {};
  a.rows = d->rows; a.C = d->C; a.sx = d->x_stride; a.sy = d->y_stride; a.sdx = d->dx_stride; a.eps = d->eps; a.inv_c = 1.f / (float)d->C; a.group = p.group;
  while ((1 << a.shift) < p.group) ++a.shift;
  return a;
}

template <typename T, typename P, int VEC>
cudaError_t forward_of(const NormPlan& p, const NormArgs& a, cudaStream_t st) {
  const dim3 grid((unsigned)p.blocks), block(p.threads);
#define XC_NORM(N, R) if (p.V == N && p.rows_per == R) { norm_forward_kernel<T, P, VEC, N, R><<<grid, block, 0, st>>>(a); return cudaGetLastError(); }
  XC_NORM(1, 1) XC_NORM(1, 4) XC_NORM(2, 1) XC_NORM(2, 2) XC_NORM(3, 1) XC_NORM(4, 1) XC_NORM(8, 1)
  if constexpr (VEC == 1) { XC_NORM(5, 1) XC_NORM(6, 1) XC_NORM(7, 1) XC_NORM(12, 1) XC_NORM(16, 1) }
#undef XC_NORM
  return cudaErrorInvalidValue;
}
template <typename T, typename P, int VEC>
cudaError_t backward_of(const NormPlan& p, const NormArgs& a, cudaStream_t st) {
  const dim3 grid((unsigned)p.blocks), block(p.threads);
  const size_t smem = a.part ? 2 * sizeof(float) * (size_t)a.C : 0;
#define XC_NORM(N) \
  if (p.V == N) { \
    if (smem > 40 * 1024) { \
      const cudaError_t e = cudaFuncSetAttribute(norm_backward_kernel<T, P, VEC, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); \
      if (e != cudaSuccess) return e; \
    } \
    norm_backward_kernel<T, P, VEC, N><<<grid, block, smem, st>>>(a); \
    return cudaGetLastError(); \
  }
  XC_NORM(1) XC_NORM(2)
  if constexpr (VEC <= 4) { XC_NORM(3) XC_NORM(4) }
  if constexpr (VEC == 1) { XC_NORM(5) XC_NORM(6) XC_NORM(7) XC_NORM(8) XC_NORM(12) XC_NORM(16) }
#undef XC_NORM
  return cudaErrorInvalidValue;
}

// f(T, P) with the types of the activations and the parameters.
template <typename F>
cudaError_t with_types(const xconv_norm_desc* d, F&& f) {
  if (d->dtype == XCONV_F32) return f(float(), float());
  if (d->dtype == XCONV_BF16) return d->param_dtype == XCONV_F32 ? f(bf16(), float()) : f(bf16(), bf16());
  return d->param_dtype == XCONV_F32 ? f(f16(), float()) : f(f16(), f16());
}

constexpr long WIDE_ROWS = 64;                               // rows that a block of norm_columns_wide_kernel adds, at least

}  // namespace

NormPlan plan_norm_forward(const xconv_norm_desc* d, const void* X, const void* weight, const void* bias, const void* Y) {
  NormPlan p = {};
  p.vec = vec_fits(d, [&](int vec) {
    return d->x_stride % vec == 0 && d->y_stride % vec == 0 && aligned(X, 16) && aligned(Y, 16) && aligned(weight, 16) && aligned(bias, 16); });
  const long nv = p.vec ? d->C / (d->dtype == XCONV_F32 ? 4 : 8) : d->C;
  const int es = d->dtype == XCONV_F32 ? 4 : 2;
  pick_group(nv, true, es, &p);
  if (!p.wide && d->rows * p.group < NORM_SMS * 256L) {      // few rows: a thread has little to do, and more of them do it
    p.group = std::min(NORM_THREADS, pow2_at_least(nv));
    p.V = vectors((nv + p.group - 1) / p.group, true, p.vec, es);
  }
  p.threads = p.wide ? 1024 : std::max(p.group, 256);
  p.rows_per = 1;
  const long groups = p.threads / p.group;
  if (!p.wide && d->rows >= NORM_SMS * 8 * groups) p.rows_per = p.V == 1 ? 4 : p.V == 2 ? 2 : 1;
  p.blocks = p.wide ? std::min<long>(d->rows, 8 * NORM_SMS) : (d->rows + groups * p.rows_per - 1) / (groups * p.rows_per);
  return p;
}

// Blocks of the backward pass (each leaves a partial sum): as many as the SMs hold at once.
static NormPlan plan_backward(const xconv_norm_desc* d, bool vec) {
  NormPlan p = {};
  p.vec = vec;
  const long nv = vec ? d->C / (d->dtype == XCONV_F32 ? 4 : 8) : d->C;
  pick_group(nv, false, d->dtype == XCONV_F32 ? 4 : 2, &p);
  p.threads = p.wide ? 1024 : NORM_THREADS;
  const long groups = p.threads / p.group;
  p.blocks = std::min<long>((d->rows + groups - 1) / groups, NORM_SMS * (1024 / p.threads));
  if (p.wide) {
    const long chunks = std::min<long>((d->rows + WIDE_ROWS - 1) / WIDE_ROWS, 512);
    p.parts = chunks;
    p.blocks = std::min<long>(d->rows, 2 * NORM_SMS);
  } else {
    p.parts = p.blocks;
  }
  return p;
}
NormPlan plan_norm_backward(const xconv_norm_desc* d, const void* dY, const void* X, const void* weight, const void* dX) {
  return plan_backward(d, vec_fits(d, [&](int vec) {
    return d->x_stride % vec == 0 && d->y_stride % vec == 0 && d->dx_stride % vec == 0 && aligned(X, 16) && aligned(dY, 16) && aligned(dX, 16) && aligned(weight, 16); }));
}
long norm_backward_parts(const xconv_norm_desc* d) {
  const long a = plan_backward(d, false).parts;
  return vec_fits(d, [](int) { return true; }) ? std::max(a, plan_backward(d, true).parts) : a;
}

cudaError_t launch_norm_forward(const xconv_norm_desc* d, const NormPlan& p, const void* X, const void* weight, const void* bias, void* Y, float* mean, float* rstd,
                                cudaStream_t st) {
  NormArgs a = args_of(d, p);
  a.X = X; a.weight = weight; a.bias = bias; a.Y = Y; a.mean = mean; a.rstd = rstd;
  return with_types(d, [&](auto t, auto w) {
    using T = decltype(t); using P = decltype(w);
    if (p.wide) { norm_forward_wide_kernel<T, P><<<(unsigned)p.blocks, 1024, 0, st>>>(a); return cudaGetLastError(); }
    return p.vec ? forward_of<T, P, vec_of<T>()>(p, a, st) : forward_of<T, P, 1>(p, a, st);
  });
}
cudaError_t launch_norm_backward(const xconv_norm_desc* d, const NormPlan& p, const void* dY, const void* X, const float* mean, const float* rstd, const void* weight,
                                 void* dX, float* part, cudaStream_t st) {
  NormArgs a = args_of(d, p);
  a.X = X; a.dY = dY; a.weight = weight; a.dX = dX; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd); a.part = part;
  return with_types(d, [&](auto t, auto w) {
    using T = decltype(t); using P = decltype(w);
    if (p.wide) {
      norm_backward_wide_kernel<T, P><<<(unsigned)p.blocks, 1024, 0, st>>>(a);
      cudaError_t e = cudaGetLastError();
      if (e != cudaSuccess || !part) return e;
      const long rows_per = (d->rows + p.parts - 1) / p.parts;
      norm_columns_wide_kernel<T><<<dim3((unsigned)((d->C + 255) / 256), (unsigned)p.parts), 256, 0, st>>>(a, rows_per);
      return cudaGetLastError();
    }
    return p.vec ? backward_of<T, P, vec_of<T>()>(p, a, st) : backward_of<T, P, 1>(p, a, st);
  });
}
cudaError_t launch_norm_sums(const xconv_norm_desc* d, const float* part, long parts, float* dweight, float* dbias, cudaStream_t st) {
  return launch_pdl(norm_sums_kernel, dim3((unsigned)((2L * d->C + 31) / 32)), dim3(1024), 0, st, part, parts, (int)d->C, dweight, dbias);
}

}  // namespace xconv
