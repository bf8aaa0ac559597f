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
// What keeps the memory busy are asynchronous copies: persistent blocks fetch the next rows of their threads into shared memory while they work on these ones, each
// thread its own 16-byte pieces, so that no thread waits for another's.  Dense rows that do not begin on 16-byte boundaries (odd channel counts) are fetched and
// written as runs of several rows that do, and picked apart in shared memory.  Other rows (some of the channels of a wider tensor, at odd offsets) are read element by
// element; rows that do not fit the registers of a block are read again for every sum.
//
// Measured (B200, copy rate 6.55 TB/s; launches replayed from a graph): forward, 200704 rows of 128 bfloat16 values, 103 MB, 19.0 us = 5.4 TB/s (a sum of two tensors
// moving as much takes 17.4); backward, 8192 rows of 4096 bfloat16 values, 201 MB, 46 us = 4.4 TB/s, of which the sums of the columns 2; issue slots 52 % busy, one
// block of 512 threads with 126 registers an SM, whose sums over a row nothing covers (two rows at once: 65 us; a barrier a group instead of the block's: 56).  47250
// rows of 97 float16 values by runs: forward 10.3, backward 15.3 us (one value at a time 12.0 and 20.0).  One row: 2.6 us, a launch.
#include "layer_norm.h"

#include <algorithm>
#include <type_traits>

#include "common.cuh"

namespace xconv {

namespace {

constexpr int NORM_SMS = 148;
constexpr int NORM_THREADS = 512;            // of a block whose threads hold the row

template <typename T> constexpr int VEC_OF = 16 / (int)sizeof(T);

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
__device__ __forceinline__ void copy16_async(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// ... or 16 bytes of zeros.
__device__ __forceinline__ void copy16_async_if(uint32_t dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Two values of 16 bits in a word.
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t u) {
  if constexpr (std::is_same<T, bf16>::value) return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
  else return __half22float2(*reinterpret_cast<const __half2*>(&u));
}
template <typename T>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  if constexpr (std::is_same<T, bf16>::value) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    const __half2 v = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&v);
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
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < group)
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
#pragma unroll
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
  int C, group, shift, run;        // group = 2^shift threads a row; rows of a run
  float eps, inv_c;
};

// Two values an instruction where a piece has an even number of them.
struct Pair {
  float2 v;
  template <int VEC> static __device__ __forceinline__ Pair of(const float (&x)[VEC], int i) { return {VEC > 1 ? make_float2(x[i], x[i + 1]) : make_float2(x[0], 0.f)}; }
  template <int VEC> __device__ __forceinline__ void to(float (&x)[VEC], int i) const { x[i] = v.x; if (VEC > 1) x[i + (VEC > 1)] = v.y; }
};
template <int VEC> __device__ __forceinline__ Pair add(Pair a, Pair b) { return {VEC > 1 ? __fadd2_rn(a.v, b.v) : make_float2(a.v.x + b.v.x, 0.f)}; }
template <int VEC> __device__ __forceinline__ Pair mul(Pair a, Pair b) { return {VEC > 1 ? __fmul2_rn(a.v, b.v) : make_float2(a.v.x * b.v.x, 0.f)}; }
template <int VEC> __device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c) { return {VEC > 1 ? __ffma2_rn(a.v, b.v, c.v) : make_float2(fmaf(a.v.x, b.v.x, c.v.x), 0.f)}; }
__device__ __forceinline__ Pair both(float x) { return {make_float2(x, x)}; }

// Whether every thread of a row has a v-th vector: V is the least number of vectors that reaches all of the row (see `vectors`).
template <int V> __device__ __forceinline__ constexpr bool all_have(int v) { return v < (V <= 8 ? V - 1 : V == 12 ? 8 : 12); }

// A row's values less their mean in x, and y's factor.  FULL: every thread of the row has V whole vectors.
struct NormAll { __device__ __forceinline__ constexpr bool operator()(int, int) const { return true; } };
template <int VEC, int V, bool FULL, class Has = NormAll>
__device__ __forceinline__ void norm_row(const NormArgs& a, int lane, float (&x)[V][VEC], float& mean, float& rstd, float (*sums)[32][1], Has has = Has()) {
  constexpr int STEP = VEC > 1 ? 2 : 1;
  Pair t = both(0.f);
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < VEC; e += STEP) t = add<VEC>(t, Pair::of(x[v], e));
  float s[1] = {t.v.x + t.v.y};
  if (VEC == 1) s[0] = t.v.x;
  group_sum<1>(s, a.group, sums[0]);
  mean = s[0] * a.inv_c;
  t = both(0.f);
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (FULL || all_have<V>(v) || (lane + v * a.group) * VEC < a.C)
#pragma unroll
      for (int e = 0; e < VEC; e += STEP) {
        Pair d = add<VEC>(Pair::of(x[v], e), both(-mean));
        if (!has(v, e)) d.v.x = 0.f;
        if (VEC > 1 && !has(v, e + 1)) d.v.y = 0.f;
        d.to(x[v], e);
        t = fma<VEC>(d, d, t);
      }
  s[0] = VEC == 1 ? t.v.x : t.v.x + t.v.y;
  group_sum<1>(s, a.group, sums[1]);
  rstd = rsqrtf(fmaf(s[0], a.inv_c, a.eps));
}
template <typename P, int VEC, int V>
__device__ __forceinline__ void norm_params(const NormArgs& a, int lane, float (&w)[V][VEC], float (&b)[V][VEC]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = (lane + v * a.group) * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) { w[v][e] = 1.f; b[v][e] = 0.f; }
    if (a.weight && c < a.C) load_params<P, VEC>(static_cast<const P*>(a.weight) + c, w[v]);
    if (a.bias && c < a.C) load_params<P, VEC>(static_cast<const P*>(a.bias) + c, b[v]);
  }
}
// The gradients of a row (x and dy of it; dy becomes dx), and its part of dw and db.  has: which of the thread's values are the row's; x and dy are zeros elsewhere.
template <int VEC, int V, bool FULL, class Has = NormAll>
__device__ __forceinline__ void norm_row_backward(const NormArgs& a, int lane, float mean, float rstd, float (&x)[V][VEC], float (&dy)[V][VEC],
                                                  const float (&w)[V][VEC], float (&dw)[V][VEC], float (&db)[V][VEC], float (*sums)[2], Has has = Has()) {
  constexpr int STEP = VEC > 1 ? 2 : 1;
  Pair t0 = both(0.f), t1 = both(0.f);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (!FULL && !all_have<V>(v) && (lane + v * a.group) * VEC >= a.C) continue;
#pragma unroll
    for (int e = 0; e < VEC; e += STEP) {
      // (a row that is not there is zeros, with a mean and rstd of zero)
      Pair h = mul<VEC>(add<VEC>(Pair::of(x[v], e), both(-mean)), both(rstd));
      const Pair d = Pair::of(dy[v], e);
      // (mean * rstd may be beyond the floats where x - mean is not)
      if (!has(v, e)) h.v.x = 0.f;
      if (VEC > 1 && !has(v, e + 1)) h.v.y = 0.f;
      fma<VEC>(d, h, Pair::of(dw[v], e)).to(dw[v], e);
      add<VEC>(d, Pair::of(db[v], e)).to(db[v], e);
      const Pair g = mul<VEC>(d, Pair::of(w[v], e));
      t0 = add<VEC>(t0, g);
      t1 = fma<VEC>(g, h, t1);
      h.to(x[v], e);
      g.to(dy[v], e);
    }
  }
  float s[2] = {VEC == 1 ? t0.v.x : t0.v.x + t0.v.y, VEC == 1 ? t1.v.x : t1.v.x + t1.v.y};
  group_sum<2>(s, a.group, sums);
  const Pair m0 = both(-s[0] * a.inv_c), m1 = both(-s[1] * a.inv_c), r = both(rstd);
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < VEC; e += STEP) mul<VEC>(r, fma<VEC>(Pair::of(x[v], e), m1, add<VEC>(Pair::of(dy[v], e), m0))).to(dy[v], e);
}
// The block's sums of dw and db, over its groups: those of a warp by shuffles, the warps' (or the groups' of several warps) side by side in shared memory, then
// column by column in order.  cols: 2 C floats for each team of a warp, or of a group of several.  APART: the groups' columns are not the same (`odd` less than a
// multiple of VEC): every group is a team.
template <int VEC, int V, bool APART = false>
__device__ __forceinline__ void norm_block_sums(const NormArgs& a, int lane, float (&dw)[V][VEC], float (&db)[V][VEC], float* cols, int odd = 0) {
  const int width = APART ? 32 : min(a.group, 32), team = APART ? threadIdx.x >> a.shift : threadIdx.x / max(a.group, 32);
  const int teams = APART ? blockDim.x >> a.shift : blockDim.x / max(a.group, 32);
  for (int o = width; o < 32; o <<= 1)
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        dw[v][e] += __shfl_xor_sync(0xffffffffu, dw[v][e], o);
        db[v][e] += __shfl_xor_sync(0xffffffffu, db[v][e], o);
      }
  __syncthreads();                                         // (the memory held rows before)
  if ((threadIdx.x & 31) < width)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = (lane + v * a.group) * VEC - odd;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if (c + e < 0 || c + e >= a.C) continue;
        cols[(size_t)team * 2 * a.C + c + e] = dw[v][e];
        cols[(size_t)team * 2 * a.C + a.C + c + e] = db[v][e];
      }
    }
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * a.C; c += blockDim.x) {
    float s = cols[c];
    for (int t = 1; t < teams; ++t) s += cols[(size_t)t * 2 * a.C + c];
    a.part[(size_t)blockIdx.x * 2 * a.C + c] = s;
  }
}

// Rows whose pieces are aligned (VEC > 1), fetched STAGES - 1 rows ahead, or read as they come (VEC = 1).  A group's rows: from its number on, every gridDim.x * groups-th.
template <typename T, typename P, int VEC, int V, int STAGES, bool FULL>
__global__ void __launch_bounds__(NORM_THREADS) norm_forward_kernel(const NormArgs a) {
  extern __shared__ uint4 ring[];
  __shared__ float sums[2][32][1];
  const int lane = threadIdx.x & (a.group - 1), groups = blockDim.x >> a.shift, apart = a.group * VEC;      // apart: of a thread's vectors
  const int step = (int)gridDim.x * groups;
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring + threadIdx.x), slot = blockDim.x * 16;
  const uint4* own = ring + threadIdx.x;
  long row = (long)blockIdx.x * groups + (threadIdx.x >> a.shift);
  int left = (int)(a.rows - row), ahead = left;              // rows from this one (the next one fetched) on
  const T *from = static_cast<const T*>(a.X) + row * a.sx + lane * VEC, *at = from;
  T* to = static_cast<T*>(a.Y) + row * a.sy + lane * VEC;
  const long from_step = step * a.sx, to_step = step * a.sy;
  const auto fetch = [&](int stage) {
    if (VEC > 1) {
      // (what is not there is fetched as zeros: the rows' arithmetic asks for nothing)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const bool in = ahead > 0 && (FULL || all_have<V>(v) || lane * VEC + v * apart < a.C);
        copy16_async_if(mine + (uint32_t)(stage * V + v) * slot, in ? from + v * apart : static_cast<const T*>(a.X), in);
      }
      copies_commit();
      from += from_step;
      ahead -= step;
    }
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) fetch(i);
  float w[V][VEC], b[V][VEC];
  norm_params<P, VEC, V>(a, lane, w, b);
  int blocks_left = (int)(a.rows - (long)blockIdx.x * groups);     // (the same in all threads of the block)
  while (blocks_left > 0) {
#pragma unroll
    for (int stage = 0; stage < STAGES; ++stage) {
      if (blocks_left <= 0) break;
      if (VEC > 1) copies_wait<(STAGES > 1 ? STAGES - 2 : 0)>();
      float x[V][VEC];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (VEC > 1) {
          load_elems<T, VEC>(reinterpret_cast<const T*>(own + (size_t)(stage * V + v) * blockDim.x), x[v]);
        } else if (left > 0 && (all_have<V>(v) || lane * VEC + v * apart < a.C)) {
          load_elems<T, VEC>(at + v * apart, x[v]);
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) x[v][e] = 0.f;
        }
      }
      fetch((stage + STAGES - 1) % STAGES);
      float mean, rstd;
      norm_row<VEC, V, FULL>(a, lane, x, mean, rstd, sums);
      if (left > 0) {
        if (lane == 0 && a.mean) { a.mean[row] = mean; a.rstd[row] = rstd; }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (!FULL && !all_have<V>(v) && lane * VEC + v * apart >= a.C) continue;
#pragma unroll
          for (int e = 0; e < VEC; e += VEC > 1 ? 2 : 1) fma<VEC>(mul<VEC>(Pair::of(x[v], e), both(rstd)), Pair::of(w[v], e), Pair::of(b[v], e)).to(x[v], e);
          store_elems<T, VEC>(to + v * apart, x[v]);
        }
      }
      row += step; left -= step; blocks_left -= step; to += to_step;
      if (VEC == 1) at += from_step;
    }
  }
}

template <typename T, typename P, int VEC, int V, int STAGES, bool FULL>
__global__ void __launch_bounds__(NORM_THREADS) norm_backward_kernel(const NormArgs a) {
  extern __shared__ uint4 ring[];
  __shared__ float sums[2][32][2];
  const int lane = threadIdx.x & (a.group - 1), groups = blockDim.x >> a.shift, apart = a.group * VEC;
  const int step = (int)gridDim.x * groups;
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring + threadIdx.x), slot = blockDim.x * 16;
  const uint4* own = ring + threadIdx.x;
  long row = (long)blockIdx.x * groups + (threadIdx.x >> a.shift);
  int left = (int)(a.rows - row), ahead = left;
  const T *from = static_cast<const T*>(a.X) + row * a.sx + lane * VEC, *at = from, *from_dy = static_cast<const T*>(a.dY) + row * a.sy + lane * VEC, *at_dy = from_dy;
  T* to = static_cast<T*>(a.dX) + row * a.sdx + lane * VEC;
  const long x_step = step * a.sx, dy_step = step * a.sy, to_step = step * a.sdx;
  const auto fetch = [&](int stage) {
    if (VEC > 1) {
      if (ahead > 0)
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (FULL || all_have<V>(v) || lane * VEC + v * apart < a.C) {
            copy16_async(mine + (uint32_t)(stage * 2 * V + 2 * v) * slot, from + v * apart);
            copy16_async(mine + (uint32_t)(stage * 2 * V + 2 * v + 1) * slot, from_dy + v * apart);
          }
      copies_commit();
      from += x_step; from_dy += dy_step;
      ahead -= step;
    }
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) fetch(i);
  float dw[V][VEC], db[V][VEC], w[V][VEC];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int c = lane * VEC + v * apart;
#pragma unroll
    for (int e = 0; e < VEC; ++e) { dw[v][e] = db[v][e] = 0.f; w[v][e] = 1.f; }
    if (a.weight && c < a.C) load_params<P, VEC>(static_cast<const P*>(a.weight) + c, w[v]);
  }
  float next_mean = left > 0 ? __ldg(a.mean + row) : 0.f, next_rstd = left > 0 ? __ldg(a.rstd + row) : 0.f;
  int blocks_left = (int)(a.rows - (long)blockIdx.x * groups);
  int turn = 0;
  while (blocks_left > 0) {
#pragma unroll
    for (int stage = 0; stage < STAGES; ++stage) {
      if (blocks_left <= 0) break;
      const float mean = next_mean, rstd = next_rstd;
      next_mean = next_rstd = 0.f;
      if (left > step) { next_mean = __ldg(a.mean + row + step); next_rstd = __ldg(a.rstd + row + step); }
      if (VEC > 1) copies_wait<(STAGES > 1 ? STAGES - 2 : 0)>();
      float x[V][VEC], dy[V][VEC];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (left > 0 && (FULL || all_have<V>(v) || lane * VEC + v * apart < a.C)) {
          if (VEC > 1) {
            load_elems<T, VEC>(reinterpret_cast<const T*>(own + (size_t)(stage * 2 * V + 2 * v) * blockDim.x), x[v]);
            load_elems<T, VEC>(reinterpret_cast<const T*>(own + (size_t)(stage * 2 * V + 2 * v + 1) * blockDim.x), dy[v]);
          } else {
            load_elems<T, VEC>(at + v * apart, x[v]);
            load_elems<T, VEC>(at_dy + v * apart, dy[v]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) x[v][e] = dy[v][e] = 0.f;
        }
      }
      fetch((stage + STAGES - 1) % STAGES);
      norm_row_backward<VEC, V, FULL>(a, lane, mean, rstd, x, dy, w, dw, db, sums[turn]);
      turn ^= 1;
      if (left > 0)
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (FULL || all_have<V>(v) || lane * VEC + v * apart < a.C) store_elems<T, VEC>(to + v * apart, dy[v]);
      row += step; left -= step; blocks_left -= step; to += to_step;
      if (VEC == 1) { at += x_step; at_dy += dy_step; }
    }
  }
  pdl_trigger();
  if (a.part) norm_block_sums<VEC, V>(a, lane, dw, db, reinterpret_cast<float*>(ring));
}

// ---- dense rows that are not aligned: runs of `a.run` rows, whose bytes are a multiple of 16, through shared memory

// The run from `first` on into (or from) shared memory, `count` values; what is left behind the last whole 16 bytes (the last run) one by one.
template <typename T>
__device__ __forceinline__ void run_fetch(uint32_t dst, T* at, const T* from, long count) {
  constexpr int VEC = VEC_OF<T>;
  const long whole = count / VEC;
  for (long i = threadIdx.x; i < whole; i += blockDim.x) copy16_async(dst + (uint32_t)i * 16, from + i * VEC);
  for (long i = whole * VEC + threadIdx.x; i < count; i += blockDim.x) at[i] = from[i];
}
template <typename T>
__device__ __forceinline__ void run_store(T* to, const T* at, long count) {
  constexpr int VEC = VEC_OF<T>;
  const long whole = count / VEC;
  for (long i = threadIdx.x; i < whole; i += blockDim.x) reinterpret_cast<uint4*>(to)[i] = reinterpret_cast<const uint4*>(at)[i];
  for (long i = whole * VEC + threadIdx.x; i < count; i += blockDim.x) to[i] = at[i];
}

constexpr int RUN_STAGES = 4;

// W values a word: two of 16 bits.  A row of an odd number of values then begins within a word where its number is odd -- as its group's number is, runs being
// multiples of eight rows and groups even in number -- and a thread's columns are the same in all its rows: one less than in the even ones.
template <typename T, typename P, int W, int V, bool BACKWARD>
__global__ void __launch_bounds__(NORM_THREADS, BACKWARD ? 1 : 2) norm_runs_kernel(const NormArgs a) {
  extern __shared__ uint4 ring[];
  __shared__ __align__(16) float sums[2][32][2], sum1[2][32][1];
  const int lane = threadIdx.x & (a.group - 1), groups = blockDim.x >> a.shift, own = threadIdx.x >> a.shift;
  const int odd = W == 2 ? own & a.C & 1 : 0;              // values of the row before in the row's first word
  const long runs = (a.rows + a.run - 1) / a.run;
  const size_t run_values = (size_t)a.run * a.C, run_pieces = run_values / VEC_OF<T>;
  const T *X = static_cast<const T*>(a.X), *dY = static_cast<const T*>(a.dY);
  T* out = static_cast<T*>(BACKWARD ? a.dX : a.Y);
  constexpr int TENSORS = BACKWARD ? 2 : 1;
  long ahead = blockIdx.x;
  const auto fetch = [&](int stage) {
    if (ahead < runs) {
      const long first = ahead * a.run, count = min((long)a.run, a.rows - first) * a.C;
      uint4* at = ring + (size_t)stage * TENSORS * run_pieces;
      run_fetch<T>((uint32_t)__cvta_generic_to_shared(at), reinterpret_cast<T*>(at), X + first * a.C, count);
      if (BACKWARD) run_fetch<T>((uint32_t)__cvta_generic_to_shared(at + run_pieces), reinterpret_cast<T*>(at + run_pieces), dY + first * a.C, count);
    }
    copies_commit();
    ahead += gridDim.x;
  };
#pragma unroll
  for (int i = 0; i < RUN_STAGES - 1; ++i) fetch(i);
  // Columns of a thread's v-th word, and whether the row has them: all of it but the first word's first value (odd) and the last words.
  const auto column = [&](int v) { return (lane + v * a.group) * W - odd; };
  const auto has = [&](int v, int k) {
    const int c = column(v) + k;
    return (v > 0 || W == 1 || k > 0 || c >= 0) && (all_have<V>(v) || c < a.C);
  };
  float w[V][W], b[V][W], dw[V][W], db[V][W];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < W; ++k) {
      w[v][k] = a.weight && has(v, k) ? to_f(static_cast<const P*>(a.weight)[column(v) + k]) : 1.f;
      b[v][k] = a.bias && has(v, k) ? to_f(static_cast<const P*>(a.bias)[column(v) + k]) : 0.f;
      dw[v][k] = db[v][k] = 0.f;
    }
  const auto read = [&](const T* row, bool in, float (&f)[V][W]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (W == 2) {
        float2 t = make_float2(0.f, 0.f);
        if (in && (has(v, 0) || has(v, 1))) t = unpack2<T>(*reinterpret_cast<const uint32_t*>(row + column(v)));
        f[v][0] = has(v, 0) ? t.x : 0.f;
        f[v][1] = has(v, 1) ? t.y : 0.f;
      } else {
        f[v][0] = in && has(v, 0) ? to_f(row[column(v)]) : 0.f;
      }
    }
  };
  const auto write = [&](T* row, const float (&f)[V][W]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (W == 2) {
        const uint32_t t = pack2<T>(f[v][0], f[v][1]);
        T* at = row + column(v);
        if (has(v, 0) && has(v, 1)) *reinterpret_cast<uint32_t*>(at) = t;
        else if (has(v, 0)) *reinterpret_cast<unsigned short*>(at) = (unsigned short)t;
        else if (has(v, 1)) *reinterpret_cast<unsigned short*>(at + 1) = (unsigned short)(t >> 16);
      } else if (has(v, 0)) {
        row[column(v)] = from_f<T>(f[v][0]);
      }
    }
  };
  int stage = 0, turn = 0;
  for (long i = blockIdx.x; i < runs; i += gridDim.x) {
    copies_wait<RUN_STAGES - 2>();
    __syncthreads();
    T *xs = reinterpret_cast<T*>(ring + (size_t)stage * TENSORS * run_pieces), *ds = reinterpret_cast<T*>(ring + ((size_t)stage * TENSORS + 1) * run_pieces);
    const long first = i * a.run, here = min((long)a.run, a.rows - first);
    for (int r0 = 0; r0 < a.run; r0 += groups, turn ^= 1) {
      const int r = r0 + own;
      const bool in = r < here;
      float x[V][W];
      read(xs + r * a.C, in, x);
      if constexpr (BACKWARD) {
        float dy[V][W];
        read(ds + r * a.C, in, dy);
        const float mean = in ? __ldg(a.mean + first + r) : 0.f, rstd = in ? __ldg(a.rstd + first + r) : 0.f;
        norm_row_backward<W, V, true>(a, lane, mean, rstd, x, dy, w, dw, db, sums[turn], has);
        if (in) write(xs + r * a.C, dy);
      } else {
        float mean, rstd;
        norm_row<W, V, true>(a, lane, x, mean, rstd, sum1, has);
        if (in) {
          if (lane == 0 && a.mean) { a.mean[first + r] = mean; a.rstd[first + r] = rstd; }
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int k = 0; k < W; k += W) fma<W>(mul<W>(Pair::of(x[v], k), both(rstd)), Pair::of(w[v], k), Pair::of(b[v], k)).to(x[v], k);
          write(xs + r * a.C, x);
        }
      }
    }
    __syncthreads();
    run_store<T>(out + first * a.C, xs, here * a.C);
    // (the stage before this one was written out before the barrier above: its memory takes the next run)
    fetch(stage == 0 ? RUN_STAGES - 1 : stage - 1);
    stage = stage == RUN_STAGES - 1 ? 0 : stage + 1;
  }
  if constexpr (BACKWARD) {
    pdl_trigger();
    copies_wait<0>();
    if (a.part) norm_block_sums<W, V, W == 2>(a, lane, dw, db, reinterpret_cast<float*>(ring), odd);
  }
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

// Vectors a thread for which there is a kernel: at least `v`, or 0.  (Sixteen values: five times as many floats fit a thread's registers.)
int vectors(long v, bool vec, bool words, int es) {
  if (words) return v <= 8 ? (int)v : 0;
  if (vec) return v <= (es == 4 ? 4 : 2) ? (int)v : 0;
  return v <= 8 ? (int)v : v <= 12 ? 12 : v <= 16 ? 16 : 0;
}
// Threads a row and vectors a thread: as few idle ones as possible, then rather many vectors a thread, but eight threads that read one line where the row has
// them.
void pick_group(long nv, int es, NormPlan* p) {
  long best = -1;
  for (int g = 1; g <= NORM_THREADS; g *= 2) {
    const int v = vectors((nv + g - 1) / g, p->vec, p->words, es);
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
  a.rows = d->rows; a.C = d->C; a.sx = d->x_stride; a.sy = d->y_stride; a.sdx = d->dx_stride; a.eps = d->eps; a.inv_c = 1.f / (float)d->C; a.group = p.group; a.run = p.run;
  while ((1 << a.shift) < p.group) ++a.shift;
  return a;
}

// Shared memory of a launch at most: 192 KB of ring, 200 KB of runs, 64 KB of columns' sums.
constexpr int NORM_SMEM_MAX = 200 * 1024;

template <typename K>
cudaError_t norm_launch(K kernel, const NormPlan& p, const NormArgs& a, cudaStream_t st) {
  if (p.smem > 40 * 1024) {
    // (the same for every size, so that no other thread finds it lowered)
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, NORM_SMEM_MAX);
    if (e != cudaSuccess) return e;
  }
  kernel<<<dim3((unsigned)p.blocks), dim3(p.threads), p.smem, st>>>(a);
  return cudaGetLastError();
}
// Vectors a thread fetches ahead: as many as the plan's shared memory is made for (plan_ring).
constexpr int norm_stages(int V, int VEC, bool backward) { return VEC == 1 ? 1 : backward ? (V == 1 ? 6 : V == 2 ? 4 : 3) : V == 1 ? 8 : V == 2 ? 6 : 4; }

template <typename T, typename P, int VEC>
cudaError_t forward_of(const NormPlan& p, const NormArgs& a, cudaStream_t st) {
  if constexpr (VEC == 1) {
    if constexpr (sizeof(T) == 2) {
#define XC_NORM(N) if (p.V == N && p.words) return norm_launch(norm_runs_kernel<T, P, 2, N, false>, p, a, st);
      XC_NORM(1) XC_NORM(2) XC_NORM(3) XC_NORM(4) XC_NORM(5) XC_NORM(6) XC_NORM(7) XC_NORM(8)
#undef XC_NORM
    }
#define XC_NORM(N) if (p.V == N && p.run) return norm_launch(norm_runs_kernel<T, P, 1, N, false>, p, a, st);
    XC_NORM(1) XC_NORM(2) XC_NORM(3) XC_NORM(4) XC_NORM(5) XC_NORM(6) XC_NORM(7) XC_NORM(8) XC_NORM(12) XC_NORM(16)
#undef XC_NORM
  }
#define XC_NORM(N) if (p.V == N) return p.full ? norm_launch(norm_forward_kernel<T, P, VEC, N, norm_stages(N, VEC, false), (VEC > 1)>, p, a, st) : norm_launch(norm_forward_kernel<T, P, VEC, N, norm_stages(N, VEC, false), false>, p, a, st);
  XC_NORM(1) XC_NORM(2)
  if constexpr (VEC <= 4) { XC_NORM(3) XC_NORM(4) }
  if constexpr (VEC == 1) { XC_NORM(5) XC_NORM(6) XC_NORM(7) XC_NORM(8) XC_NORM(12) XC_NORM(16) }
#undef XC_NORM
  return cudaErrorInvalidValue;
}
template <typename T, typename P, int VEC>
cudaError_t backward_of(const NormPlan& p, const NormArgs& a, cudaStream_t st) {
  if constexpr (VEC == 1) {
    if constexpr (sizeof(T) == 2) {
#define XC_NORM(N) if (p.V == N && p.words) return norm_launch(norm_runs_kernel<T, P, 2, N, true>, p, a, st);
      XC_NORM(1) XC_NORM(2) XC_NORM(3) XC_NORM(4) XC_NORM(5) XC_NORM(6) XC_NORM(7) XC_NORM(8)
#undef XC_NORM
    }
#define XC_NORM(N) if (p.V == N && p.run) return norm_launch(norm_runs_kernel<T, P, 1, N, true>, p, a, st);
    XC_NORM(1) XC_NORM(2) XC_NORM(3) XC_NORM(4) XC_NORM(5) XC_NORM(6) XC_NORM(7) XC_NORM(8) XC_NORM(12) XC_NORM(16)
#undef XC_NORM
  }
#define XC_NORM(N) if (p.V == N) return p.full ? norm_launch(norm_backward_kernel<T, P, VEC, N, norm_stages(N, VEC, true), (VEC > 1)>, p, a, st) : norm_launch(norm_backward_kernel<T, P, VEC, N, norm_stages(N, VEC, true), false>, p, a, st);
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

// Rows that a block of norm_columns_wide_kernel adds, at least, and partial sums at most: with the header in front 4 KB of scratch memory a channel.
constexpr long WIDE_ROWS = 64, WIDE_PARTS = 511;

}  // namespace

// What the threads and blocks are: `vec` by pieces of 16 bytes; `dense` rows without gaps from a 16-byte boundary on, which go by runs where they are not `vec`.
static NormPlan plan(const xconv_norm_desc* d, bool vec, bool dense, bool backward) {
  NormPlan p = {};
  p.vec = vec;
  const int es = d->dtype == XCONV_F32 ? 4 : 2, tensors = backward ? 2 : 1;
  const long nv = vec ? d->C / (16 / es) : d->C;
  // (words of two values, where a block has several groups)
  if (!vec && dense && es == 2) {
    p.words = true;
    pick_group(d->C / 2 + 1, es, &p);
    p.words = !p.wide && p.group <= 128 && RUN_STAGES * (size_t)tensors * std::max(256 / p.group, 8) * d->C * es <= (size_t)NORM_SMEM_MAX;
  }
  if (!p.words) pick_group(nv, es, &p);
  if (p.wide) {
    p.threads = 1024;
    p.parts = std::min<long>((d->rows + WIDE_ROWS - 1) / WIDE_ROWS, WIDE_PARTS);
    p.blocks = std::min<long>(d->rows, (backward ? 2 : 8) * NORM_SMS);
    return p;
  }
  if (!backward && !p.words && d->rows * p.group < NORM_SMS * 256L) {    // few rows: a thread has little to do, and more of them do it
    p.group = std::min(NORM_THREADS, pow2_at_least(nv));
    p.V = vectors((nv + p.group - 1) / p.group, vec, false, es);
  }
  p.full = vec && (long)p.V * p.group == nv;
  // A block's threads: fewer where its rows would not reach all SMs.
  p.threads = NORM_THREADS;
  while (p.threads > std::max(p.group, 128) && d->rows * p.group < (long)NORM_SMS * p.threads) p.threads /= 2;
  const long groups = p.threads / p.group;
  const int resident = vec || backward ? 1 : 2;              // of 512 threads: 128 or 64 registers each
  p.blocks = std::min<long>((d->rows + groups - 1) / groups, (long)NORM_SMS * resident * (NORM_THREADS / p.threads));
  const size_t stages = norm_stages(p.V, vec ? 2 : 1, backward);
  if (!vec && dense) p.threads = p.words ? 256 : std::max(p.group, std::min(p.threads, 256));
  if (vec) p.smem = (int)(stages * p.V * tensors * p.threads * 16);
  else if (dense) {
    const long groups = p.threads / p.group, run = std::max<long>(groups, 8);              // (8 rows of any type are a multiple of 16 bytes)
    const size_t bytes = RUN_STAGES * (size_t)tensors * run * d->C * es;
    if (bytes <= (size_t)NORM_SMEM_MAX) {
      p.run = (int)run;
      p.smem = (int)bytes;
      p.blocks = std::min<long>((d->rows + run - 1) / run, (long)NORM_SMS * std::max<long>(1, std::min<long>(resident * (NORM_THREADS / p.threads), 220 * 1024 / ((long)bytes + 2048))));
    }
  }
  if (backward) p.smem = std::max(p.smem, (int)(p.threads / (p.words ? p.group : std::max(p.group, 32)) * 2 * sizeof(float)) * d->C);
  p.parts = p.blocks;
  return p;
}
static bool is_dense(const xconv_norm_desc* d, int64_t s0, int64_t s1, int64_t s2) { return s0 == d->C && s1 == d->C && s2 == d->C; }

NormPlan plan_norm_forward(const xconv_norm_desc* d, const void* X, const void* weight, const void* bias, const void* Y) {
  const bool at16 = aligned(X, 16) && aligned(Y, 16);
  const bool vec = at16 && vec_fits(d, [&](int n) { return d->x_stride % n == 0 && d->y_stride % n == 0 && aligned(weight, 16) && aligned(bias, 16); });
  return plan(d, vec, at16 && is_dense(d, d->x_stride, d->y_stride, d->C), false);
}

NormPlan plan_norm_backward(const xconv_norm_desc* d, const void* dY, const void* X, const void* weight, const void* dX) {
  const bool at16 = aligned(X, 16) && aligned(dY, 16) && aligned(dX, 16);
  const bool vec = at16 && vec_fits(d, [&](int n) { return d->x_stride % n == 0 && d->y_stride % n == 0 && d->dx_stride % n == 0 && aligned(weight, 16); });
  return plan(d, vec, at16 && is_dense(d, d->x_stride, d->y_stride, d->dx_stride), true);
}
long norm_backward_parts(const xconv_norm_desc* d) {         // (of any pointers and strides)
  long most = std::max(plan(d, false, false, true).parts, plan(d, false, true, true).parts);
  return vec_fits(d, [](int) { return true; }) ? std::max(most, plan(d, true, false, true).parts) : most;
}

cudaError_t launch_norm_forward(const xconv_norm_desc* d, const NormPlan& p, const void* X, const void* weight, const void* bias, void* Y, float* mean, float* rstd,
                                cudaStream_t st) {
  NormArgs a = args_of(d, p);
  a.X = X; a.weight = weight; a.bias = bias; a.Y = Y; a.mean = mean; a.rstd = rstd;
  return with_types(d, [&](auto t, auto w) {
    using T = decltype(t); using P = decltype(w);
    if (p.wide) { norm_forward_wide_kernel<T, P><<<(unsigned)p.blocks, 1024, 0, st>>>(a); return cudaGetLastError(); }
    return p.vec ? forward_of<T, P, VEC_OF<T>>(p, a, st) : forward_of<T, P, 1>(p, a, st);
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
    return p.vec ? backward_of<T, P, VEC_OF<T>>(p, a, st) : backward_of<T, P, 1>(p, a, st);
  });
}
cudaError_t launch_norm_sums(const xconv_norm_desc* d, const float* part, long parts, float* dweight, float* dbias, cudaStream_t st) {
  return launch_pdl(norm_sums_kernel, dim3((unsigned)((2L * d->C + 31) / 32)), dim3(1024), 0, st, part, parts, (int)d->C, dweight, dbias);
}

}  // namespace xconv
