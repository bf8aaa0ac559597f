// What the kernels on rows share: eight neighbouring values of a row (an octet: what one Philox block decides about) as floats, the mask, sums over a row.
#pragma once

#include <type_traits>

#include "../common.cuh"
#include "rows.h"

namespace xconv {

constexpr int ROWS_SMS = 148;

// ---- octets

// VEC: rows and pointers are at 16-byte boundaries, and C is a multiple of 16 bytes' values: accesses of 16 bytes; element by element otherwise.
// Values from C on are zeros, and are not written.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int c, int C, float (&f)[8]) {
  if constexpr (!VEC) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = c + e < C ? to_f(row[c + e]) : 0.f;
  } else if constexpr (sizeof(T) == 4) {
    const float4 u = *reinterpret_cast<const float4*>(row + c);
    const float4 v = c + 4 < C ? *reinterpret_cast<const float4*>(row + c + 4) : make_float4(0.f, 0.f, 0.f, 0.f);
    f[0] = u.x; f[1] = u.y; f[2] = u.z; f[3] = u.w; f[4] = v.x; f[5] = v.y; f[6] = v.z; f[7] = v.w;
  } else {
    const uint4 u = *reinterpret_cast<const uint4*>(row + c);
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
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* row, int c, int C, const float (&f)[8]) {
  if constexpr (!VEC) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < C) row[c + e] = from_f<T>(f[e]);
  } else if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(row + c) = make_float4(f[0], f[1], f[2], f[3]);
    if (c + 4 < C) *reinterpret_cast<float4*>(row + c + 4) = make_float4(f[4], f[5], f[6], f[7]);
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
    *reinterpret_cast<uint4*>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// A weight of floats, or of the activations' type.
struct Weight {
  const void* p;                   // null: ones
  int f32;
  template <typename T, bool VEC>
  __device__ __forceinline__ void load(int c, int C, float (&f)[8]) const {
    if (!p) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = 1.f;
    } else if (sizeof(T) == 4 || f32) {
      load8<float, VEC>(static_cast<const float*>(p), c, C, f);
    } else {
      load8<T, VEC>(static_cast<const T*>(p), c, C, f);
    }
  }
};

// ---- the mask

struct Drop {
  uint32_t bound, last;            // T - 1 of the header's T: its upper half with all bits below it set, and its lower half
  uint32_t k0, k1;
  const unsigned long long* add;
  float scale;                     // 1 / (1 - p)
  int on;
  long per;                        // rows of a mask row
  // the key, when the kernel runs
  __device__ __forceinline__ uint2 key() const {
    if (!add) return make_uint2(k0, k1);
    const unsigned long long s = ((unsigned long long)k1 << 32 | k0) + *add;
    return make_uint2((uint32_t)s, (uint32_t)(s >> 32));
  }
  __device__ __forceinline__ long mask_row(long row) const { return per == 1 ? row : row / per; }
};

// What the mask leaves of an octet.  dropped where u <= T - 1: decided by the upper halves, except where one equals T - 1's, which about one octet of 8192 meets: then
// the lower halves are drawn too.
__device__ __forceinline__ void drop8(const Drop& d, uint2 key, unsigned long long block, float (&f)[8]) {
  const uint4 u = philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), key.x, key.y, 3u);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  const uint32_t top = d.bound >> 16, twice = top * 0x10001u;
  uint32_t tie = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = w[i] ^ twice;
    tie |= (x - 0x00010001u) & ~x & 0x80008000u;             // a half of zeros
  }
  bool gone[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    gone[2 * i] = (w[i] << 16) <= d.bound;
    gone[2 * i + 1] = w[i] <= d.bound;
  }
  if (tie && d.last != 0xffffu) {
    const uint4 lower = philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), key.x, key.y, 4u);
    const uint32_t l[4] = {lower.x, lower.y, lower.z, lower.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if ((w[i] & 0xffffu) == top) gone[2 * i] = (l[i] & 0xffffu) <= d.last;
      if ((w[i] >> 16) == top) gone[2 * i + 1] = (l[i] >> 16) <= d.last;
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = gone[e] ? 0.f : f[e] * d.scale;
}

// ---- over the threads of a row: `group` of them, a power of two up to 32, or all of the block

// buf: 32 entries that no thread uses before the next barrier but one.
__device__ __forceinline__ float row_sum(float v, int group, float* buf) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < group) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (group <= 32) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = lane < (group >> 5) ? buf[lane] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// (of magnitudes by their bits: a NaN is above all)
__device__ __forceinline__ uint32_t row_max(uint32_t v, int group, uint32_t* buf) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < group) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  if (group <= 32) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = lane < (group >> 5) ? buf[lane] : 0u;
  return __reduce_max_sync(0xffffffffu, v);
}

// ---- host side

inline bool at(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline int pow2_from(long n) { int p = 1; while (p < n) p *= 2; return p; }

inline Drop drop_of(const xconv_rows_desc* d) {
  Drop r = {};
  const unsigned long long T = (unsigned long long)(d->p * 4294967296.0);
  r.per = d->rows_per_mask;
  r.on = T > 0;
  if (!r.on) return r;
  const uint32_t t = (uint32_t)(T - 1);
  r.bound = t | 0xffffu; r.last = t & 0xffffu;
  r.k0 = (uint32_t)d->seed; r.k1 = (uint32_t)(d->seed >> 32);
  r.add = d->seed_add;
  r.scale = d->p < 1.0 ? (float)(1.0 / (1.0 - d->p)) : 0.f;
  return r;
}
// f(T()) with the type of the activations.
template <typename F>
cudaError_t with_type(int dtype, F&& f) {
  if (dtype == XCONV_F32) return f(float());
  return dtype == XCONV_BF16 ? f(bf16()) : f(f16());
}

}  // namespace xconv
