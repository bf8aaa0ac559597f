// What the kernels on rows share: eight neighbouring values of a row (an octet: what one Philox block decides about) as floats, the mask, sums over a row.
//
// All kernels of this folder may start while the kernel before them still runs: they wait for it before they read or write anything, and read nothing through the read-only cache.
// (A launch of that kind also costs the host half a microsecond less.)
#pragma once

#include <algorithm>
#include <type_traits>

#include "../common.cuh"
#include "rows.h"

namespace xconv {

constexpr int ROWS_SMS = 148;

// Division of numbers below 2^31 by one that is known before the launch: the high part of a product with ceil(2^(32 + l) / d) - 2^32, l = ceil(log2 d) (Granlund, Montgomery,
// "Division by invariant integers using multiplication", PLDI'94).
struct Divisor {
  uint32_t d, m, l;
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (__umulhi(m, n) + n) >> l; }
};
inline Divisor divisor(uint32_t d) {
  uint32_t l = 0;
  while ((1ull << l) < d) ++l;
  return {d, (uint32_t)(((1ull << 32) * ((1ull << l) - d)) / d + 1), l};
}

// ---- octets in memory

// A tensor's rows.  An octet is read in pieces of 16 bytes (of 8-bit values: 8) at their own boundaries, whatever the octet's alignment: those that hold one of its values,
// from which it is cut out by shifts -- the same ones for all octets of a row.  (Value by value that takes eight accesses, of lanes that are 16 bytes apart.)  A piece that reaches beyond
// the tensor's own bytes is read value by value.  VEC: every row begins on such a boundary, and C is a multiple of a piece's values.
struct Rows {
  const char* p;                   // null: no such tensor
  long stride;                     // bytes
  const char* end;                 // of its own bytes
  long inner;                      // rows but the first and the last one, where no piece of theirs can reach beyond the tensor's bytes
};

template <typename T>
struct Octet {
  static constexpr int WORDS = 2 * sizeof(T), PIECE = sizeof(T) == 1 ? 2 : 4, PER = 4 * PIECE / sizeof(T);      // words of an octet and of a piece, values of a piece
};
template <typename T, bool VEC>
struct Fetched {
  uint32_t w[Octet<T>::WORDS + (VEC ? 0 : Octet<T>::PIECE)];
  int shift;                       // (not VEC) values between the boundary before the row and the row
};

// ... as a pointer that moves on from row to row.
template <typename T>
struct Walk {
  const T* row;
  long step;                       // bytes
  __device__ __forceinline__ Walk(const Rows& t, long first, long rows) : row(reinterpret_cast<const T*>(t.p + first * t.stride)), step(rows * t.stride) {}
  __device__ __forceinline__ void next() { row = reinterpret_cast<const T*>(reinterpret_cast<const char*>(row) + step); }
  __device__ __forceinline__ T* out() const { return const_cast<T*>(row); }
};
template <typename T>
__device__ __forceinline__ const T* row_of(const Rows& t, long row) { return reinterpret_cast<const T*>(t.p + row * t.stride); }
// Values between the boundary before a row and the row.
template <typename T, bool VEC>
__device__ __forceinline__ int shift_of(const T* row) { return VEC ? 0 : (int)(reinterpret_cast<uintptr_t>(row) % (4 * Octet<T>::PIECE) / sizeof(T)); }

// The octet from value c on (a multiple of 8) of the n-th row, as its pieces lie in memory: pieces that are not needed (`in` false, or from C on) as zeros.
template <typename T, bool VEC>
__device__ __forceinline__ void fetch8(const Rows& t, const T* row, long n, int c, int C, bool in, Fetched<T, VEC>& f) {
  constexpr int PIECE = Octet<T>::PIECE, PER = Octet<T>::PER, PIECES = sizeof(f.w) / (4 * PIECE);
  f.shift = shift_of<T, VEC>(row);
  const char* at = reinterpret_cast<const char*>(row + (c - f.shift));
  const auto needed = [&](int i) { return in && (i == 0 || c - f.shift + i * PER < C) && (i + 1 < PIECES || VEC || f.shift + 8 > i * PER); };
  const auto whole = [&](int i) {
    uint32_t* w = f.w + PIECE * i;
    if constexpr (PIECE == 4) {
      const uint4 u = *reinterpret_cast<const uint4*>(at + 4 * PIECE * i);
      w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(at + 4 * PIECE * i);
      w[0] = u.x; w[1] = u.y;
    }
  };
#pragma unroll
  for (int i = 0; i < PIECES * PIECE; ++i) f.w[i] = 0u;
  if (VEC || (unsigned long)(n - 1) < (unsigned long)t.inner) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
      if (needed(i)) whole(i);
  } else {
    // (the first and the last row.  A branch of their own: with the question at every piece the others are 10 % slower)
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      if (!needed(i)) continue;
      const char* piece = at + 4 * PIECE * i;
      if (piece >= t.p && piece + 4 * PIECE <= t.end) {
        whole(i);
        continue;
      }
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const char* v = piece + e * sizeof(T);
        uint32_t* w = f.w + PIECE * i;
        if (v < t.p || v >= t.end) continue;
        if constexpr (sizeof(T) == 4) w[e] = *reinterpret_cast<const uint32_t*>(v);
        else if constexpr (sizeof(T) == 2) w[e / 2] |= (uint32_t)*reinterpret_cast<const unsigned short*>(v) << (16 * (e % 2));
        else w[e / 4] |= (uint32_t)*reinterpret_cast<const unsigned char*>(v) << (8 * (e % 4));
      }
    }
  }
}

// Word i + skip of the n words of w, for a skip of 0 to MOST (4 at most) that is known when the kernel runs; beyond them zeros.
template <int MOST, int n>
__device__ __forceinline__ uint32_t word_from(const uint32_t (&w)[n], int i, int skip) {
  const uint32_t x0 = i < n ? w[i < n ? i : 0] : 0u, x1 = i + 1 < n ? w[i + 1 < n ? i + 1 : 0] : 0u, x2 = i + 2 < n ? w[i + 2 < n ? i + 2 : 0] : 0u,
                 x3 = i + 3 < n ? w[i + 3 < n ? i + 3 : 0] : 0u, x4 = i + 4 < n ? w[i + 4 < n ? i + 4 : 0] : 0u;
  const uint32_t lo = skip & 1 ? x1 : x0, hi = skip & 1 ? x3 : x2;
  const uint32_t up = MOST < 2 ? lo : skip & 2 ? hi : lo;
  return MOST < 4 ? up : skip & 4 ? x4 : up;
}
// N words from byte `first` on (a multiple of the values' size, 4 MOST + 3 at most).
template <typename T, int MOST, int N, int M>
__device__ __forceinline__ void bytes_from(const uint32_t (&w)[M], int first, uint32_t (&out)[N]) {
  uint32_t a = word_from<MOST>(w, 0, first >> 2);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t b = sizeof(T) < 4 || i + 1 < N ? word_from<MOST>(w, i + 1, first >> 2) : 0u;
    out[i] = sizeof(T) == 4 ? a : __funnelshift_r(a, b, 8 * (first & 3));
    a = b;
  }
}
// The octet's own words.
template <typename T, bool VEC>
__device__ __forceinline__ void words_of(const Fetched<T, VEC>& f, uint32_t (&w)[Octet<T>::WORDS]) {
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < Octet<T>::WORDS; ++i) w[i] = f.w[i];
  } else {
    bytes_from<T, Octet<T>::PIECE - 1>(f.w, f.shift * (int)sizeof(T), w);
  }
}
template <typename T>
__device__ __forceinline__ void floats_of(const uint32_t (&w)[Octet<T>::WORDS], float (&f)[8]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(w[e]);
  } else {
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
template <typename T>
__device__ __forceinline__ void words_for(const float (&f)[8], uint32_t (&w)[Octet<T>::WORDS]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(f[e]);
  } else {
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
  }
}
// The octet's values as floats: zeros where `in` is false and from C on.  CLEAN = false: whatever, there.
template <typename T, bool VEC, bool CLEAN = true>
__device__ __forceinline__ void values_of(const Fetched<T, VEC>& f, int c, int C, bool in, float (&v)[8]) {
  uint32_t w[Octet<T>::WORDS];
  words_of<T, VEC>(f, w);
  if constexpr (CLEAN && !VEC) {                             // (VEC: pieces that are not there are zeros already)
    const int bits = in ? 8 * (int)sizeof(T) * min(8, C - c) : 0;
#pragma unroll
    for (int i = 0; i < Octet<T>::WORDS; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = bits > 32 * i ? w[i] : 0u;
      else w[i] = bits - 32 * i >= 32 ? w[i] : w[i] & ((1u << max(bits - 32 * i, 0)) - 1u);
    }
  }
  floats_of<T>(w, v);
}

// An octet to memory: values c to c + 7 of the row, those below C, of the lanes whose `in` says so.  Of rows at any alignment a lane writes the pieces from the boundary
// before its octet on that are full, the first with what the lane before it has of it; values that no such piece takes, at the ends of a row and of a warp, go one by one.  All lanes of
// the warp take part, and the octets of a row are those of neighbouring lanes.
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* row, int c, int C, bool in, const uint32_t (&w)[Octet<T>::WORDS]) {
  constexpr int N = Octet<T>::WORDS, PIECE = Octet<T>::PIECE, PER = Octet<T>::PER, PIECES = N / PIECE;
  const auto whole = [](T* to, const uint32_t* w) {
    if constexpr (PIECE == 4) *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
  };
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
      if (in && (i == 0 || c + i * PER < C)) whole(row + c + i * PER, w + PIECE * i);
  } else {
    uint32_t all[PIECE + N];                                 // a piece's worth of the lane before, and the octet
#pragma unroll
    for (int i = 0; i < PIECE; ++i) all[i] = __shfl_up_sync(0xffffffffu, w[N - PIECE + i], 1);
#pragma unroll
    for (int i = 0; i < N; ++i) all[PIECE + i] = w[i];
    if (!in) return;
    const int shift = shift_of<T, false>(row), lane = threadIdx.x & 31, m = C - c;      // (values from this one on: more than 8, but for the last octet)
    uint32_t out[N];                                         // from the boundary on
    bytes_from<T, PIECE>(all, 4 * PIECE - shift * (int)sizeof(T), out);
    // the octet's values that no piece takes, by bits: those of the i-th piece from the boundary on are PER of them from i PER - shift on
    uint32_t left = m >= 8 ? 0xffu : (1u << m) - 1u;
    T* to = row + c;
#pragma unroll
    for (int i = 0; i < PIECES + 1; ++i) {
      const uint32_t its = ((1u << PER) - 1u) << 8 << (i * PER) >> shift >> 8;
      // (the piece behind the last one is the next lane's first)
      const bool full = i < PIECES ? shift + m >= (i + 1) * PER && (i > 0 || (c > 0 && lane > 0)) : lane < 31 && shift + m - 8 >= PER;
      if (full) left &= ~its;
      if (i < PIECES && full) whole(to - shift + i * PER, out + PIECE * i);
    }
    if (left)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (!(left >> e & 1)) continue;
        if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(to + e) = w[e];
        else if constexpr (sizeof(T) == 2) *reinterpret_cast<unsigned short*>(to + e) = (unsigned short)(w[e / 2] >> (16 * (e % 2)));
        else *reinterpret_cast<unsigned char*>(to + e) = (unsigned char)(w[e / 4] >> (8 * (e % 4)));
      }
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* row, int c, int C, bool in, const float (&f)[8]) {
  uint32_t w[Octet<T>::WORDS];
  words_for<T>(f, w);
  store8<T, VEC>(row, c, C, in, w);
}

// A weight of floats, or of the activations' type; read value by value where it is not aligned as its rows are.
struct Weight {
  const void* p;                   // null: ones
  int f32;
  template <typename P, bool VEC>
  __device__ __forceinline__ void load_as(int c, int C, float (&f)[8]) const {
    const P* q = static_cast<const P*>(p) + c;
    if constexpr (VEC) {
      Fetched<P, true> t;
      const Rows r = {};
      fetch8<P, true>(r, static_cast<const P*>(p), 0, c, C, c < C, t);
      values_of<P, true>(t, c, C, c < C, f);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = c + e < C ? to_f(q[e]) : 0.f;
    }
  }
  template <typename T, bool VEC>
  __device__ __forceinline__ void load(int c, int C, float (&f)[8]) const {
    if (!p) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = 1.f;
    } else if (sizeof(T) == 4 || f32) {
      load_as<float, VEC>(c, C, f);
    } else {
      load_as<T, VEC>(c, C, f);
    }
  }
};

// ---- the mask

// How a kernel gets its key: no mask, from the host, or with a number in device memory (which the compiler does not know to be the same in all lanes: it keeps the rounds' keys
// in registers of each).
enum { DROP_NONE = 0, DROP_HOST = 1, DROP_DEVICE = 2 };

struct Drop {
  uint32_t bound, last;            // T - 1 of the header's T: its upper half with all bits below it set, and its lower half
  uint32_t k0, k1;
  const unsigned long long* add;
  float scale;                     // 1 / (1 - p)
  int how;
  Divisor per;                     // rows of a mask row
  template <int HOW>
  __device__ __forceinline__ uint2 key() const {
    if (HOW != DROP_DEVICE) return make_uint2(k0, k1);
    const unsigned long long s = ((unsigned long long)k1 << 32 | k0) + *add;
    return make_uint2((uint32_t)s, (uint32_t)(s >> 32));
  }
  __device__ __forceinline__ unsigned long long first_block(long row, int octets) const { return (unsigned long long)per((uint32_t)row) * (uint32_t)octets; }
};

// Which values of an octet are dropped: where u <= T - 1.  The upper halves decide, except where one equals T - 1's, which about one octet of 8192 meets: then the lower halves
// are drawn too.
__device__ __forceinline__ void mask8(const Drop& d, uint2 key, unsigned long long block, bool (&gone)[8]) {
  const uint4 u = philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), key.x, key.y, 3u);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  const uint32_t top = d.bound >> 16, twice = top * 0x10001u;
  // the least half of what differs: zero where one is the border
  const uint32_t off = __vminu2(__vminu2(w[0] ^ twice, w[1] ^ twice), __vminu2(w[2] ^ twice, w[3] ^ twice));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    gone[2 * i] = (w[i] << 16) <= d.bound;
    gone[2 * i + 1] = w[i] <= d.bound;
  }
  if (((off - 0x00010001u) & ~off & 0x80008000u) != 0 && d.last != 0xffffu) {
    const uint4 lower = philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), key.x, key.y, 4u);
    const uint32_t l[4] = {lower.x, lower.y, lower.z, lower.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if ((w[i] & 0xffffu) == top) gone[2 * i] = (l[i] & 0xffffu) <= d.last;
      if ((w[i] >> 16) == top) gone[2 * i + 1] = (l[i] >> 16) <= d.last;
    }
  }
}

// The same as bits of a byte: a value is kept where its half carries out of a sum with what the border lacks to 2^32, and the carries are taken into the byte as they come (34 cycles of an SM
// for the octets of a warp; by comparisons 47; 24 without the mask, ten rounds alone).
__device__ __forceinline__ uint32_t mask_bits(const Drop& d, uint2 key, unsigned long long block) {
  const uint4 u = philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), key.x, key.y, 3u);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  const uint32_t top = d.bound >> 16, twice = top * 0x10001u, lacks = ~d.bound;
  const uint32_t off = __vminu2(__vminu2(w[0] ^ twice, w[1] ^ twice), __vminu2(w[2] ^ twice, w[3] ^ twice));
  uint32_t kept = 0;
#pragma unroll
  for (int i = 3; i >= 0; --i) {
    asm("{.reg .u32 sum;\n\tadd.cc.u32 sum, %1, %2;\n\taddc.u32 %0, %0, %0;}" : "+r"(kept) : "r"(w[i]), "r"(lacks));
    asm("{.reg .u32 sum;\n\tadd.cc.u32 sum, %1, %2;\n\taddc.u32 %0, %0, %0;}" : "+r"(kept) : "r"(w[i] << 16), "r"(lacks));
  }
  uint32_t b = kept ^ 0xffu;
  if (((off - 0x00010001u) & ~off & 0x80008000u) != 0 && d.last != 0xffffu) {
    const uint4 lower = philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), key.x, key.y, 4u);
    const uint32_t l[4] = {lower.x, lower.y, lower.z, lower.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if ((w[i] & 0xffffu) == top) b = (b & ~(1u << 2 * i)) | ((l[i] & 0xffffu) <= d.last ? 1u << 2 * i : 0u);
      if ((w[i] >> 16) == top) b = (b & ~(2u << 2 * i)) | ((l[i] >> 16) <= d.last ? 2u << 2 * i : 0u);
    }
  }
  return b;
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
// ---- host side

// The rows of a tensor of `size` bytes a value.
inline Rows rows_of(const void* p, long rows, int C, long stride, size_t size) {
  const char* q = static_cast<const char*>(p);
  const long bytes = stride * (long)size;
  return {q, bytes, q ? q + (rows - 1) * bytes + C * (long)size : nullptr, bytes >= 16 ? std::max(rows - 2, 0L) : 0L};
}
inline bool whole(const Rows& t, size_t a) { return !t.p || (reinterpret_cast<uintptr_t>(t.p) % a == 0 && t.stride % a == 0); }
inline bool at(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline int pow2_from(long n) { int p = 1; while (p < n) p *= 2; return p; }

// Threads a row and octets a thread.  Two octets a thread: what it keeps beside them once for two, half the steps of a sum over the row, and twice the bytes on their way (gradients of
// 131072 x 128 bf16 26 us, with one 30; of 8192 x 4096 47 us, with one 59).  One, where two of floats with all their companions do not fit the registers (`one`: gradients of 131072 x 64
// floats 26 us, with two 30; norm of as many into 8 bits 19, with two 22) or octets have to be in neighbouring lanes (rows at any alignment), or more threads would go without.  Rows of up to 64 octets take part of a warp each and meet no barrier; longer ones have a block of their own.
// Four, where `four` says so, of rows that 512 threads with two do not hold (4096 x 12288 bf16: norm 69 us, read again for every step 113; gradients, by a kernel of their own, 97
// and 199).  V = 0: more than they hold.
struct Team { int V, group, threads; long groups; };
inline Team team_of(int octets, bool one, bool four = false) {
  Team t = {};
  const auto up = [](int n) { return (n + 31) / 32 * 32; };
  if (octets <= (one ? 32 : 64)) {
    t.V = one || octets == 1 ? 1 : 2;
    t.group = pow2_from((octets + t.V - 1) / t.V);
    t.threads = 128;
  } else {
    const int n1 = up(octets), n2 = up((octets + 1) / 2);
    const int n4 = up((octets + 3) / 4);
    t.V = n1 <= 512 && (one || n1 < 2 * n2) ? 1 : n2 <= 512 ? 2 : four && n4 <= 512 ? 4 : 0;
    t.group = t.threads = t.V == 1 ? n1 : t.V == 2 ? n2 : t.V == 4 ? n4 : 1024;
  }
  t.groups = t.threads / t.group;
  return t;
}
inline Drop drop_of(const xconv_rows_desc* d) {
  Drop r = {};
  const unsigned long long T = (unsigned long long)(d->p * 4294967296.0);
  if (T == 0) return r;
  r.how = d->seed_add ? DROP_DEVICE : DROP_HOST;
  r.per = divisor((uint32_t)std::min<long>(d->rows_per_mask, 0x7fffffff));          // (rows are fewer)
  const uint32_t t = (uint32_t)(T - 1);
  r.bound = t | 0xffffu; r.last = t & 0xffffu;
  r.k0 = (uint32_t)d->seed; r.k1 = (uint32_t)(d->seed >> 32);
  r.add = d->seed_add;
  r.scale = d->p < 1.0 ? (float)(1.0 / (1.0 - d->p)) : 0.f;
  return r;
}
// Blocks of a kernel that an SM of the current device holds.  (Asked in every launch: nothing is kept between calls.)
template <typename... A>
int resident_blocks(void (*kernel)(A...), int threads, int smem) {
  int n = 0;
  return cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) == cudaSuccess ? std::max(n, 1) : 1;
}
// f(VEC, how the key comes) as types.
template <typename F>
auto with_kinds(bool vec, int how, F&& f) {
  const auto g = [&](auto h) { return vec ? f(std::true_type(), h) : f(std::false_type(), h); };
  return how == DROP_NONE ? g(std::integral_constant<int, DROP_NONE>()) : how == DROP_HOST ? g(std::integral_constant<int, DROP_HOST>()) : g(std::integral_constant<int, DROP_DEVICE>());
}
// f(T()) with the type of the activations.
template <typename F>
cudaError_t with_type(int dtype, F&& f) {
  if (dtype == XCONV_F32) return f(float());
  return dtype == XCONV_BF16 ? f(bf16()) : f(f16());
}

}  // namespace xconv
