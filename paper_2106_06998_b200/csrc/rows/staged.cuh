// Dense rows that do not begin on 16-byte boundaries, by runs of rows through shared memory: what the forward and the backward kernel share.
//
// A run's bytes are copied as whole pieces of 16 bytes (asynchronously, stages - 1 runs ahead) to a place in shared memory that has the same position about a boundary, worked on there two
// values at a time, neighbouring lanes on neighbouring pairs, and results go back over the inputs and out in pieces again.  Instructions count for such rows: a thread's rows are all
// even or all odd in number, so that what of its pairs is the row's is known before the first one.
#pragma once

#include "rows.cuh"

namespace xconv {

constexpr int STAGED_SMEM = 200 * 1024;

struct Staged {
  int C, group, groups, run, octets;             // threads of a row, rows of a pass and of a run
  int slot, slots;                               // bytes of a tensor's run, tensors of a stage
  int stages;
  long rows, runs, values;                       // of a tensor
  Drop drop;
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Where a run lies: values between the boundary before it and it, and from that boundary to its end; rows of it.
struct Run {
  long begin;                      // the boundary, in values
  int shift, end, rows;
  template <int PER>
  __device__ __forceinline__ static Run of(const Staged& s, long run) {
    Run r;
    const long first = run * s.run * s.C;
    r.shift = (int)(first & (PER - 1));
    r.begin = first - r.shift;
    r.rows = (int)min((long)s.run, s.rows - run * s.run);
    r.end = r.shift + r.rows * s.C;
    return r;
  }
};

// A run into shared memory.  (The tensor begins on a boundary; of a piece that reaches beyond its end the values go one by one.)
template <typename T>
__device__ __forceinline__ void run_in(const Staged& s, const Run& r, char* at, const T* tensor) {
  constexpr int PER = 16 / sizeof(T);
  const int pieces = (int)(min((long)(r.end + PER - 1), s.values - r.begin) / PER);
  const T* from = tensor + r.begin + threadIdx.x * PER;
  uint32_t to = (uint32_t)__cvta_generic_to_shared(at) + 16 * threadIdx.x;
  for (int i = threadIdx.x; i < pieces; i += blockDim.x, from += blockDim.x * PER, to += 16 * blockDim.x) copy16(to, from);
  const int rest = pieces * PER + (int)threadIdx.x;
  if (rest < r.end) reinterpret_cast<T*>(at)[rest] = tensor[r.begin + rest];           // (fewer than a piece's)
}
// ... and out again: whole pieces, and the values at both ends.
template <typename T>
__device__ __forceinline__ void run_out(const Run& r, const char* at, T* tensor) {
  constexpr int PER = 16 / sizeof(T);
  T* to = tensor + r.begin;
  const T* from = reinterpret_cast<const T*>(at);
  const int first = (r.shift + PER - 1) / PER, pieces = r.end / PER;
  for (int i = first + threadIdx.x; i < pieces; i += blockDim.x) reinterpret_cast<uint4*>(to)[i] = reinterpret_cast<const uint4*>(from)[i];
  const int head = r.shift + (int)threadIdx.x, tail = max(pieces, first) * PER + (int)threadIdx.x;
  if (head < min(first * PER, r.end)) to[head] = from[head];
  if (tail < r.end) to[tail] = from[tail];
}
// A thread's pairs of a row: V of them, `group` pairs from one to the next.  A row with an odd number of values before it has its first one in the second place of its first pair.
template <typename T, int V>
struct Pairs {
  int lane, group, C, odd;
  int column;                      // of the first pair
  bool begins, one, two;           // the first pair's first value is the row's; of the last pair, the first one and both are
  __device__ __forceinline__ Pairs(int lane, int group, int C, int odd) : lane(lane), group(group), C(C), odd(odd), column(2 * lane - odd) {
    begins = column >= 0;
    const int left = C - (column + 2 * (V - 1) * group);
    one = left >= 1; two = left >= 2;
  }
  // (V is the least number of pairs that reaches all of the row)
  __device__ __forceinline__ bool has(int v, int k) const { return (v > 0 || k > 0 || begins) && (v < V - 1 || (k ? two : one)); }
  __device__ __forceinline__ void read(const T* row, float (&f)[V][2]) const {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const T* at = row + column + 2 * v * group;
      float2 t;
      if constexpr (sizeof(T) == 4) t = *reinterpret_cast<const float2*>(at);
      else if constexpr (std::is_same<T, bf16>::value) { const uint32_t u = *reinterpret_cast<const uint32_t*>(at); t = make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)); }
      else t = __half22float2(*reinterpret_cast<const __half2*>(at));
      f[v][0] = has(v, 0) ? t.x : 0.f;
      f[v][1] = has(v, 1) ? t.y : 0.f;
    }
  }
  __device__ __forceinline__ void write(T* row, const float (&f)[V][2]) const {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      T* at = row + column + 2 * v * group;
      if constexpr (sizeof(T) == 4) {
        if (has(v, 0) && has(v, 1)) *reinterpret_cast<float2*>(at) = make_float2(f[v][0], f[v][1]);
        else if (has(v, 0)) at[0] = f[v][0];
        else if (has(v, 1)) at[1] = f[v][1];
      } else {
        uint32_t t;
        if constexpr (std::is_same<T, bf16>::value) { const __nv_bfloat162 p = __floats2bfloat162_rn(f[v][0], f[v][1]); t = *reinterpret_cast<const uint32_t*>(&p); }
        else { const __half2 p = __floats2half2_rn(f[v][0], f[v][1]); t = *reinterpret_cast<const uint32_t*>(&p); }
        if (has(v, 0) && has(v, 1)) *reinterpret_cast<uint32_t*>(at) = t;
        else if (has(v, 0)) *reinterpret_cast<unsigned short*>(at) = (unsigned short)t;
        else if (has(v, 1)) *reinterpret_cast<unsigned short*>(at + 1) = (unsigned short)(t >> 16);
      }
    }
  }
  template <typename P>
  __device__ __forceinline__ void weights(const void* weight, float (&w)[V][2]) const {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int k = 0; k < 2; ++k) w[v][k] = has(v, k) ? (weight ? to_f(static_cast<const P*>(weight)[column + 2 * v * group + k]) : 1.f) : 0.f;
  }
};

// Whether a thread's values are dropped.  The lanes of a row draw an octet each for every four pairs of a thread -- the octets of the pairs that lie side by side in their lanes -- and
// each asks the lane that has its pair's.  In an odd row a pair's second value is the first of its two in the octets' count: bytes are moved on by one, and take in the last bit of the
// octet before.
template <int V>
struct PairMask {
  static constexpr int ROUNDS = (V + 3) / 4;
  uint32_t bits[ROUNDS];
  uint32_t row;                    // the mask row that they are of
  __device__ __forceinline__ PairMask() : row(0xffffffffu) {}
  __device__ __forceinline__ void draw(const Staged& s, uint2 key, int lane, int odd, uint32_t mask_row) {
    if (!__any_sync(0xffffffffu, mask_row != row)) return;    // (whole channels: the row before had the same)
    row = mask_row;
    const unsigned long long first = (unsigned long long)mask_row * (uint32_t)s.octets;
    const int l = threadIdx.x & 31, group = s.group;
    if (group <= 32) {
      uint32_t last = 0;
#pragma unroll
      for (int j = 0; j < ROUNDS; ++j) {
        const uint32_t b = mask_bits(s.drop, key, first + (j * group + lane));
        uint32_t before = __shfl_up_sync(0xffffffffu, b, 1, group);
        if (lane == 0) before = last;
        last = __shfl_sync(0xffffffffu, b, group - 1, group);
        bits[j] = odd ? b << 1 | before >> 7 : b;
      }
    } else {
      const int apart = group >> 2, base = (int)(threadIdx.x >> 5) * 8;       // octets from a pair to the thread's next; of the warp's first one
      uint32_t ahead = 0;          // the octet before those of the lane-th pairs
      if (odd) ahead = mask_bits(s.drop, key, first + max(base + (l & 7) * apart - 1, 0));
#pragma unroll
      for (int j = 0; j < ROUNDS; ++j) {
        const int v = 4 * j + (l >> 3);
        const uint32_t b = mask_bits(s.drop, key, first + (base + v * apart + (l & 7)));
        uint32_t before = __shfl_up_sync(0xffffffffu, b, 1);
        const uint32_t other = __shfl_sync(0xffffffffu, ahead, v);
        if ((l & 7) == 0) before = other;
        bits[j] = odd ? b << 1 | before >> 7 : b;
      }
    }
  }
  __device__ __forceinline__ void gone(const Staged& s, int lane, bool (&g)[V][2]) const {
    const int width = min(s.group, 32), l = lane & (width - 1), apart = width >> 2, by = 2 * (l & 3);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const uint32_t b = __shfl_sync(0xffffffffu, bits[v >> 2], (l >> 2) + (v & 3) * apart, width) >> by;
      g[v][0] = b & 1; g[v][1] = b & 2;
    }
  }
};

// ---- host side

// slots: tensors that are read or written; eight: and one of bytes.  threads = 0: rows that do not fit.
struct StagedPlan { int V, threads, smem; long blocks; };
inline StagedPlan staged_plan(const xconv_rows_desc* d, int slots, bool backward, bool eight, Staged* s) {
  StagedPlan p = {};
  const int es = d->dtype == XCONV_F32 ? 4 : 2, pairs = d->C / 2 + (d->C & 1);       // (of even and odd rows the same)
  // threads of a row: as little work as possible, of which a thread has about three pairs' beside its pairs (31189 x 513 bf16, 64 threads of 5 pairs: norm 50 us, 288 of one: 65)
  int best = 0;
  for (int g = 4; g <= 512; g = g < 32 ? 2 * g : g + 32) {
    const int V = (pairs + g - 1) / g;
    if (V > 8 || (best && (V + 3) * g >= best)) continue;
    best = (V + 3) * g; s->group = g; p.V = V;
  }
  if (!best) return p;
  p.threads = s->group <= 32 ? 256 : s->group;
  s->groups = p.threads / s->group;
  s->C = d->C; s->octets = (d->C + 7) / 8;
  s->rows = d->rows; s->values = d->rows * d->C; s->slots = slots;
  // rows of a run: passes of the block's groups (an even number of rows, or one), about 6 KB a tensor, but runs for all SMs
  const long row_bytes = (long)d->C * es;
  int passes = s->groups == 1 ? 1 : (int)std::max(1L, std::min(8L, 6 * 1024 / (row_bytes * s->groups)));
  while (passes > 1 && d->rows < (long)passes * s->groups * ROWS_SMS * 4) --passes;
  s->run = passes * s->groups;
  s->runs = (d->rows + s->run - 1) / s->run;
  // (a boundary's shift in front; behind, what lanes without values of the row read)
  s->slot = (int)((s->run * row_bytes + 16 + 2 * s->group * es + 15) / 16 * 16);
  // Two runs ahead, or one, where more blocks then fit an SM.  (An even number of blocks: a block of one row a run meets even rows or odd ones only.)
  int resident = 0;
  for (int stages = 3; stages >= 2; --stages) {
    int smem = stages * slots * s->slot + (eight ? (s->run * d->C + 15 + 15) / 16 * 16 : 0);
    if (backward) smem = std::max(smem, s->groups * d->C * 4);
    if (smem > STAGED_SMEM) continue;
    const int n = std::max(1, std::min((p.V <= 4 ? 1024 : 512) / p.threads, 220 * 1024 / (smem + 1024)));
    if (n <= resident) continue;
    resident = n; s->stages = stages; p.smem = smem;
  }
  if (!resident) { p.threads = 0; return p; }
  p.blocks = std::min(s->runs, (long)ROWS_SMS * resident);
  return p;
}

}  // namespace xconv
