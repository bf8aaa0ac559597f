// Orthogonalisation by Newton-Schulz products: X0 = U / max(|U|_F, eps), n x m with n <= m (transposed where it is taller than wide), then `steps` times
//
//   A = X X^T,   B = a I + b A + c A A,   X <- B X
//
// which maps every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors.  Any number of matrices of any shapes goes through the same launches: the
// unit of work is a 256 x 256 tile of some matrix's product.
//
// Arithmetic.  A step multiplies small singular values by a (3.4): an error of the operands' roundings grows by 485 in five steps where X has large singular
// values beside small ones.  With operands rounded to bfloat16 the result is off by 1e-2 (normal values) to 0.3 (eight directions above noise), with one float16 part
// by 1e-3 to 4e-2; with float arithmetic by 1e-7 to 5e-6.  So every operand is two float16 parts here, x 2^13 = h + l (11 + 11 bits and the sign between
// them; |X| < 2, |A| < 4, |B| < 8: nothing overflows, and what is lost is below 2^-38), and a product is l h + h l + h h on the tensor cores, as exact as one of floats.
// The tensor cores' accumulator is not rounded to nearest; a chain of MMAs is 32 terms long (four MMAs of the small products, then two of h h), and the chains are
// added in float registers.  Error against 64 bits, times that of the same steps in float arithmetic (root mean square over up to 2000 random matrices): smaller sides of 129 and
// more 0.1 to 0.9, of 33 to 128 0.1 to 1.95 (33 x 161), of up to 32 0.3 to 2.6 (4 x 4660).  Where every result is rounded to 16 bits anyway a chain is 128 terms, since the wait for a free set of sums
// costs 150 clocks a chain (4096 x 4096 bfloat16: 3440 -> 3040 us; 64 terms 3150, 256 terms 2930, whose largest errors pass four times those of float arithmetic).  That
// error is 0.5 to 2.1 times that of float arithmetic (40 x 5000: 2.9), and the rounding of the result 11 (float16, 4096 x 4096, eight directions above noise) to 800 times it.
//
// Layout.  X, A and B lie in the scratch memory as blocks of 128 x 64 values, each part 16 KB in the order that the MMA wants in shared memory without a swizzle
// (eight rows' 16-byte pieces side by side): whatever the matrices' sizes one tensor map describes them all, eight lanes with a row each write whole lines, and the
// same block serves as a tile whose rows run along the result (X X^T, A A, B of B X) and as one whose rows run along the sum (X of B X).  Behind a matrix's last row and column lie zeros.
// A and B are symmetric: only tiles of 256 x 256 on and below the diagonal are computed and kept, and what lies above is read as the transposed of a tile below:
// the same memory with its rows along the sum.
//
// A pair of CTAs works on a tile of 256 x 256: each brings 128 rows of either operand, 64 terms (64 KB) a stage, and the two tensor cores read both halves of the second
// one.  The copies' latency bounds smaller tiles: 192 KB of ring, 2800 clocks from a copy to its arrival, 768 clocks of MMAs for the 64 KB of a
// tile of 128 x 128 by one CTA (measured there: 1250 clocks a stage), 1536 here.  In a CTA a warp copies, one (of the first CTA) issues the MMAs, sixteen add
// chains and write results.  Where there are fewer tiles than pairs, clusters of two or four pairs share the terms of the tiles with the longest
// sums; each pair then has a part of the tile's columns, and reads the others' sums of them over the SMs' network.
//
// What bounds it (B200, 4096 x 4096 bfloat16, five steps, 3.0 to 3.4 ms on different boards): the tensor cores at the clock that the power limit leaves; 4.1 TFLOP of float16
// products at 1.2 to 1.35 PFLOP/s, cuBLAS's sustained rate on this board being 1.37.  Smaller calls: 15 kernels of 7 us and more, one behind the other, of which a tile's own
// products are a third (8 x 1000 x 523 float16 350 us, a residual network's 19 convolutions 570 us).
#include "newton_schulz.h"

#include <algorithm>

#include "../split_f32.cuh"

namespace xconv {

namespace {

constexpr int NS_SMS = 148;
constexpr int NS_STAGES = 3, NS_SETS = 2, NS_CHAIN = 2, NS_LONG = 2;      // NS_CHAIN: steps of 16 terms, NS_LONG: stages
constexpr uint32_t NS_OPERAND = 32 * 1024, NS_STAGE = 2 * NS_OPERAND, NS_PART = NS_OPERAND / 2;
constexpr int NS_ADDERS = 16, NS_THREADS = 32 * (2 + NS_ADDERS);
constexpr int NS_TILE = 256;
constexpr int NS_PITCH = 129;                            // rows of a column group of the sums that pairs exchange, and one
constexpr float NS_SCALE = 8192.f, NS_UNSCALE = 1.f / 8192.f;
constexpr size_t NS_HEADER = 256;

enum { NS_GRAM, NS_SQUARE, NS_APPLY, NS_LAST };

struct NsArgs {
  CUtensorMap whole, across;   // the blocks as rows of 2 KB, 16 (both parts of a block) a copy; as rows of 1 KB, 8 of two neighbouring blocks a copy
  NsTable t;
  char* blocks;                // the blocks of the scratch memory
  double* sums;                // partial sums of squares, NS_CHUNK values each
  unsigned *status, tag;
  float a, b, c, momentum, keep;
  double eps;
  int muon, nesterov, which;   // which: the buffer that X is in (ns_small_kernel: the number of steps)
  int cs, heavy;               // pairs of CTAs of a cluster, tiles that they share (the first ones; ns_small_kernel: CTAs a matrix)
};

__host__ __device__ __forceinline__ int chunks_of(const NsEntry& e) { return (int)(((long)e.n * e.m + NS_CHUNK - 1) / NS_CHUNK); }
__host__ __device__ __forceinline__ int row_blocks(const NsEntry& e) { return (e.n + NS_ROWS - 1) / NS_ROWS; }
__host__ __device__ __forceinline__ int x_cols(const NsEntry& e) { return (e.m + NS_COLS - 1) / NS_COLS; }
__host__ __device__ __forceinline__ int a_cols(const NsEntry& e) { return 2 * row_blocks(e); }
__host__ __device__ __forceinline__ int a_terms(const NsEntry& e) { return (e.n + NS_COLS - 1) / NS_COLS; }      // blocks of A's columns that hold anything
__host__ __device__ __forceinline__ int tiles(int blocks, int per) { return (blocks + per - 1) / per; }

// The parts of eight values that are scaled already, packed.
__device__ __forceinline__ void parts8(const float (&v)[8], uint4& hi, uint4& lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 p = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
    const float2 f = __half22float2(p);
    const __half2 q = __floats2half2_rn(v[2 * i] - f.x, v[2 * i + 1] - f.y);
    h[i] = *reinterpret_cast<const uint32_t*>(&p);
    l[i] = *reinterpret_cast<const uint32_t*>(&q);
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}
// Byte of a block's first part at which the 16-byte piece `piece` of `row` lies.
__device__ __forceinline__ uint32_t piece_at(int row, int piece) { return (uint32_t)((row >> 3) * 1024 + piece * 128 + (row & 7) * 16); }

// ---- momenta and sums of squares: a block of threads per NS_CHUNK values

__device__ __forceinline__ float update_of(float g, float m, float mu, int nesterov) { return nesterov ? fmaf(mu, m - g, g) : m; }

template <typename G>
__device__ __forceinline__ double squares_of(const NsArgs& p, const NsEntry& e, size_t first, size_t last) {
  const G* g = static_cast<const G*>(e.g);
  double s = 0.0;
  // (The tensors lie on 16-byte boundaries, but not every entry of a table: where a batch is cut it begins at any of the batch's matrices, of any number of values.  The
  // accesses of four or eight values elsewhere are those of rows of a multiple of four or eight, whose matrices are too.)
  const auto fours = [](const void* at, size_t each) { return reinterpret_cast<uintptr_t>(at) % (4 * each) == 0; };
  if ((last - first) % 4 == 0 && fours(g + first, sizeof(G)) && (!p.muon || fours(e.mom + first, sizeof(float)))) {
    constexpr int DEEP = 4;                                  // loads that are under way together
#pragma unroll
    for (int k0 = 0; k0 < NS_CHUNK / 1024; k0 += DEEP) {
      float4 u[DEEP], m[DEEP];
#pragma unroll
      for (int k = 0; k < DEEP; ++k) {
        const size_t i = first + (size_t)((k0 + k) * 256 + threadIdx.x) * 4;
        u[k] = i < last ? ld4(g + i) : make_float4(0.f, 0.f, 0.f, 0.f);
        if (p.muon) m[k] = i < last ? ld4(e.mom + i) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int k = 0; k < DEEP; ++k) {
        if (p.muon) {
          const float f = 1.f - p.momentum;
          m[k] = make_float4(fmaf(f, u[k].x - m[k].x, m[k].x), fmaf(f, u[k].y - m[k].y, m[k].y), fmaf(f, u[k].z - m[k].z, m[k].z), fmaf(f, u[k].w - m[k].w, m[k].w));
          const size_t i = first + (size_t)((k0 + k) * 256 + threadIdx.x) * 4;
          if (i < last) st4(e.mom + i, m[k]);
          u[k] = make_float4(update_of(u[k].x, m[k].x, p.momentum, p.nesterov), update_of(u[k].y, m[k].y, p.momentum, p.nesterov),
                             update_of(u[k].z, m[k].z, p.momentum, p.nesterov), update_of(u[k].w, m[k].w, p.momentum, p.nesterov));
        }
        s += ((double)u[k].x * u[k].x + (double)u[k].y * u[k].y) + ((double)u[k].z * u[k].z + (double)u[k].w * u[k].w);
      }
    }
  } else {
#pragma unroll 8
    for (int k = 0; k < NS_CHUNK / 256; ++k) {
      const size_t i = first + (size_t)(k * 256 + threadIdx.x);
      if (i >= last) break;
      float u = to_f(g[i]);
      if (p.muon) {
        const float m = fmaf(1.f - p.momentum, u - e.mom[i], e.mom[i]);
        e.mom[i] = m;
        u = update_of(u, m, p.momentum, p.nesterov);
      }
      s += (double)u * u;
    }
  }
  return s;
}

__global__ void __launch_bounds__(256) ns_squares_kernel(const __grid_constant__ NsArgs p) {
  __shared__ double sums[8];
  int k = 0;
  while (k + 1 < p.t.entries && (int)blockIdx.x >= p.t.e[k + 1].chunk0) ++k;
  const NsEntry& e = p.t.e[k];
  const int local = (int)blockIdx.x - e.chunk0, per = chunks_of(e), mat = local / per;
  const size_t size = (size_t)e.n * e.m, base = (size_t)mat * size, first = base + (size_t)(local - mat * per) * NS_CHUNK;
  const size_t last = first + NS_CHUNK < base + size ? first + NS_CHUNK : base + size;
  pdl_wait();
  double s = e.g_dtype == XCONV_F32 ? squares_of<float>(p, e, first, last) : e.g_dtype == XCONV_BF16 ? squares_of<bf16>(p, e, first, last) : squares_of<f16>(p, e, first, last);
  pdl_trigger();
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) s += sums[w];
    p.sums[blockIdx.x] = s;
  }
}

// Values times 2^13 / norm: a float in [0.5, 1) and a power of two that is applied in halves, so that neither the factor nor a product leaves the floats' range.
struct NsScale {
  float f, s1, s2;
  __device__ __forceinline__ NsScale(double squares, double eps) {
    const double norm = sqrt(squares);
    int ex = 0;
    f = (float)frexp((double)NS_SCALE / (norm < eps ? eps : norm), &ex);
    const int e1 = min(126, max(-126, ex / 2)), e2 = min(126, max(-126, ex - e1));
    s1 = __int_as_float((e1 + 127) << 23);
    s2 = __int_as_float((e2 + 127) << 23);
  }
  __device__ __forceinline__ float operator()(float x) const { return x * s1 * f * s2; }
};

// ---- X0 in blocks: a block of threads per block of 128 x 64 values

// Eight neighbouring values of a row of U (X's columns c0 on), `left` of them there; G: the gradients' type.
template <typename G>
__device__ __forceinline__ void ns_load8(const NsArgs& p, const NsEntry& e, size_t base, long row, long c0, int left, float (&u)[8]) {
  const G* g = static_cast<const G*>(e.g) + base;
  const float* mom = p.muon ? e.mom + base : nullptr;
  const bool tall = e.rows > e.cols;
  const size_t at = tall ? (size_t)c0 * e.n + row : (size_t)row * e.m + c0, apart = tall ? e.n : 1;
  if (!tall && e.m % 8 == 0) {
    const float4 z = make_float4(0.f, 0.f, 0.f, 0.f), a = left > 0 ? ld4(g + at) : z, b = left > 0 ? ld4(g + at + 4) : z;
    u[0] = a.x; u[1] = a.y; u[2] = a.z; u[3] = a.w; u[4] = b.x; u[5] = b.y; u[6] = b.z; u[7] = b.w;
    if (mom && left > 0) {
      const float4 c = __ldcg(reinterpret_cast<const float4*>(mom + at)), d = __ldcg(reinterpret_cast<const float4*>(mom + at + 4));
      const float m[8] = {c.x, c.y, c.z, c.w, d.x, d.y, d.z, d.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = update_of(u[j], m[j], p.momentum, p.nesterov);
    }
  } else {
    float m[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      u[j] = j < left ? to_f(g[at + j * apart]) : 0.f;
      if (mom) m[j] = j < left ? __ldcg(mom + at + j * apart) : 0.f;
    }
    if (mom)
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = update_of(u[j], m[j], p.momentum, p.nesterov);
  }
}

__global__ void __launch_bounds__(256) ns_blocks_kernel(const __grid_constant__ NsArgs p) {
  __shared__ double sums[8];
  int k = 0;
  while (k + 1 < p.t.entries && (int)blockIdx.x >= p.t.e[k + 1].block0) ++k;
  const NsEntry& e = p.t.e[k];
  const int kt = x_cols(e), per = row_blocks(e) * kt, local = (int)blockIdx.x - e.block0, mat = local / per, at = local - mat * per;
  const int rb = at / kt, cb = at - rb * kt, tid = threadIdx.x;
  pdl_wait();
  pdl_trigger();
  // the norm, from the matrix's partial sums in fixed order
  const int chunks = chunks_of(e);
  double s = 0.0;
  for (int i = tid; i < chunks; i += 256) s += __ldcg(p.sums + e.chunk0 + (long)mat * chunks + i);
  // U of these rows and columns, pieces of eight values: neighbouring threads have neighbouring rows, whose pieces lie side by side
  const size_t base = (size_t)mat * e.n * e.m;
  const long row = (long)rb * NS_ROWS + (tid & (NS_ROWS - 1));
  float u[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long c0 = (long)cb * NS_COLS + (i * 2 + tid / NS_ROWS) * 8;
    const int left = row < e.n ? (int)max(0L, min(8L, e.m - c0)) : 0;
    if (e.g_dtype == XCONV_F32) ns_load8<float>(p, e, base, row, c0, left, u[i]);
    else if (e.g_dtype == XCONV_BF16) ns_load8<bf16>(p, e, base, row, c0, left, u[i]);
    else ns_load8<f16>(p, e, base, row, c0, left, u[i]);
  }
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((tid & 31) == 0) sums[tid >> 5] = s;
  __syncthreads();
  s = sums[0];
  for (int w = 1; w < 8; ++w) s += sums[w];
  const NsScale f(s, p.eps);
  char* out = p.blocks + ((size_t)e.x0 + (size_t)mat * per + at) * NS_BLOCK;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) u[i][j] = f(u[i][j]);
    uint4 hi, lo;
    parts8(u[i], hi, lo);
    const uint32_t to = piece_at(tid & (NS_ROWS - 1), i * 2 + tid / NS_ROWS);
    *reinterpret_cast<uint4*>(out + to) = hi;
    *reinterpret_cast<uint4*>(out + NS_PART + to) = lo;
  }
}

// ---- products

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
// ... that orders no memory: for what only has to outlive the other CTAs' accesses, which they have seen the end of.
__device__ __forceinline__ void cluster_sync_relaxed() {
  asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
  asm volatile("barrier.cluster.wait;" ::: "memory");
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr, uint32_t rank) {      // (several are under way together)
  float4 v;
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr), "r"(rank));
  return v;
}
__device__ __forceinline__ void st_cluster_u32(uint32_t addr, uint32_t rank, uint32_t v) {
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.u32 [a], %2;\n\t}" ::"r"(addr), "r"(rank), "r"(v) : "memory");
}
__device__ __forceinline__ void arrive_at(uint64_t* bar, uint32_t rank) {      // ... of the same barrier in another CTA of the cluster
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tmbarrier.arrive.shared::cluster.b64 _, [a];\n\t}"
               ::"r"(smem_u32(bar)), "r"(rank) : "memory");
}
// Tensor memory of a pair: a warp of either CTA allocates, behind it the go-ahead for the next kernel is given.
__device__ __forceinline__ void pair_alloc_then_trigger(uint32_t* slot) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(slot)) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  pdl_trigger();
}
__device__ __forceinline__ void pair_dealloc(uint32_t tmem) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}
// Rows of the blocks into this CTA's shared memory; the bytes count at the barrier of the pair's first CTA.
__device__ __forceinline__ void pair_load(uint32_t dst, const CUtensorMap* map, uint32_t row, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(smem_u32(bar) & 0xFEFFFFFFu) : "memory");
}
__device__ __forceinline__ void pair_load_across(uint32_t dst, const CUtensorMap* map, uint32_t block, uint32_t row, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(block), "r"(row), "r"(smem_u32(bar) & 0xFEFFFFFFu) : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "mov.b64 da, {%1, %2};\n\t"
      "mov.b64 db, {%3, %4};\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %5, p;\n\t}"
      ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
}
// An arrival at the barrier in the CTAs of `mask` once every MMA issued so far has finished.
__device__ __forceinline__ void pair_commit(uint64_t* bar, uint32_t mask) {
  asm volatile("{\n\t.reg .pred e;\n\t.reg .b16 m;\n\tcvt.u16.u32 m, %1;\n\telect.sync _|e, 0xffffffff;\n\t"
               "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n\t}" ::"r"(smem_u32(bar)), "r"(mask) : "memory");
}

// A unit of work: tile (I, J) of matrix `mat` of an entry, and the stages (64 terms each) that its sums have.
struct NsUnit { int k, mat, I, J, stages; };
template <int MODE>
__device__ __forceinline__ NsUnit ns_unit(const NsEntry* es, int entries, int u, int& k) {
  constexpr bool SYM = MODE == NS_GRAM || MODE == NS_SQUARE;
  while (k + 1 < entries && u >= (SYM ? es[k + 1].sym0 : es[k + 1].prod0)) ++k;
  const NsEntry& e = es[k];
  NsUnit w;
  w.k = k;
  const int rows = tiles(row_blocks(e), 2);
  if (SYM) {
    const int per = rows * (rows + 1) / 2, local = u - e.sym0;
    w.mat = local / per;
    const int t = local - w.mat * per;
    int i = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while (i * (i + 1) / 2 > t) --i;
    while ((i + 1) * (i + 2) / 2 <= t) ++i;
    w.I = i;
    w.J = t - i * (i + 1) / 2;
    w.stages = MODE == NS_GRAM ? x_cols(e) : a_terms(e);
  } else {
    const int per = rows * tiles(x_cols(e), 4), local = u - e.prod0;
    w.mat = local / per;
    const int t = local - w.mat * per;
    w.J = t / rows;                                  // (neighbouring units read the same columns of X)
    w.I = t - w.J * rows;
    w.stages = a_terms(e);
  }
  return w;
}

// Elements of the result, from their sums: the orthogonalised matrix's, or the weights that they move.
__device__ __forceinline__ float ns_result(const NsArgs& p, const NsEntry& e, float sum, float weight) {
  const float o = sum * (NS_UNSCALE * NS_UNSCALE);
  return p.muon ? fmaf(-e.scale, o, p.keep * weight) : o;
}
// COUNT groups of four neighbouring ones, `apart` elements from each other, of which `left` values are there in each and `groups` groups; the weights are loaded
// together.
template <typename T, int COUNT>
__device__ __forceinline__ void ns_finish4_of(const NsArgs& p, const NsEntry& e, size_t at, size_t apart, long left, int groups, const float (*v)[4]) {
  T* out = static_cast<T*>(e.out) + at;
  float4 w[COUNT];
  if (e.m % 4 == 0) {
    if (left <= 0) return;
    if (p.muon)
#pragma unroll
      for (int k = 0; k < COUNT; ++k) w[k] = k < groups ? ld4(out + k * apart) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < COUNT; ++k)
      if (k < groups)
        st4(out + k * apart, make_float4(ns_result(p, e, v[k][0], w[k].x), ns_result(p, e, v[k][1], w[k].y), ns_result(p, e, v[k][2], w[k].z), ns_result(p, e, v[k][3], w[k].w)));
    return;
  }
#pragma unroll
  for (int k = 0; k < COUNT; ++k) {
    if (k >= groups) continue;
    float a[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = p.muon && j < left ? to_f(out[k * apart + j]) : 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) out[k * apart + j] = from_f<T>(ns_result(p, e, v[k][j], a[j]));
  }
}
template <int COUNT>
__device__ __forceinline__ void ns_finish4(const NsArgs& p, const NsEntry& e, size_t at, size_t apart, long left, int groups, const float (*v)[4]) {
  if (e.out_dtype == XCONV_F32) ns_finish4_of<float, COUNT>(p, e, at, apart, left, groups, v);
  else if (e.out_dtype == XCONV_BF16) ns_finish4_of<bf16, COUNT>(p, e, at, apart, left, groups, v);
  else ns_finish4_of<f16, COUNT>(p, e, at, apart, left, groups, v);
}
// Eight elements of a column of a tall matrix's result, a row's length apart.
template <typename T>
__device__ __forceinline__ void ns_finish_across_of(const NsArgs& p, const NsEntry& e, size_t at, long left, const float (&v)[8]) {
  T* out = static_cast<T*>(e.out) + at;
  float w[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = p.muon && k < left ? to_f(out[(size_t)k * e.n]) : 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < left) out[(size_t)k * e.n] = from_f<T>(ns_result(p, e, v[k], w[k]));
}

// N groups of eight neighbouring sums of a row of this CTA's half of a tile, from column 8 * q8 on (within a block's 64 columns).
template <int MODE, int N>
__device__ __forceinline__ void ns_emit(const NsArgs& p, const NsEntry& e, const NsUnit& w, int half, int row, int q8, float (&v)[N][8]) {
  const int nt = row_blocks(e), i = 2 * w.I + half, cb = 4 * w.J + (q8 >> 3);
  if (i >= nt) return;
  if (MODE != NS_LAST) {
    const int columns = MODE == NS_APPLY ? x_cols(e) : 2 * nt;
    if (cb >= columns) return;
    const size_t at = (((size_t)w.mat * nt + i) * columns + cb) * NS_BLOCK + piece_at(row, q8 & 7);
    char* to = p.blocks + (size_t)(MODE == NS_GRAM ? e.a : MODE == NS_SQUARE ? e.b : p.which ? e.x0 : e.x1) * NS_BLOCK + at;
    const char* from = p.blocks + (size_t)e.a * NS_BLOCK + at;
    uint4 ah[N], al[N];
    if (MODE == NS_SQUARE)
#pragma unroll
      for (int g = 0; g < N; ++g) {
        ah[g] = __ldcg(reinterpret_cast<const uint4*>(from + g * 128));
        al[g] = __ldcg(reinterpret_cast<const uint4*>(from + g * 128 + NS_PART));
      }
#pragma unroll
    for (int g = 0; g < N; ++g) {
      if (MODE == NS_SQUARE) {
        const uint32_t h[4] = {ah[g].x, ah[g].y, ah[g].z, ah[g].w}, l[4] = {al[g].x, al[g].y, al[g].z, al[g].w};
        const int r = i * NS_ROWS + row, d = r < e.n ? r - (w.J * NS_TILE + (q8 + g) * 8) : -1;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h[k])), y = __half22float2(*reinterpret_cast<const __half2*>(&l[k]));
          v[g][2 * k] = fmaf(p.c * NS_UNSCALE, v[g][2 * k], p.b * (x.x + y.x)) + (d == 2 * k ? p.a * NS_SCALE : 0.f);
          v[g][2 * k + 1] = fmaf(p.c * NS_UNSCALE, v[g][2 * k + 1], p.b * (x.y + y.y)) + (d == 2 * k + 1 ? p.a * NS_SCALE : 0.f);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[g][k] *= NS_UNSCALE;
      }
      uint4 hi, lo;
      parts8(v[g], hi, lo);
      *reinterpret_cast<uint4*>(to + g * 128) = hi;
      *reinterpret_cast<uint4*>(to + g * 128 + NS_PART) = lo;
    }
  } else {
    const long r = (long)i * NS_ROWS + row;
    if (r >= e.n) return;
    const size_t base = (size_t)w.mat * e.n * e.m;
#pragma unroll
    for (int g = 0; g < N; ++g) {
      const long c0 = (long)w.J * NS_TILE + (q8 + g) * 8;
      if (e.rows > e.cols) {
        const size_t at = base + (size_t)c0 * e.n + r;
        if (e.out_dtype == XCONV_F32) ns_finish_across_of<float>(p, e, at, e.m - c0, v[g]);
        else if (e.out_dtype == XCONV_BF16) ns_finish_across_of<bf16>(p, e, at, e.m - c0, v[g]);
        else ns_finish_across_of<f16>(p, e, at, e.m - c0, v[g]);
      } else {
        const float f[2][4] = {{v[g][0], v[g][1], v[g][2], v[g][3]}, {v[g][4], v[g][5], v[g][6], v[g][7]}};
        ns_finish4<1>(p, e, base + (size_t)r * e.m + c0, 0, e.m - c0, 1, &f[0]);
        ns_finish4<1>(p, e, base + (size_t)r * e.m + c0 + 4, 0, e.m - c0 - 4, 1, &f[1]);
      }
    }
  }
}

// The last product of a matrix that is not tall, 64 columns of a row each lane: eight lanes exchange pieces of four columns, so that together they have 32 of a row.
__device__ __forceinline__ void ns_emit_rows(const NsArgs& p, const NsEntry& e, const NsUnit& w, int half, int row, int quarter, const float (&sum)[64]) {
  const int lane = threadIdx.x & 7;
  const long r0 = (long)(2 * w.I + half) * NS_ROWS + (row & ~7), c0 = (long)w.J * NS_TILE + quarter * 64 + lane * 4;
  const size_t base = (size_t)w.mat * e.n * e.m;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    float v[8][4];
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[u][k] = sum[b * 32 + u * 4 + k];
#pragma unroll
    for (int d = 1; d < 8; d *= 2)
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        if (u & d) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float got = __shfl_xor_sync(0xffffffffu, lane & d ? v[u][k] : v[u | d][k], d);
          if (lane & d) v[u][k] = got;
          else v[u | d][k] = got;
        }
      }
    const long c = c0 + b * 32;
#pragma unroll
    for (int u = 0; u < 8; u += 2)
      ns_finish4<2>(p, e, base + (size_t)(r0 + u) * e.m + c, e.m, e.m - c, (int)max(0L, min(2L, e.n - r0 - u)), &v[u]);
  }
}

template <int MODE, bool LONG>
__global__ void __launch_bounds__(NS_THREADS, 1) ns_product_kernel(const __grid_constant__ NsArgs p) {
  constexpr bool SYM = MODE == NS_GRAM || MODE == NS_SQUARE;
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t full[NS_STAGES], empty[NS_STAGES], acc_full[NS_SETS], acc_empty[NS_SETS];
  __shared__ NsEntry es[NS_MOST];
  __shared__ NsUnit first;
  __shared__ uint32_t tmem_slot;
  __shared__ uint32_t lost;                          // whether a wait for the sums of a shared tile ran out, in any CTA of the cluster
  const uint32_t smem = (smem_u32(raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, entries = p.t.entries;
  const uint32_t rank = cluster_rank(), half = rank & 1u, leader = rank & ~1u;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NS_STAGES; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < NS_SETS; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], 2 * NS_ADDERS); }
    lost = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_tmap(&p.whole);
    prefetch_tmap(&p.across);
  }
  // A cluster of one pair takes every so-manyth tile; a larger one shares a tile that is heavy, or each of its pairs has a tile of its own.
  const int units = SYM ? p.t.syms : p.t.prods, pair = (int)(rank >> 1), cluster = (int)blockIdx.x / (2 * p.cs);
  const bool shared = p.cs > 1 && cluster < p.heavy;
  const int split = shared ? p.cs : 1, part = shared ? pair : 0;      // of the tile's terms
  const int u0 = p.cs == 1 || shared ? cluster : p.heavy + (cluster - p.heavy) * p.cs + pair, step = p.cs == 1 ? (int)gridDim.x / 2 : units;
  for (int i = threadIdx.x; i < entries * (int)(sizeof(NsEntry) / 4); i += NS_THREADS)
    reinterpret_cast<uint32_t*>(es)[i] = reinterpret_cast<const uint32_t*>(p.t.e)[i];
  if (warp == 1) pair_alloc_then_trigger(&tmem_slot);
  __syncwarp();
  cluster_sync();                                    // (the other CTAs' barriers are there)
  __syncthreads();
  if (threadIdx.x == 0) {                            // (while the kernel before still runs)
    int k = 0;
    first = ns_unit<MODE>(es, entries, min(u0, units - 1), k);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();
  if (blockIdx.x == 0 && threadIdx.x == 64) reinterpret_cast<volatile unsigned*>(p.status)[1] = p.tag;
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&tmem_slot);

  if (warp == 0) {
    if (lane == 0) {
      uint32_t slot = 0, lap = 0, issued = 0;
      int k = first.k;
      bool ok = true;
      for (int u = u0; u < units && ok; u += step) {
        const NsUnit w = u == u0 ? first : ns_unit<MODE>(es, entries, u, k);
        const NsEntry& e = es[w.k];
        const int nt = row_blocks(e), kt = x_cols(e), i = 2 * w.I + (int)half, j = 2 * w.J + (int)half;
        const uint32_t xb = (p.which ? e.x1 : e.x0) + (uint32_t)w.mat * nt * kt, sb = (MODE == NS_SQUARE ? e.a : e.b) + (uint32_t)w.mat * nt * 2 * nt;
        const bool same = SYM && w.I == w.J;
        // What both CTAs of the pair copy a stage: rows of the first operand, rows (columns) of the second.
        uint32_t bytes = (uint32_t)min(2, nt - 2 * w.I) * NS_OPERAND;
        if (SYM) bytes += same ? 0u : (uint32_t)min(2, nt - 2 * w.J) * NS_OPERAND;
        else bytes += kt - 4 * w.J > 2 ? 2 * NS_OPERAND : NS_OPERAND;
        const int s0 = w.stages * part / split, s1 = w.stages * (part + 1) / split;
        for (int s = s0; s < s1; ++s) {
          if (issued >= NS_STAGES && !mbar_wait(&empty[slot], lap ^ 1u, p.status, p.tag)) { ok = false; break; }
          const uint32_t to = smem + slot * NS_STAGE;
          uint64_t* bar = &full[slot];
          if (half == 0) mbar_arrive_expect_tx(bar, bytes);
          // 64 rows of two neighbouring blocks, both parts of each: a tile with its rows along the sum (behind a matrix's last block another's, for columns that
          // nothing reads)
          const auto load_across = [&](uint32_t dst, uint32_t block) {
            pair_load_across(dst, &p.across, block, (uint32_t)(s & 1) * 8u, bar);
            pair_load_across(dst + NS_PART, &p.across, block, (uint32_t)(s & 1) * 8u + 16u, bar);
          };
          // block (i, s) of a symmetric matrix
          const auto load_symmetric = [&](uint32_t dst, int row_block) {
            if (s / 4 <= row_block / 2) pair_load(dst, &p.whole, (sb + (uint32_t)row_block * 2 * nt + s) * 16u, bar);
            else load_across(dst, sb + (uint32_t)(s >> 1) * 2 * nt + 2 * row_block);
          };
          if (MODE == NS_GRAM) {
            if (i < nt) pair_load(to, &p.whole, (xb + (uint32_t)i * kt + s) * 16u, bar);
            if (!same && j < nt) pair_load(to + NS_OPERAND, &p.whole, (xb + (uint32_t)j * kt + s) * 16u, bar);
          } else {
            if (i < nt) load_symmetric(to, i);
            if (MODE == NS_SQUARE) {
              if (!same && j < nt) load_symmetric(to + NS_OPERAND, j);
            } else {
              const int c = 4 * w.J + 2 * (int)half;
              if (c < kt) load_across(to + NS_OPERAND, xb + (uint32_t)(s >> 1) * kt + c);
            }
          }
          ++issued;
          if (++slot == NS_STAGES) { slot = 0; lap ^= 1u; }
        }
      }
      // Behind an error: no copy is under way when the block ends (the first CTA's barriers count both CTAs' copies; the second one ends behind it).
      if (!ok && half == 0)
        for (uint32_t i = 0; i < NS_STAGES && i < issued; ++i) {
          if (slot == 0) { slot = NS_STAGES; lap ^= 1u; }
          --slot;
          mbar_wait(&full[slot], lap, p.status, p.tag);
        }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (half == 0) {
      uint32_t slot = 0, lap = 0, set = 0, set_lap = 0, used = 0;
      int k = first.k;
      bool ok = true;
      // Shared-memory descriptors, no swizzle.  Rows along the result: a row's pieces 128 bytes apart, groups of eight rows 1024, a step of 16 terms 256.
      // Rows along the sum: groups of eight rows 2048 bytes apart (of both blocks), columns' pieces 128, a step 4096.
      constexpr uint32_t ALONG = (128u >> 4) << 16, ALONG_HI = (1024u >> 4) | (1u << 14), ALONG_STEP = 256u >> 4;
      constexpr uint32_t ACROSS = (2048u >> 4) << 16, ACROSS_HI = (128u >> 4) | (1u << 14), ACROSS_STEP = 4096u >> 4;
      constexpr uint32_t IDESC = (1u << 4) | ((uint32_t)(NS_TILE >> 3) << 17) | ((uint32_t)(NS_TILE >> 4) << 24);
      const uint32_t pair_mask = 3u << leader;
      for (int u = u0; u < units && ok; u += step) {
        const NsUnit w = u == u0 ? first : ns_unit<MODE>(es, entries, u, k);
        const bool same = SYM && w.I == w.J;
        const int s0 = w.stages * part / split, s1 = w.stages * (part + 1) / split;
        for (int s = s0; s < s1 && ok; ++s) {
          if (!mbar_wait_warp(&full[slot], lap, p.status, p.tag)) { ok = false; break; }
          tc_fence_after();
          const bool a_across = MODE != NS_GRAM && s / 4 > w.I, b_across = MODE == NS_SQUARE ? s / 4 > w.J : !SYM;
          const uint32_t at = (smem + slot * NS_STAGE) & 0x3FFFFu;      // (in a cluster an address has the CTA's rank above these bits)
          const uint32_t a = (a_across ? ACROSS : ALONG) | (at >> 4), b = (b_across ? ACROSS : ALONG) | ((at + (same ? 0u : NS_OPERAND)) >> 4);
          const uint32_t a_hi = a_across ? ACROSS_HI : ALONG_HI, b_hi = b_across ? ACROSS_HI : ALONG_HI;
          const uint32_t a_step = a_across ? ACROSS_STEP : ALONG_STEP, b_step = b_across ? ACROSS_STEP : ALONG_STEP;
          const uint32_t idesc = IDESC | (a_across ? 1u << 15 : 0u) | (b_across ? 1u << 16 : 0u);
          constexpr uint32_t L = NS_PART >> 4;
          // (chains begin and end within a stage, or with the first and the last of NS_LONG stages)
          constexpr int STEPS = LONG ? 4 : NS_CHAIN;
          const bool begins = !LONG || (s - s0) % NS_LONG == 0, ends = !LONG || (s - s0) % NS_LONG == NS_LONG - 1 || s + 1 == s1;
#pragma unroll
          for (int c = 0; c < 4; c += STEPS) {
            if (begins && used >= NS_SETS && !mbar_wait_warp(&acc_empty[set], set_lap ^ 1u, p.status, p.tag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t d = tmem + set * NS_TILE;
#pragma unroll
            for (int t = c; t < c + STEPS; ++t) pair_mma(d, a + L + t * a_step, a_hi, b + t * b_step, b_hi, idesc, t > c || !begins);
#pragma unroll
            for (int t = c; t < c + STEPS; ++t) pair_mma(d, a + t * a_step, a_hi, b + L + t * b_step, b_hi, idesc, 1u);
#pragma unroll
            for (int t = c; t < c + STEPS; ++t) pair_mma(d, a + t * a_step, a_hi, b + t * b_step, b_hi, idesc, 1u);
            if (c + STEPS == 4) pair_commit(&empty[slot], pair_mask);
            if (ends) {
              pair_commit(&acc_full[set], pair_mask);
              ++used;
              if (++set == NS_SETS) { set = 0; set_lap ^= 1u; }
            }
          }
          if (++slot == NS_STAGES) { slot = 0; lap ^= 1u; }
        }
      }
      // Behind an error: no MMA is under way when its tensor memory is given back.
      if (!ok)
        for (uint32_t i = 0; i < NS_SETS && i < used; ++i) {
          if (set == 0) { set = NS_SETS; set_lap ^= 1u; }
          --set;
          mbar_wait_warp(&acc_full[set], set_lap, p.status, p.tag);
        }
    }
  } else {
    const int quadrant = warp & 3, quarter = (warp - 2) >> 2, row = quadrant * 32 + lane;
    uint32_t set = 0, set_lap = 0;
    int k = first.k;
    bool ok = true;
    for (int u = u0; u < units && ok; u += step) {
      const NsUnit w = u == u0 ? first : ns_unit<MODE>(es, entries, u, k);
      float sum[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) sum[i] = 0.f;
      const int s0 = w.stages * part / split, s1 = w.stages * (part + 1) / split;
      const int chains = LONG ? (s1 - s0 + NS_LONG - 1) / NS_LONG : (s1 - s0) * (4 / NS_CHAIN);
      for (int c = 0; c < chains; ++c) {
        if (!mbar_wait_warp(&acc_full[set], set_lap, p.status, p.tag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t from = tmem + set * NS_TILE + quarter * 64 + ((uint32_t)(quadrant * 32) << 16);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t x[16], y[16];
          tmem_ld16_issue(from + q * 32, x);
          tmem_ld16_issue(from + q * 32 + 16, y);
          tmem_ld_wait(x); tmem_ld_wait(y);
          if (q == 1) {                              // all of the set's columns are read
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_at(&acc_empty[set], leader);
          }
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float2 f = __fadd2_rn(make_float2(sum[q * 32 + i], sum[q * 32 + i + 1]), make_float2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])));
            const float2 g = __fadd2_rn(make_float2(sum[q * 32 + 16 + i], sum[q * 32 + 17 + i]), make_float2(__uint_as_float(y[i]), __uint_as_float(y[i + 1])));
            sum[q * 32 + i] = f.x; sum[q * 32 + i + 1] = f.y; sum[q * 32 + 16 + i] = g.x; sum[q * 32 + 17 + i] = g.y;
          }
        }
        if (++set == NS_SETS) { set = 0; set_lap ^= 1u; }
      }
      if (!ok) break;
      if (!shared && MODE == NS_LAST && es[w.k].rows <= es[w.k].cols) {
        ns_emit_rows(p, es[w.k], w, (int)half, row, quarter, sum);
      } else if (!shared) {
#pragma unroll
        for (int q = 0; q < 8; q += 2) {
          float v[2][8];
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i / 8][i % 8] = sum[q * 8 + i];
          ns_emit<MODE, 2>(p, es[w.k], w, (int)half, row, quarter * 8 + q, v);
        }
      } else {
        // (one unit a cluster: every stage of this pair has been multiplied, and the ring's memory is free)
#pragma unroll
        for (int q = 0; q < 16; ++q)
          asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(smem + (uint32_t)(((quarter * 16 + q) * NS_PITCH + row) * 16)), "f"(sum[4 * q]), "f"(sum[4 * q + 1]),
                       "f"(sum[4 * q + 2]), "f"(sum[4 * q + 3]) : "memory");
      }
    }
    // (sums that are not there: none of the tile's is written)
    if (!ok && shared && lane < 2 * p.cs) st_cluster_u32(smem_u32(&lost), (uint32_t)lane, 1u);
  }
  __syncwarp();
  tc_fence_before();
  // No arrival and no copy of the pair comes behind this.
  if (!shared) {
    cluster_sync_relaxed();
  } else {
    cluster_sync();
    if (warp >= 2 && *reinterpret_cast<volatile uint32_t*>(&lost) == 0) {
      const NsUnit& w = first;
      const NsEntry& e = es[w.k];
      // This CTA's groups of eight columns; neighbouring lanes have neighbouring rows, or, where rows of the result are written, neighbouring columns.
      const int t = threadIdx.x - 64, groups = 32 / p.cs;
      const bool by_row = MODE == NS_LAST && e.rows <= e.cols;
      for (int x = t; x < 128 * groups; x += 512) {
        const int row = by_row ? x / groups : x & 127, q8 = part * groups + (by_row ? x % groups : x >> 7);
        float4 f[4], g[4];                             // (p.cs is 2 or 4)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (c < p.cs) {
            const uint32_t from = smem + (uint32_t)((2 * q8 * NS_PITCH + row) * 16);
            f[c] = ld_cluster_f4(from, 2u * c + half);
            g[c] = ld_cluster_f4(from + NS_PITCH * 16, 2u * c + half);
          }
        float v[1][8] = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (c < p.cs) {
            v[0][0] += f[c].x; v[0][1] += f[c].y; v[0][2] += f[c].z; v[0][3] += f[c].w;
            v[0][4] += g[c].x; v[0][5] += g[c].y; v[0][6] += g[c].z; v[0][7] += g[c].w;
          }
        ns_emit<MODE, 1>(p, e, w, (int)half, row, q8, v);
      }
    }
    __syncwarp();
    cluster_sync_relaxed();                          // (no CTA ends while its sums are read)
  }
  if (warp == 1) pair_dealloc(tmem);
}

// ---- matrices whose smaller side is at most 128, in one kernel: a cluster of up to eight CTAs a matrix, X in their shared memory

// Small matrices are bound by latencies: 17 kernels of 7 to 9 us each, of which the products take one (64 x 576, five steps: 136 us; here 55, with the tensor cores
// idle most of the time).  Here a CTA holds up to three blocks of 64 columns of X for all steps.  A
// step: the products of the CTA's own columns, summed over the cluster through the SMs' network (each CTA sums some columns and gives them to the others), then A A
// and B X in every CTA by itself.  Three chains of MMAs with a wait behind each; twelve in all where the cluster is one CTA.
constexpr int SMALL_THREADS = 512, SMALL_COLUMN_BLOCKS = 3;
constexpr int SMALL_ISSUERS = 4;                         // warps that issue MMAs, chains in turn: one warp takes some 80 clocks an MMA
// X: 128 rows of 192 values, a part behind the other; as in a block, eight rows' pieces lie side by side, with 24 pieces a row.
constexpr int SMALL_X_PIECES = SMALL_COLUMN_BLOCKS * 8;
constexpr uint32_t SMALL_X_GROUP = SMALL_X_PIECES * 128, SMALL_X_PART = 16 * SMALL_X_GROUP;
__device__ __forceinline__ uint32_t small_x_at(int row, int piece) { return (uint32_t)(row >> 3) * SMALL_X_GROUP + (uint32_t)(piece * 128 + (row & 7) * 16); }
constexpr uint32_t SMALL_X = 0, SMALL_A = SMALL_COLUMN_BLOCKS * NS_OPERAND, SMALL_E = SMALL_A + 2 * NS_OPERAND, SMALL_BYTES = SMALL_E + 2 * NS_OPERAND;
constexpr int SMALL_CLUSTER = 8;
static_assert(SMALL_COLUMN_BLOCKS * 2 * SMALL_THREADS * 32 <= SMALL_BYTES - SMALL_A, "rows of U");

__device__ __forceinline__ void st_cluster_v4(uint32_t addr, uint32_t rank, uint4 v) {
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.v4.b32 [a], {%2, %3, %4, %5};\n\t}"
               ::"r"(addr), "r"(rank), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void st_cluster_f64(uint32_t addr, uint32_t rank, double v) {
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.f64 [a], %2;\n\t}" ::"r"(addr), "r"(rank), "d"(v) : "memory");
}
__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async;" ::: "memory"); }

// An operand of the MMAs: its descriptor's halves, and what leads on to the next step of 16 terms and to the second part.
struct SmallOperand { uint32_t lo, hi, step, part; };
// A chain of a product: two steps of 16 terms, the small products first, into columns `d` of the tensor memory.
__device__ __forceinline__ void small_chain(uint32_t d, const SmallOperand& a, const SmallOperand& b, uint32_t idesc) {
  umma_warp(d, a.lo + a.part, a.hi, b.lo, b.hi, idesc, 0u);
  umma_warp(d, a.lo + a.part + a.step, a.hi, b.lo + b.step, b.hi, idesc, 1u);
  umma_warp(d, a.lo, a.hi, b.lo + b.part, b.hi, idesc, 1u);
  umma_warp(d, a.lo + a.step, a.hi, b.lo + b.part + b.step, b.hi, idesc, 1u);
  umma_warp(d, a.lo, a.hi, b.lo, b.hi, idesc, 1u);
  umma_warp(d, a.lo + a.step, a.hi, b.lo + b.step, b.hi, idesc, 1u);
}

struct SmallWait {             // for the MMAs that were issued last, by all threads; false where it ran out (the same in all lanes of a warp)
  uint64_t* bar;
  uint32_t parity;
  unsigned *status, tag;
  __device__ __forceinline__ bool operator()() {
    if (!mbar_wait_warp(bar, parity, status, tag)) return false;
    parity ^= 1u;
    tc_fence_after();
    return true;
  }
};

// GROUPS groups of 16 columns of the chains' sums from `from` on, chains `pitch` columns apart; two chains are loaded at once.
template <int GROUPS>
__device__ __forceinline__ void small_sums(float (&sum)[GROUPS * 16], uint32_t from, int chains, uint32_t pitch) {
#pragma unroll 1
  for (int c = 0; c < chains; c += 2) {
    const bool two = c + 1 < chains;
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) {
      uint32_t x[16], y[16];
      tmem_ld16_issue(from + c * pitch + q * 16, x);
      if (two) tmem_ld16_issue(from + (c + 1) * pitch + q * 16, y);
      tmem_ld_wait(x);
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[q * 16 + i] += __uint_as_float(x[i]);
      if (two) {
        tmem_ld_wait(y);
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[q * 16 + i] += __uint_as_float(y[i]);
      }
    }
  }
}

// Four columns of row r of the result in shared memory, rows of `pitch` floats.
__device__ __forceinline__ uint32_t small_result_at(uint32_t from, int r, int four, uint32_t pitch) {
  return from + (uint32_t)r * pitch * 4u + (uint32_t)((four ^ (r & 7)) << 4);
}
// The result's columns from col0 on leave in whole lines.  (A function of its own: its code and registers stay out of the steps'.)
template <typename T>
__device__ __forceinline__ void small_write_of(const NsArgs& p, const NsEntry& e, int mat, uint32_t from, uint32_t pitch, long col0) {
  T* out = static_cast<T*>(e.out) + (size_t)mat * e.n * e.m;
  const int width = (int)min((long)pitch, e.m - col0);
  if (e.rows > e.cols) {
#pragma unroll 4
    for (int i = threadIdx.x; i < 128 * width; i += SMALL_THREADS) {
      const int r = i & 127, c = i >> 7;
      if (r >= e.n) continue;
      float v;
      asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(small_result_at(from, r, c >> 2, pitch) + (uint32_t)(c & 3) * 4));
      T* to = out + (size_t)(col0 + c) * e.n + r;
      *to = from_f<T>(ns_result(p, e, v, p.muon ? to_f(*to) : 0.f));
    }
  } else {
    const int fours = (width + 3) / 4;
    const bool vec = e.m % 4 == 0;
#pragma unroll 2
    for (int i = threadIdx.x; i < e.n * fours; i += SMALL_THREADS) {
      const int r = i / fours, c4 = i - r * fours, left = width - c4 * 4;
      const float4 f = ld_shared_f4(small_result_at(from, r, c4, pitch));
      T* to = out + (size_t)r * e.m + col0 + c4 * 4;
      if (vec) {
        const float4 w = p.muon ? ld4(to) : make_float4(0.f, 0.f, 0.f, 0.f);
        st4(to, make_float4(ns_result(p, e, f.x, w.x), ns_result(p, e, f.y, w.y), ns_result(p, e, f.z, w.z), ns_result(p, e, f.w, w.w)));
      } else {
        const float v[4] = {f.x, f.y, f.z, f.w};
        float w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = p.muon && j < left ? to_f(to[j]) : 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < left) to[j] = from_f<T>(ns_result(p, e, v[j], w[j]));
      }
    }
  }
}
__device__ __noinline__ void small_write(const NsArgs& p, const NsEntry& e, int mat, uint32_t from, uint32_t pitch, long col0) {
  if (e.out_dtype == XCONV_F32) small_write_of<float>(p, e, mat, from, pitch, col0);
  else if (e.out_dtype == XCONV_BF16) small_write_of<bf16>(p, e, mat, from, pitch, col0);
  else small_write_of<f16>(p, e, mat, from, pitch, col0);
}

// N: columns of A that are worked on (n rounded up to 64 or 128).
// Where a wait runs out, its warp leaves what the MMAs read and write alone, the block issues nothing more and writes no result, and the warp waits once more (with
// the same limit) before the tensor memory is given back.  The CTAs of a cluster learn of it between the two barriers of the next step's sums, and end together: `gone`
// (a word of shared memory) is written before the first of these barriers and read behind it, so that all of a cluster's threads read the same.
template <int N>
__device__ __forceinline__ void small_steps(const NsArgs& p, const NsEntry& e, int mat, uint32_t smem, uint32_t tmem, SmallWait wait, int blocks, int cb0, int rank,
                                            uint32_t* gone) {
  constexpr int COLS = N / 4, CAP = 512 / N;                 // a thread's columns of A; chains that the tensor memory holds at once
  constexpr uint32_t ID = (1u << 4) | ((uint32_t)(TILE_M >> 4) << 24), ID_A = ID | ((uint32_t)(N >> 3) << 17);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quadrant = warp & 3, part = warp >> 2, row = quadrant * 32 + lane;
  const uint32_t lanes = (uint32_t)(quadrant * 32) << 16, base = smem & 0x3FFFFu;
  const int k_chains = (e.n + 31) / 32;
  // The operands of chain c: rows of X or A along the result, terms 32 c on; rows of X along the sum.
  const auto x_along = [&](int c) {
    return SmallOperand{((128u >> 4) << 16) | ((base + SMALL_X + (uint32_t)c * 512u) >> 4), (SMALL_X_GROUP >> 4) | (1u << 14), 256u >> 4, SMALL_X_PART >> 4};
  };
  const auto a_along = [&](int c) {
    return SmallOperand{((128u >> 4) << 16) | ((base + SMALL_A + (uint32_t)(c >> 1) * NS_OPERAND + (uint32_t)(c & 1) * 512u) >> 4), (1024u >> 4) | (1u << 14), 256u >> 4,
                        NS_PART >> 4};
  };
  const auto x_across = [&](int c, int block) {
    return SmallOperand{((SMALL_X_GROUP >> 4) << 16) | ((base + SMALL_X + (uint32_t)c * 4u * SMALL_X_GROUP + (uint32_t)block * 1024u) >> 4), (128u >> 4) | (1u << 14), 2u * SMALL_X_GROUP >> 4,
                        SMALL_X_PART >> 4};
  };
  bool ok = true, lost = false;                              // the warp's last wait; any of the block's (the same in all its threads)
#pragma unroll 1
  for (int step = 0; step < p.which; ++step) {
    float sum[COLS];
#pragma unroll
    for (int i = 0; i < COLS; ++i) sum[i] = 0.f;
    // the products of the CTA's own columns
    for (int c0 = 0; c0 < 2 * blocks && !lost; c0 += CAP) {
      const int chains = min(CAP, 2 * blocks - c0);
      if (warp < SMALL_ISSUERS) {
        for (int c = warp; c < chains; c += SMALL_ISSUERS) {
          const SmallOperand x = x_along(c0 + c);
          small_chain(tmem + c * N, x, x, ID_A);
        }
        umma_commit_warp(wait.bar);
      }
      ok = wait();
      if (ok) small_sums<COLS / 16>(sum, tmem + lanes + part * COLS, chains, N);
      tc_fence_before();
      lost = __syncthreads_or(!ok);
      tc_fence_after();
    }
    if (p.cs > 1) {
      // Their sum over the cluster: this CTA adds N / cs columns, and gives them to all.
#pragma unroll
      for (int q = 0; q < COLS / 4; ++q)
        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(smem + SMALL_E + (uint32_t)(((part * (COLS / 4) + q) * 128 + row) * 16)), "f"(sum[4 * q]),
                     "f"(sum[4 * q + 1]), "f"(sum[4 * q + 2]), "f"(sum[4 * q + 3]) : "memory");
      if (lost && threadIdx.x < p.cs) st_cluster_u32(smem_u32(gone), threadIdx.x, 1u);
      cluster_sync();
      if (*reinterpret_cast<volatile uint32_t*>(gone) != 0) break;
      const int groups = N / 8 / p.cs;                       // of eight columns
      for (int x = threadIdx.x; x < 128 * groups; x += SMALL_THREADS) {
        const int r = x & 127, q8 = rank * groups + (x >> 7);
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if ((r & ~31) < e.n) {
          for (int c0 = 0; c0 < p.cs; c0 += 4) {
            float4 f[4], g[4];
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if (c0 + c < p.cs) {
                f[c] = ld_cluster_f4(smem + SMALL_E + (uint32_t)((2 * q8 * 128 + r) * 16), c0 + c);
                g[c] = ld_cluster_f4(smem + SMALL_E + (uint32_t)(((2 * q8 + 1) * 128 + r) * 16), c0 + c);
              }
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if (c0 + c < p.cs) {
                v[0] += f[c].x; v[1] += f[c].y; v[2] += f[c].z; v[3] += f[c].w;
                v[4] += g[c].x; v[5] += g[c].y; v[6] += g[c].z; v[7] += g[c].w;
              }
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= NS_UNSCALE;
        uint4 hi, lo;
        parts8(v, hi, lo);
        const uint32_t at = smem + SMALL_A + (uint32_t)(q8 >> 3) * NS_OPERAND + piece_at(r, q8 & 7);
        if (step == 0 || (r & ~31) < e.n)                    // (rows of zeros stay zeros)
#pragma unroll
          for (int c = 0; c < SMALL_CLUSTER; ++c)
            if (c < p.cs) {
              st_cluster_v4(at, c, hi);
              st_cluster_v4(at + NS_PART, c, lo);
            }
      }
      fence_async();
      cluster_sync();
      fence_async();
    } else {
      if (lost) break;
#pragma unroll
      for (int q = 0; q < COLS / 8; ++q) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = sum[q * 8 + i] * NS_UNSCALE;
        uint4 hi, lo;
        parts8(v, hi, lo);
        const int q8 = part * (COLS / 8) + q;
        const uint32_t at = smem + SMALL_A + (uint32_t)(q8 >> 3) * NS_OPERAND + piece_at(row, q8 & 7);
        st_shared_v4(at, hi);
        st_shared_v4(at + NS_PART, lo);
      }
      fence_async_smem();
      __syncthreads();
    }
    // A A, and B in A's place
    if (warp < SMALL_ISSUERS) {
      tc_fence_after();
      for (int c = warp; c < k_chains; c += SMALL_ISSUERS) {
        const SmallOperand x = a_along(c);
        small_chain(tmem + c * N, x, x, ID_A);
      }
      umma_commit_warp(wait.bar);
    }
    ok = wait();
    if (ok) {
#pragma unroll
      for (int i = 0; i < COLS; ++i) sum[i] = 0.f;
      small_sums<COLS / 16>(sum, tmem + lanes + part * COLS, k_chains, N);
#pragma unroll
      for (int q = 0; q < COLS / 8; ++q) {
        const int q8 = part * (COLS / 8) + q;
        const uint32_t at = smem + SMALL_A + (uint32_t)(q8 >> 3) * NS_OPERAND + piece_at(row, q8 & 7);
        const uint4 ah = ld_shared_v4(at), al = ld_shared_v4(at + NS_PART);
        const uint32_t h[4] = {ah.x, ah.y, ah.z, ah.w}, l[4] = {al.x, al.y, al.z, al.w};
        const int d = row < e.n ? row - q8 * 8 : -1;
        float v[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h[k])), y = __half22float2(*reinterpret_cast<const __half2*>(&l[k]));
          v[2 * k] = fmaf(p.c * NS_UNSCALE, sum[q * 8 + 2 * k], p.b * (x.x + y.x)) + (d == 2 * k ? p.a * NS_SCALE : 0.f);
          v[2 * k + 1] = fmaf(p.c * NS_UNSCALE, sum[q * 8 + 2 * k + 1], p.b * (x.y + y.y)) + (d == 2 * k + 1 ? p.a * NS_SCALE : 0.f);
        }
        uint4 hi, lo;
        parts8(v, hi, lo);
        st_shared_v4(at, hi);
        st_shared_v4(at + NS_PART, lo);
      }
    }
    fence_async_smem();
    tc_fence_before();
    lost = __syncthreads_or(!ok);
    // B X: as many of the CTA's blocks of columns at once as the tensor memory holds the chains of
    const bool last = step + 1 == p.which;
    const int at_once = k_chains <= 2 ? SMALL_COLUMN_BLOCKS : 2;
#pragma unroll 1
    for (int b0 = 0; b0 < blocks && !lost; b0 += at_once) {
      const int here = min(at_once, blocks - b0);
      const uint32_t pitch = (uint32_t)here * 64u;
      if (warp < SMALL_ISSUERS) {
        tc_fence_after();
        const uint32_t id_x = ID | (1u << 16) | ((pitch >> 3) << 17);
        for (int c = warp; c < k_chains; c += SMALL_ISSUERS) small_chain(tmem + c * pitch, a_along(c), x_across(c, b0), id_x);
        umma_commit_warp(wait.bar);
      }
      ok = wait();
#pragma unroll 1
      for (int b = 0; ok && b < here; ++b) {
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
        small_sums<1>(x, tmem + lanes + b * 64 + part * 16, k_chains, pitch);
        const int c8 = (b0 + b) * 8 + part * 2;              // of the CTA's pieces of eight columns
        if (!last) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = x[q * 8 + i] * NS_UNSCALE;
            uint4 hi, lo;
            parts8(v, hi, lo);
            const uint32_t at = smem + SMALL_X + small_x_at(row, c8 + q);
            st_shared_v4(at, hi);
            st_shared_v4(at + SMALL_X_PART, lo);
          }
        } else if (row < e.n) {                              // (128 rows of 128 columns, or 64 of 192: where the cluster's sums were)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(small_result_at(smem + SMALL_E, row, b * 16 + part * 4 + k, pitch)), "f"(x[4 * k]), "f"(x[4 * k + 1]), "f"(x[4 * k + 2]),
                         "f"(x[4 * k + 3]) : "memory");
        }
      }
      tc_fence_before();
      if (!last) fence_async_smem();
      lost = __syncthreads_or(!ok);
      if (last && !lost) {
        small_write(p, e, mat, smem + SMALL_E, pitch, (long)(cb0 + b0) * NS_COLS);
        __syncthreads();
      }
    }
    if (warp < SMALL_ISSUERS) tc_fence_after();
    if (lost && p.cs == 1) break;
  }
  if (!ok) wait();
}

// ---- the same with a smaller side of at most 32, by FP32 multiply-adds in the same kernel
//
// Their sums are rounded to nearest, where the tensor cores cut them off; with few terms that shows: error against 64 bits, times that of float arithmetic by
// the library, root mean square over 200 to 2000 normal matrices, 1.25 on the tensor cores and 0.68 here (16 x 75; 24 x 40: 1.67 and 0.67; 32 x 64: 1.89 and 0.66; 32 x 288: 1.61
// and 0.47).  Nothing waits for MMAs either.  Bound by the loads from shared memory, of which a thread shares each among its products.  Measured, five steps, tensor cores and this: 6 x 75 30.7 and
// 16.4 us, 16 x 384 47 and 31, 32 x 32 24.6 and 22.6, 32 x 192 36.9 and 43.0, 32 x 256 41.0 and 36.9; three layers of 16 x 75 to 32 x 800 (a cluster of eight) 45 and 45.

constexpr int TINY = 32, TINY_X = SMALL_COLUMN_BLOCKS * 64 + 4, TINY_A = TINY + 4;      // rows; floats of a row of X, of A and B (16 bytes more: eight rows in different banks)

__device__ __forceinline__ float ld_shared_f(uint32_t addr) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ void st_shared_f(uint32_t addr, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }
__device__ __forceinline__ float4 add4(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
// The products of row i with rows j and, with TWO, j + 16 over `fours` groups of four columns (eight lanes read eight rows in a row: different banks).
template <bool TWO>
__device__ __forceinline__ float2 tiny_products(uint32_t rows, int pitch, int i, int j, int fours) {
  float2 s = make_float2(0.f, 0.f), t = s;
  uint32_t at = rows + (uint32_t)(i * pitch) * 4, to = rows + (uint32_t)(j * pitch) * 4;
  const uint32_t next = (uint32_t)pitch * 64;
#pragma unroll 4
  for (int c = 0; c < fours; ++c, at += 16, to += 16) {
    const float4 a = ld_shared_f4(at), x = ld_shared_f4(to);
    s.x = fmaf(a.x, x.x, s.x); t.x = fmaf(a.y, x.y, t.x);
    s.x = fmaf(a.z, x.z, s.x); t.x = fmaf(a.w, x.w, t.x);
    if (TWO) {
      const float4 y = ld_shared_f4(to + next);
      s.y = fmaf(a.x, y.x, s.y); t.y = fmaf(a.y, y.y, t.y);
      s.y = fmaf(a.z, y.z, s.y); t.y = fmaf(a.w, y.w, t.y);
    }
  }
  return make_float2(s.x + t.x, s.y + t.y);
}
template <typename T>
__device__ __forceinline__ void tiny_write(const NsArgs& p, const NsEntry& e, int mat, int row, long col, float v) {
  T* to = static_cast<T*>(e.out) + (size_t)mat * e.n * e.m + (e.rows > e.cols ? (size_t)col * e.n + row : (size_t)row * e.m + col);
  *to = from_f<T>(ns_result(p, e, v * (NS_SCALE * NS_SCALE), p.muon ? to_f(*to) : 0.f));
}

// X X^T of 32 rows over groups of four columns, by 4 x 2 products a thread (six 16-byte loads for 32 multiply-adds, which is what bounds it) and a quarter of the
// columns a warp: the quarters' sums to `to`.
__device__ __forceinline__ void tiny_gram(uint32_t X, uint32_t to, int fours) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, i = lane >> 2, j = (warp & 3) * 8 + (lane & 3), quarter = warp >> 2;
  float s[4][2] = {}, t[4][2] = {};
  const int end = fours * (quarter + 1) >> 2;
#pragma unroll 2
  for (int c = fours * quarter >> 2; c < end; ++c) {
    float4 a[4], b[2];
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] = ld_shared_f4(X + (uint32_t)((i + 8 * k) * TINY_X + c * 4) * 4);
#pragma unroll
    for (int k = 0; k < 2; ++k) b[k] = ld_shared_f4(X + (uint32_t)((j + 4 * k) * TINY_X + c * 4) * 4);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int l = 0; l < 2; ++l) {
        s[k][l] = fmaf(a[k].x, b[l].x, s[k][l]); t[k][l] = fmaf(a[k].y, b[l].y, t[k][l]);
        s[k][l] = fmaf(a[k].z, b[l].z, s[k][l]); t[k][l] = fmaf(a[k].w, b[l].w, t[k][l]);
      }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int l = 0; l < 2; ++l) st_shared_f(to + (uint32_t)(quarter * TINY * TINY_A + (i + 8 * k) * TINY_A + j + 4 * l) * 4, s[k][l] + t[k][l]);
}

// X: 32 rows of TINY_X floats at SMALL_X, of which the CTA's columns are there and zeros. N: 16 or 32 rows at most.
template <int N>
__device__ __noinline__ void tiny_steps(const NsArgs& p, const NsEntry& e, int mat, uint32_t smem, int blocks, int cb0) {
  constexpr bool TWO = N > 16;
  constexpr int COLS = N / 16, ROWS = N / (4 * COLS);       // of B X a thread, the columns 128 / COLS apart
  const int t = threadIdx.x, i = t >> 4, j = t & 15;
  const uint32_t X = smem + SMALL_X, A = smem + SMALL_A, B = A + TINY * TINY_A * 4, at = (uint32_t)(i * TINY_A + j) * 4;
  const int columns = min(blocks * 64, e.m - cb0 * NS_COLS);
#pragma unroll 1
  for (int step = 0; step < p.which; ++step) {
    // The CTA's sums, then the cluster's, four neighbouring ones a thread (those sums in two buffers in turn: one is written again two barriers later).
    const uint32_t parts = smem + SMALL_E + 2u * (TINY * TINY_A * 4), sums = smem + SMALL_E + (uint32_t)(step & 1) * (TINY * TINY_A * 4);
    const uint32_t at4 = (uint32_t)((t >> 3) * TINY_A + (t & 7) * 4) * 4;
    const bool adds = t < N * 8 && (TWO || (t & 7) < 4);
    if (TWO) tiny_gram(X, parts, (columns + 3) >> 2);
    else if (i < N) st_shared_f(parts + at, tiny_products<false>(X, TINY_X, i, j, (columns + 3) >> 2).x);
    __syncthreads();
    if (adds) {
      float4 v = ld_shared_f4(parts + at4);
      if (TWO) {
#pragma unroll
        for (int q = 1; q < 4; ++q) v = add4(v, ld_shared_f4(parts + at4 + (uint32_t)(q * TINY * TINY_A) * 4));
      }
      st_shared_v4((p.cs > 1 ? sums : A) + at4, make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)));
    }
    if (p.cs > 1) {
      cluster_sync();
      if (adds) {
        float4 f[SMALL_CLUSTER];
#pragma unroll
        for (int c = 0; c < SMALL_CLUSTER; ++c) f[c] = c < p.cs ? ld_cluster_f4(sums + at4, c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int c = 1; c < SMALL_CLUSTER; ++c) f[0] = add4(f[0], f[c]);
        st_shared_v4(A + at4, make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[0].z), __float_as_uint(f[0].w)));
      }
    }
    __syncthreads();
    if (i < N) {
      const float2 q = tiny_products<TWO>(A, TINY_A, i, j, N / 4);
      st_shared_f(B + at, fmaf(p.c, q.x, p.b * ld_shared_f(A + at)) + (i == j && i < e.n ? p.a : 0.f));
      if (TWO) st_shared_f(B + at + 64, fmaf(p.c, q.y, p.b * ld_shared_f(A + at + 64)) + (i == j + 16 && i < e.n ? p.a : 0.f));
    }
    const bool last = step + 1 == p.which;
    // 128 columns at a time: all have read them before one writes.
#pragma unroll 1
    for (int c0 = 0; c0 < columns; c0 += 128) {
      const int c = c0 + t % (128 / COLS), r0 = t / (128 / COLS) * ROWS;
      const uint32_t col = X + (uint32_t)c * 4;
      float x[COLS][N];
#pragma unroll
      for (int l = 0; l < COLS; ++l)
#pragma unroll
        for (int k = 0; k < N; ++k) x[l][k] = c + l * (128 / COLS) < columns ? ld_shared_f(col + (uint32_t)(k * TINY_X + l * (128 / COLS)) * 4) : 0.f;
      __syncthreads();
#pragma unroll 1
      for (int r = r0; r < r0 + ROWS; ++r) {
        float y[COLS] = {}, z[COLS] = {};
#pragma unroll
        for (int k = 0; k < N; k += 4) {
          const float4 w = ld_shared_f4(B + (uint32_t)(r * TINY_A + k) * 4);
#pragma unroll
          for (int l = 0; l < COLS; ++l) {
            y[l] = fmaf(w.x, x[l][k], y[l]); z[l] = fmaf(w.y, x[l][k + 1], z[l]);
            y[l] = fmaf(w.z, x[l][k + 2], y[l]); z[l] = fmaf(w.w, x[l][k + 3], z[l]);
          }
        }
#pragma unroll
        for (int l = 0; l < COLS; ++l) {
          const int cl = c + l * (128 / COLS);
          if (cl >= columns) continue;
          const float v = y[l] + z[l];
          if (!last) st_shared_f(X + (uint32_t)(r * TINY_X + cl) * 4, v);
          else if (r < e.n) {
            const long to = (long)cb0 * NS_COLS + cl;
            if (e.out_dtype == XCONV_F32) tiny_write<float>(p, e, mat, r, to, v);
            else if (e.out_dtype == XCONV_BF16) tiny_write<bf16>(p, e, mat, r, to, v);
            else tiny_write<f16>(p, e, mat, r, to, v);
          }
        }
      }
    }
    __syncthreads();
  }
}

// Pieces 4 i + q0 of row r of the CTA's columns of U, as floats where the thread finds them again; the momenta take in the gradients on the way.  Returns the sum of
// their squares.
template <typename G>
__device__ __forceinline__ double small_load(const NsArgs& p, const NsEntry& e, size_t base, int r, int q0, int cb0, int blocks, uint32_t to) {
  const G* g = static_cast<const G*>(e.g) + base;
  float* mom = p.muon ? e.mom + base : nullptr;
  const bool tall = e.rows > e.cols, vec = !tall && e.m % 8 == 0;
  double s = 0.0;
#pragma unroll 2
  for (int i = 0; i < 2 * blocks; ++i) {
    const long c0 = (long)cb0 * NS_COLS + (i * 4 + q0) * 8;
    const int left = r < e.n ? (int)min(8L, e.m - c0) : 0;   // (columns that are there)
    const size_t at = tall ? (size_t)c0 * e.n + r : (size_t)r * e.m + c0, apart = tall ? e.n : 1;
    float u[8], m[8];
    if (vec) {
      const float4 z = make_float4(0.f, 0.f, 0.f, 0.f), a = left > 0 ? ld4(g + at) : z, b = left > 0 ? ld4(g + at + 4) : z;
      u[0] = a.x; u[1] = a.y; u[2] = a.z; u[3] = a.w; u[4] = b.x; u[5] = b.y; u[6] = b.z; u[7] = b.w;
      if (mom) {
        const float4 c = left > 0 ? ld4(mom + at) : z, d = left > 0 ? ld4(mom + at + 4) : z;
        m[0] = c.x; m[1] = c.y; m[2] = c.z; m[3] = c.w; m[4] = d.x; m[5] = d.y; m[6] = d.z; m[7] = d.w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        u[j] = j < left ? to_f(g[at + j * apart]) : 0.f;
        if (mom) m[j] = j < left ? mom[at + j * apart] : 0.f;
      }
    }
    if (mom) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = fmaf(1.f - p.momentum, u[j] - m[j], m[j]);
        u[j] = update_of(u[j], m[j], p.momentum, p.nesterov);
      }
      if (vec) {
        if (left > 0) {
          st4(mom + at, make_float4(m[0], m[1], m[2], m[3]));
          st4(mom + at + 4, make_float4(m[4], m[5], m[6], m[7]));
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < left) mom[at + j * apart] = m[j];
      }
    }
    const uint32_t own = to + (uint32_t)(i * 2 * SMALL_THREADS + threadIdx.x) * 16;
    st_shared_v4(own, make_uint4(__float_as_uint(u[0]), __float_as_uint(u[1]), __float_as_uint(u[2]), __float_as_uint(u[3])));
    st_shared_v4(own + SMALL_THREADS * 16, make_uint4(__float_as_uint(u[4]), __float_as_uint(u[5]), __float_as_uint(u[6]), __float_as_uint(u[7])));
#pragma unroll
    for (int j = 0; j < 8; ++j) s += (double)u[j] * u[j];
  }
  return s;
}

__global__ void __launch_bounds__(SMALL_THREADS, 1) ns_small_kernel(const __grid_constant__ NsArgs p) {
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t done;
  __shared__ uint32_t tmem_slot, gone;
  __shared__ double warp_sums[SMALL_THREADS / 32], cta_sums[SMALL_CLUSTER];
  const uint32_t smem = (smem_u32(raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = p.cs > 1 ? (int)cluster_rank() : 0, unit = (int)blockIdx.x / p.cs;
  if (threadIdx.x == 0) {
    mbar_init(&done, SMALL_ISSUERS);
    gone = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) tmem_alloc_then_trigger(&tmem_slot, 512);
  int k = 0;
  while (k + 1 < p.t.entries && unit >= p.t.e[k + 1].sym0) ++k;
  const NsEntry& e = p.t.e[k];
  const int mat = unit - e.sym0, kt = x_cols(e), per = (kt + p.cs - 1) / p.cs, cb0 = rank * per, blocks = max(0, min(per, kt - cb0));
  pdl_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) reinterpret_cast<volatile unsigned*>(p.status)[1] = p.tag;
  // U of the CTA's columns, two pieces of eight columns a block and thread (neighbouring threads have neighbouring rows); a tall matrix's rows are X's columns
  const size_t base = (size_t)mat * e.n * e.m;
  const int r = threadIdx.x & 127, q0 = threadIdx.x >> 7;
  const uint32_t staged = smem + SMALL_A;                    // (a thread's own values)
  double s = e.g_dtype == XCONV_F32    ? small_load<float>(p, e, base, r, q0, cb0, blocks, staged)
             : e.g_dtype == XCONV_BF16 ? small_load<bf16>(p, e, base, r, q0, cb0, blocks, staged)
                                       : small_load<f16>(p, e, base, r, q0, cb0, blocks, staged);
  // the norm, over the cluster in fixed order
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) warp_sums[warp] = s;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (p.cs > 1) {
    cluster_sync();                                          // (the others have begun)
    if (threadIdx.x < p.cs) {
      s = 0.0;
      for (int w = 0; w < SMALL_THREADS / 32; ++w) s += warp_sums[w];
      st_cluster_f64(smem_u32(&cta_sums[rank]), threadIdx.x, s);
    }
    __syncwarp();
    cluster_sync();
    s = 0.0;
    for (int c = 0; c < p.cs; ++c) s += cta_sums[c];
  } else {
    s = 0.0;
    for (int w = 0; w < SMALL_THREADS / 32; ++w) s += warp_sums[w];
  }
  const NsScale f(s, p.eps);
  for (int i = 0; i < 2 * blocks; ++i) {
    const uint32_t own = staged + (uint32_t)(i * 2 * SMALL_THREADS + threadIdx.x) * 16;
    const float4 a = ld_shared_f4(own), b = ld_shared_f4(own + SMALL_THREADS * 16);
    float v[8] = {f(a.x), f(a.y), f(a.z), f(a.w), f(b.x), f(b.y), f(b.z), f(b.w)};
    if (e.n <= TINY) {
      if (r >= TINY) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= NS_UNSCALE;
      const uint32_t at = smem + SMALL_X + (uint32_t)(r * TINY_X + (i * 4 + q0) * 8) * 4;
      st_shared_v4(at, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
      st_shared_v4(at + 16, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])));
      continue;
    }
    uint4 hi, lo;
    parts8(v, hi, lo);
    const uint32_t at = smem + SMALL_X + small_x_at(r, i * 4 + q0);
    st_shared_v4(at, hi);
    st_shared_v4(at + SMALL_X_PART, lo);
  }
  fence_async_smem();
  __syncthreads();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&tmem_slot);
  const SmallWait wait = {&done, 0u, p.status, p.tag};
  if (e.n <= 16) tiny_steps<16>(p, e, mat, smem, blocks, cb0);
  else if (e.n <= TINY) tiny_steps<TINY>(p, e, mat, smem, blocks, cb0);
  else if (e.n <= 64) small_steps<64>(p, e, mat, smem, tmem, wait, blocks, cb0, rank, &gone);
  else small_steps<128>(p, e, mat, smem, tmem, wait, blocks, cb0, rank, &gone);
  tc_fence_before();
  __syncthreads();
  if (p.cs > 1) cluster_sync_relaxed();                      // (no CTA ends while the others read its sums)
  if (warp == 0) tmem_dealloc(tmem, 512);
}

// Whether all matrices are small ones.
bool all_small(const NsTable& t) {
  for (int k = 0; k < t.entries; ++k)
    if (t.e[k].n > NS_ROWS || x_cols(t.e[k]) > SMALL_COLUMN_BLOCKS * SMALL_CLUSTER) return false;
  return true;
}

cudaError_t launch_small(NsArgs& p, int matrices, cudaStream_t st) {
  constexpr size_t smem = SMALL_BYTES + 1024;
  int kt = 1;
  for (int k = 0; k < p.t.entries; ++k) kt = std::max(kt, x_cols(p.t.e[k]));
  p.cs = 1;
  while (p.cs * SMALL_COLUMN_BLOCKS < kt) p.cs *= 2;
  const cudaError_t e = cudaFuncSetAttribute(ns_small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(matrices * p.cs));
  cfg.blockDim = dim3(SMALL_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.cs;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.cs > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, ns_small_kernel, p);
}

// How the tiles of a launch go to the pairs of CTAs: by the times that a stage (1800 clocks), a tile's results (3000) and sums that pairs exchange (11000) take.  Those that
// are shared are the first of the table, which is in the order of the matrices' larger sides: the longest sums first in X X^T, while in A A and B X, whose sums are as long
// as the smaller sides, a long sum may stand behind short ones and is then shared with all of those or not at all.
//
// Measured, five steps of float matrices, in us: no tile shared, all by two pairs, all by four (where the GPU has so many clusters), and by this rule.  256 x 256 154 155 152 154;
// 512 x 512 215 187 170 170; 512 x 4608 509 346 265 265; four of them 616 455 378 378; 200 x 8000 701 438 298 303; 1024 x 1024 326 252 270 270; two of them 329 263 329 264;
// 1024 x 4096 572 409 330 329; 16 of 256 x 256 163 169 299 162; 2048 x 2048 605 (too many tiles) 603; 512 x 4608 beside 40 of 256 x 256 584 (too many) 346.
struct NsSharing { int cs, heavy; };
template <typename Stages, typename Units>
NsSharing share(const NsTable& t, int units, Stages&& stages, Units&& units_of) {
  double all = 0.0;
  int longest = 1;
  for (int k = 0; k < t.entries; ++k) {
    all += (double)units_of(t.e[k]) * stages(t.e[k]);
    longest = std::max(longest, stages(t.e[k]));
  }
  const int pairs = NS_SMS / 2;
  NsSharing best = {1, 0};
  double least = 1800.0 * std::max<double>(longest, all / pairs) + 3000.0 * ((units + pairs - 1) / pairs);
  // (clusters that are on the SMs at once: eight CTAs within a group of 16 to 20 SMs, two or three short of the SMs' number)
  for (const NsSharing& size : {NsSharing{2, 32}, NsSharing{4, 16}}) {
    int heavy = 0, first = 1;
    for (int k = 0; k < t.entries; ++k) {
      heavy += units_of(t.e[k]);
      first = std::max(first, stages(t.e[k]));
      int rest = 0;
      for (int j = k + 1; j < t.entries; ++j) rest = std::max(rest, stages(t.e[j]));
      if (heavy + (units - heavy + size.cs - 1) / size.cs > size.heavy) break;
      const double time = std::max(1800.0 * ((first + size.cs - 1) / size.cs) + 11000.0, rest ? 1800.0 * rest + 3000.0 : 0.0);
      if (time < least) { least = time; best = {size.cs, heavy}; }
    }
  }
  return best;
}

template <int MODE, bool LONG>
cudaError_t launch_product(NsArgs& p, cudaStream_t st) {
  constexpr bool SYM = MODE == NS_GRAM || MODE == NS_SQUARE;
  constexpr size_t smem = NS_STAGES * NS_STAGE + 1024;
  const int units = SYM ? p.t.syms : p.t.prods;
  const NsSharing how = share(p.t, units, [](const NsEntry& e) { return MODE == NS_GRAM ? x_cols(e) : a_terms(e); }, [](const NsEntry& e) {
    const int rows = tiles(row_blocks(e), 2);
    return e.count * (SYM ? rows * (rows + 1) / 2 : rows * tiles(x_cols(e), 4));
  });
  p.cs = how.cs;
  p.heavy = how.heavy;
  cudaError_t e = cudaFuncSetAttribute(ns_product_kernel<MODE, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.cs > 1 ? 2 * p.cs * (p.heavy + (units - p.heavy + p.cs - 1) / p.cs) : std::min(2 * units, NS_SMS)));
  cfg.blockDim = dim3(NS_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)(2 * p.cs);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, ns_product_kernel<MODE, LONG>, p);
}

// The scratch memory's blocks as rows of 256 values of 8 bytes, 16 of them a block and a copy.  (The copy engine fetches a box row by row: long rows.)  And as rows
// of 128 such values, 32 of them a block: 8 rows of two neighbouring blocks a copy, row by row.
bool map_blocks(CUtensorMap* whole, CUtensorMap* across, void* blocks, size_t count) {
  PFN_cuTensorMapEncodeTiled_v12000 fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {256, count * 16}, strides[1] = {2048}, dims3[3] = {128, count, 32}, strides3[2] = {NS_BLOCK, 1024};
  const cuuint32_t box[2] = {256, 16}, box3[3] = {128, 2, 8}, steps[3] = {1, 1, 1};
  return fn(whole, CU_TENSOR_MAP_DATA_TYPE_INT64, 2, blocks, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS &&
         fn(across, CU_TENSOR_MAP_DATA_TYPE_INT64, 3, blocks, dims3, strides3, box3, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool LONG>
cudaError_t launch_steps(NsArgs& p, int steps, cudaStream_t st, int* launches) {
  cudaError_t e;
  for (int s = 0; s < steps; ++s) {
    p.which = s & 1;
    if ((e = launch_product<NS_GRAM, LONG>(p, st)) != cudaSuccess) return e;
    ++*launches;
    if ((e = launch_product<NS_SQUARE, LONG>(p, st)) != cudaSuccess) return e;
    ++*launches;
    if ((e = s + 1 < steps ? launch_product<NS_APPLY, LONG>(p, st) : launch_product<NS_LAST, LONG>(p, st)) != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

size_t sums_bytes(const NsTable& t) { return ((size_t)t.chunks * sizeof(double) + 1023) / 1024 * 1024; }

}  // namespace

size_t ns_blocks_of(long rows, long cols) {
  const long n = std::min(rows, cols), m = std::max(rows, cols);
  const size_t nt = (size_t)((n + NS_ROWS - 1) / NS_ROWS);
  return 2 * nt * (size_t)((m + NS_COLS - 1) / NS_COLS) + 2 * nt * 2 * nt;
}

void ns_add(NsTable* t, NsEntry e) {
  e.n = std::min(e.rows, e.cols);
  e.m = std::max(e.rows, e.cols);
  const int nt = row_blocks(e);
  const int tall = tiles(nt, 2);
  const uint32_t x = (uint32_t)e.count * nt * x_cols(e), a = (uint32_t)e.count * nt * a_cols(e);
  e.x0 = t->ws_blocks; e.x1 = e.x0 + x; e.a = e.x1 + x; e.b = e.a + a;
  t->ws_blocks = e.b + a;
  e.chunk0 = t->chunks; e.block0 = t->blocks; e.sym0 = t->syms; e.prod0 = t->prods;
  t->chunks += e.count * chunks_of(e);
  t->blocks += (int)x;
  t->syms += e.count * (tall * (tall + 1) / 2);
  t->prods += e.count * tall * tiles(x_cols(e), 4);
  t->e[t->entries++] = e;
}

size_t ns_bytes(const NsTable& t) { return all_small(t) ? 0 : sums_bytes(t) + t.ws_blocks * NS_BLOCK; }

cudaError_t launch_newton_schulz(const NsTable& t, const NsOptions& o, void* ws, unsigned tag, cudaStream_t st, int* launches) {
  NsArgs p = {};
  p.t = t;
  p.status = static_cast<unsigned*>(ws);
  p.tag = tag;
  p.sums = reinterpret_cast<double*>(static_cast<char*>(ws) + NS_HEADER);
  p.blocks = static_cast<char*>(ws) + NS_HEADER + sums_bytes(t);
  p.a = o.a; p.b = o.b; p.c = o.c; p.eps = o.eps; p.momentum = o.momentum; p.keep = o.keep; p.muon = o.muon; p.nesterov = o.nesterov;
  if (all_small(t)) {
    int matrices = 0;
    for (int k = 0; k < t.entries; ++k) {
      p.t.e[k].sym0 = matrices;
      matrices += t.e[k].count;
    }
    p.which = o.steps;
    ++*launches;
    return launch_small(p, matrices, st);
  }
  if (!map_blocks(&p.whole, &p.across, p.blocks, t.ws_blocks)) return cudaErrorInvalidValue;
  cudaError_t e = launch_pdl(ns_squares_kernel, dim3((unsigned)t.chunks), dim3(256), 0, st, p);
  if (e != cudaSuccess) return e;
  ++*launches;
  e = launch_pdl(ns_blocks_kernel, dim3((unsigned)t.blocks), dim3(256), 0, st, p);
  if (e != cudaSuccess) return e;
  ++*launches;
  bool halves = true;                                        // every result is rounded to 16 bits
  for (int k = 0; k < t.entries; ++k) halves = halves && t.e[k].out_dtype != XCONV_F32;
  return halves ? launch_steps<true>(p, o.steps, st, launches) : launch_steps<false>(p, o.steps, st, launches);
}

}  // namespace xconv
