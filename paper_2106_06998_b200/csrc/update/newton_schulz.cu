// Orthogonalisation by Newton-Schulz products: X0 = U / max(|U|_F, eps), n x m with n <= m (transposed where it is taller than wide), then `steps` times
//
//   A = X X^T,   B = a I + b A + c A A,   X <- B X
//
// which maps every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors.  Any number of matrices of any shapes goes through the same launches: the
// unit of work is a 128 x 128 tile of some matrix's product.
//
// Arithmetic.  A step multiplies small singular values by a (3.4): an error of the operands' roundings grows by 485 in five steps where X has large singular
// values beside small ones.  With operands rounded to bfloat16 the result is off by 1e-2 (normal values) to 0.3 (eight directions above noise), with one float16 part
// by 1e-3 to 4e-2; with float arithmetic by 1e-7 to 5e-6.  So every operand is two float16 parts here, x 2^13 = h + l (11 + 11 bits and the sign between
// them; |X| < 2, |A| < 4, |B| < 8: nothing overflows, and what is lost is below 2^-38), and a product is l h + h l + h h on the tensor cores, as exact as one of floats.
// The tensor cores' accumulator is not rounded to nearest; a chain is one stage (64 terms: eight MMAs of the small products, then four of h h), and the chains
// are added in float registers.
//
// Layout.  X, A and B lie in the scratch memory as blocks of 128 x 64 values, each part 16 KB in the order that the MMA wants in shared memory (rows of 128
// bytes, 16-byte pieces exchanged by the row's last three bits): one untiled bulk copy fetches a block, whatever the matrix's sizes, and the same block serves as
// a tile whose rows run along the result (X X^T, A A, B of B X) and as one whose rows run along the sum (X of B X).  Behind a matrix's last row and column lie zeros.
// A and A A are symmetric: the tiles on and below the diagonal are computed and written twice, and rows of A serve as its columns.
//
// A block of threads: a warp that copies, one that issues MMAs, eight that add chains and write results.  Where there are fewer tiles than SMs, a cluster of
// 2, 4 or 8 shares the terms of a tile; each then has a part of the tile's columns, and reads the others' sums of them over the SMs' network.
#include "newton_schulz.h"

#include <algorithm>

#include "../split_f32.cuh"

namespace xconv {

namespace {

constexpr int NS_SMS = 148;
constexpr int NS_STAGES = 3, NS_SETS = 4;
constexpr uint32_t NS_OPERAND = 32 * 1024, NS_STAGE = 2 * NS_OPERAND, NS_PART = NS_OPERAND / 2;
constexpr int NS_ADDERS = 8, NS_THREADS = 32 * (2 + NS_ADDERS);
constexpr float NS_SCALE = 8192.f, NS_UNSCALE = 1.f / 8192.f;
constexpr size_t NS_HEADER = 256;

enum { NS_GRAM, NS_SQUARE, NS_APPLY, NS_LAST };

struct NsArgs {
  NsTable t;
  char* blocks;                // the blocks of the scratch memory
  double* sums;                // partial sums of squares, NS_CHUNK values each
  unsigned *status, tag;
  float a, b, c, momentum, keep;
  double eps;
  int muon, nesterov, which;   // which: the buffer that X is in
  int cs;                      // CTAs a tile
};

__device__ __forceinline__ float load_as_float(const void* p, int dtype, size_t i) {
  if (dtype == XCONV_F32) return static_cast<const float*>(p)[i];
  if (dtype == XCONV_BF16) return to_f(static_cast<const bf16*>(p)[i]);
  return to_f(static_cast<const f16*>(p)[i]);
}
__device__ __forceinline__ void store_from_float(void* p, int dtype, size_t i, float v) {
  if (dtype == XCONV_F32) static_cast<float*>(p)[i] = v;
  else if (dtype == XCONV_BF16) static_cast<bf16*>(p)[i] = from_f<bf16>(v);
  else static_cast<f16*>(p)[i] = from_f<f16>(v);
}

__host__ __device__ __forceinline__ int chunks_of(const NsEntry& e) { return (int)(((long)e.n * e.m + NS_CHUNK - 1) / NS_CHUNK); }
__host__ __device__ __forceinline__ int row_blocks(const NsEntry& e) { return (e.n + NS_ROWS - 1) / NS_ROWS; }
__host__ __device__ __forceinline__ int x_cols(const NsEntry& e) { return (e.m + NS_COLS - 1) / NS_COLS; }
__host__ __device__ __forceinline__ int a_cols(const NsEntry& e) { return (e.n + NS_COLS - 1) / NS_COLS; }

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
__device__ __forceinline__ uint32_t piece_at(int row, int piece) { return (uint32_t)row * 128u + (uint32_t)((piece ^ (row & 7)) << 4); }

// ---- momenta and sums of squares: a block of threads per NS_CHUNK values

__device__ __forceinline__ float update_of(float g, float m, float mu, int nesterov) { return nesterov ? fmaf(mu, m - g, g) : m; }

__global__ void __launch_bounds__(256) ns_squares_kernel(const __grid_constant__ NsArgs p) {
  __shared__ double sums[8];
  pdl_wait();
  int k = 0;
  while (k + 1 < p.t.entries && (int)blockIdx.x >= p.t.e[k + 1].chunk0) ++k;
  const NsEntry& e = p.t.e[k];
  const int local = (int)blockIdx.x - e.chunk0, per = chunks_of(e), mat = local / per;
  const long size = (long)e.n * e.m, first = (long)(local - mat * per) * NS_CHUNK, last = min(size, first + NS_CHUNK), base = (long)mat * size;
  double s = 0.0;
  if (p.muon) {
    float* mom = e.mom + base;
    for (long i = first + threadIdx.x; i < last; i += 256) {
      const float g = load_as_float(e.g, e.g_dtype, (size_t)(base + i));
      const float m = fmaf(1.f - p.momentum, g - mom[i], mom[i]);
      mom[i] = m;
      const double u = (double)update_of(g, m, p.momentum, p.nesterov);
      s += u * u;
    }
  } else {
    for (long i = first + threadIdx.x; i < last; i += 256) {
      const double u = (double)load_as_float(e.g, e.g_dtype, (size_t)(base + i));
      s += u * u;
    }
  }
  pdl_trigger();
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) s += sums[w];
    p.sums[blockIdx.x] = s;
  }
}

// ---- X0 in blocks: a block of threads per block of 128 x 64 values

__global__ void __launch_bounds__(256) ns_blocks_kernel(const __grid_constant__ NsArgs p) {
  __shared__ float tile[NS_ROWS][NS_COLS + 1];
  __shared__ double sums[8];
  pdl_wait();
  pdl_trigger();
  int k = 0;
  while (k + 1 < p.t.entries && (int)blockIdx.x >= p.t.e[k + 1].block0) ++k;
  const NsEntry& e = p.t.e[k];
  const int kt = x_cols(e), per = row_blocks(e) * kt, local = (int)blockIdx.x - e.block0, mat = local / per, at = local - mat * per;
  const int rb = at / kt, cb = at - rb * kt, tid = threadIdx.x;
  // the norm, from the matrix's partial sums in fixed order
  const int chunks = chunks_of(e);
  double s = 0.0;
  for (int i = tid; i < chunks; i += 256) s += __ldcg(p.sums + e.chunk0 + (long)mat * chunks + i);
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((tid & 31) == 0) sums[tid >> 5] = s;
  // U of these rows and columns; a tall matrix's rows are X's columns
  const size_t base = (size_t)mat * e.n * e.m;
  const bool tall = e.rows > e.cols;
#pragma unroll 8
  for (int i = tid; i < NS_ROWS * NS_COLS; i += 256) {
    const int r = tall ? i % NS_ROWS : i / NS_COLS, c = tall ? i / NS_ROWS : i % NS_COLS;
    const long row = (long)rb * NS_ROWS + r, col = (long)cb * NS_COLS + c;
    float u = 0.f;
    if (row < e.n && col < e.m) {
      const size_t j = base + (tall ? (size_t)col * e.n + row : (size_t)row * e.m + col);
      u = load_as_float(e.g, e.g_dtype, j);
      if (p.muon) u = update_of(u, __ldcg(e.mom + j), p.momentum, p.nesterov);
    }
    tile[r][c] = u;
  }
  __syncthreads();
  s = sums[0];
  for (int w = 1; w < 8; ++w) s += sums[w];
  // 2^13 / norm as a float in [0.5, 1) and a power of two that is applied in halves: neither the factor nor a product leaves the floats' range
  const double norm = sqrt(s);
  int ex = 0;
  const float f = (float)frexp((double)NS_SCALE / (norm < p.eps ? p.eps : norm), &ex);
  const int e1 = min(126, max(-126, ex / 2)), e2 = min(126, max(-126, ex - e1));
  const float s1 = __int_as_float((e1 + 127) << 23), s2 = __int_as_float((e2 + 127) << 23);
  char* out = p.blocks + ((size_t)e.x0 + (size_t)mat * per + at) * NS_BLOCK;
  for (int i = tid; i < NS_ROWS * 8; i += 256) {
    const int r = i >> 3, q = i & 7;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = tile[r][q * 8 + j] * s1 * f * s2;
    uint4 hi, lo;
    parts8(v, hi, lo);
    *reinterpret_cast<uint4*>(out + piece_at(r, q)) = hi;
    *reinterpret_cast<uint4*>(out + NS_PART + piece_at(r, q)) = lo;
  }
}

// ---- products

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr, uint32_t rank) {
  float4 v;
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr), "r"(rank) : "memory");
  return v;
}

// A unit of work: tile (i, j) of matrix `mat` of an entry, and the stages (64 terms each) that its sums have.
struct NsUnit { const NsEntry* e; int mat, i, j, stages; };
template <int MODE>
__device__ __forceinline__ NsUnit ns_unit(const NsArgs& p, int u, int& k) {
  constexpr bool SYM = MODE == NS_GRAM || MODE == NS_SQUARE;
  while (k + 1 < p.t.entries && u >= (SYM ? p.t.e[k + 1].sym0 : p.t.e[k + 1].prod0)) ++k;
  NsUnit w;
  w.e = &p.t.e[k];
  const int nt = row_blocks(*w.e);
  if (SYM) {
    const int per = nt * (nt + 1) / 2, local = u - w.e->sym0;
    w.mat = local / per;
    const int t = local - w.mat * per;
    int i = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while (i * (i + 1) / 2 > t) --i;
    while ((i + 1) * (i + 2) / 2 <= t) ++i;
    w.i = i;
    w.j = t - i * (i + 1) / 2;
    w.stages = MODE == NS_GRAM ? x_cols(*w.e) : a_cols(*w.e);
  } else {
    const int per_row = (x_cols(*w.e) + 1) / 2, per = nt * per_row, local = u - w.e->prod0;
    w.mat = local / per;
    const int t = local - w.mat * per;
    w.j = t / nt;                                    // (neighbouring units read the same columns of X)
    w.i = t - w.j * nt;
    w.stages = a_cols(*w.e);
  }
  return w;
}

// Eight neighbouring sums of a row of a tile, columns 8 * q8 on.
template <int MODE>
__device__ __forceinline__ void ns_emit(const NsArgs& p, const NsUnit& w, int row, int q8, float (&v)[8]) {
  const NsEntry& e = *w.e;
  const int nt = row_blocks(e), ka = a_cols(e);
  if (MODE == NS_GRAM || MODE == NS_SQUARE) {
    char* to = p.blocks + ((size_t)(MODE == NS_GRAM ? e.a : e.b) + (size_t)w.mat * nt * ka) * NS_BLOCK;
    const int cb = 2 * w.j + (q8 >> 3), r0 = w.i * NS_ROWS + row;
    if (cb < ka) {
      const size_t at = ((size_t)w.i * ka + cb) * NS_BLOCK + piece_at(row, q8 & 7);
      if (MODE == NS_GRAM) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= NS_UNSCALE;
      } else {
        const char* from = p.blocks + ((size_t)e.a + (size_t)w.mat * nt * ka) * NS_BLOCK + at;
        const uint4 hi = __ldcg(reinterpret_cast<const uint4*>(from)), lo = __ldcg(reinterpret_cast<const uint4*>(from + NS_PART));
        const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&h[k])), b = __half22float2(*reinterpret_cast<const __half2*>(&l[k]));
          v[2 * k] = fmaf(p.c * NS_UNSCALE, v[2 * k], p.b * (a.x + b.x));
          v[2 * k + 1] = fmaf(p.c * NS_UNSCALE, v[2 * k + 1], p.b * (a.y + b.y));
        }
        const int d = r0 - (w.j * NS_ROWS + q8 * 8);
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k == d && r0 < e.n) v[k] += p.a * NS_SCALE;
      }
      uint4 hi, lo;
      parts8(v, hi, lo);
      *reinterpret_cast<uint4*>(to + at) = hi;
      *reinterpret_cast<uint4*>(to + at + NS_PART) = lo;
      const int mb = 2 * w.i + (row >> 6);
      if (w.i != w.j && mb < ka) {                   // the tile's mirror image: column `row` of it
        char* m = to + ((size_t)w.j * ka + mb) * NS_BLOCK;
        const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t b = piece_at(q8 * 8 + k, (row & 63) >> 3) + (row & 7) * 2;
          *reinterpret_cast<unsigned short*>(m + b) = (unsigned short)(h[k >> 1] >> (16 * (k & 1)));
          *reinterpret_cast<unsigned short*>(m + b + NS_PART) = (unsigned short)(l[k >> 1] >> (16 * (k & 1)));
        }
      }
    }
  } else if (MODE == NS_APPLY) {
    const int kt = x_cols(e), cb = 2 * w.j + (q8 >> 3);
    if (cb >= kt) return;
    char* to = p.blocks + ((size_t)(p.which ? e.x0 : e.x1) + ((size_t)w.mat * nt + w.i) * kt + cb) * NS_BLOCK + piece_at(row, q8 & 7);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] *= NS_UNSCALE;
    uint4 hi, lo;
    parts8(v, hi, lo);
    *reinterpret_cast<uint4*>(to) = hi;
    *reinterpret_cast<uint4*>(to + NS_PART) = lo;
  } else {
    const long r = (long)w.i * NS_ROWS + row, c0 = (long)w.j * NS_ROWS + q8 * 8;
    if (r >= e.n) return;
    const bool tall = e.rows > e.cols;
    const size_t base = (size_t)w.mat * e.n * e.m;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const long c = c0 + k;
      if (c >= e.m) break;
      const size_t at = base + (tall ? (size_t)c * e.n + r : (size_t)r * e.m + c);
      float o = v[k] * (NS_UNSCALE * NS_UNSCALE);
      if (p.muon) o = fmaf(-e.scale, o, p.keep * load_as_float(e.out, e.out_dtype, at));
      store_from_float(e.out, e.out_dtype, at, o);
    }
  }
}

template <int MODE>
__global__ void __launch_bounds__(NS_THREADS, 1) ns_product_kernel(const __grid_constant__ NsArgs p) {
  constexpr bool SYM = MODE == NS_GRAM || MODE == NS_SQUARE;
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t full[NS_STAGES], empty[NS_STAGES], acc_full[NS_SETS], acc_empty[NS_SETS];
  __shared__ uint32_t tmem_slot;
  __shared__ int go;
  const uint32_t smem = (smem_u32(raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NS_STAGES; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < NS_SETS; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], NS_ADDERS); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc_then_trigger(&tmem_slot, 512);
  pdl_wait();
  if (threadIdx.x == 0) {
    go = (*reinterpret_cast<volatile unsigned*>(p.status) != p.tag) ? 1 : 0;
    if (blockIdx.x == 0) reinterpret_cast<volatile unsigned*>(p.status)[1] = p.tag;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&tmem_slot);
  const int rank = p.cs > 1 ? (int)cluster_rank() : 0;
  const int units = SYM ? p.t.syms : p.t.prods, u0 = (int)blockIdx.x / p.cs, step = (int)gridDim.x / p.cs;

  if (go && warp == 0) {
    if (lane == 0) {
      asm volatile("fence.proxy.async;" ::: "memory");       // (the kernels before wrote the blocks by ordinary stores)
      uint32_t slot = 0, lap = 0, issued = 0;
      int k = 0;
      bool ok = true;
      for (int u = u0; u < units && ok; u += step) {
        const NsUnit w = ns_unit<MODE>(p, u, k);
        const NsEntry& e = *w.e;
        const int nt = row_blocks(e), ka = a_cols(e), kt = x_cols(e);
        const uint32_t xb = p.which ? e.x1 : e.x0;
        const char *A, *B;
        uint32_t b_bytes = NS_OPERAND;
        const bool same = SYM && w.i == w.j;
        int halves = 2;
        if (SYM) {
          const int kk = MODE == NS_GRAM ? kt : ka;
          const char* top = p.blocks + ((size_t)(MODE == NS_GRAM ? xb : e.a) + (size_t)w.mat * nt * kk) * NS_BLOCK;
          A = top + (size_t)w.i * kk * NS_BLOCK;
          B = top + (size_t)w.j * kk * NS_BLOCK;
          if (same) b_bytes = 0;
        } else {
          A = p.blocks + ((size_t)e.b + ((size_t)w.mat * nt + w.i) * ka) * NS_BLOCK;
          B = p.blocks + ((size_t)xb + (size_t)w.mat * nt * kt + 2 * w.j) * NS_BLOCK;
          halves = min(2, kt - 2 * w.j);
          b_bytes = (uint32_t)halves * (NS_OPERAND / 2);
        }
        const int s0 = w.stages * rank / p.cs, s1 = w.stages * (rank + 1) / p.cs;
        for (int s = s0; s < s1; ++s) {
          if (issued >= NS_STAGES && !mbar_wait(&empty[slot], lap ^ 1u, p.status, p.tag)) { ok = false; break; }
          const uint32_t to = smem + slot * NS_STAGE;
          mbar_arrive_expect_tx(&full[slot], NS_OPERAND + b_bytes);
          bulk_load(to, A + (size_t)s * NS_BLOCK, NS_OPERAND, &full[slot]);
          if (SYM) {
            if (!same) bulk_load(to + NS_OPERAND, B + (size_t)s * NS_BLOCK, NS_OPERAND, &full[slot]);
          } else {
            // 64 rows of X: the upper or the lower half of a block's rows, in both column blocks
            const char* from = B + (size_t)(s >> 1) * kt * NS_BLOCK + (s & 1) * (NS_PART / 2);
            for (int h = 0; h < halves; ++h) {
              bulk_load(to + NS_OPERAND + h * (NS_PART / 2), from + h * NS_BLOCK, NS_PART / 2, &full[slot]);
              bulk_load(to + NS_OPERAND + NS_PART + h * (NS_PART / 2), from + h * NS_BLOCK + NS_PART, NS_PART / 2, &full[slot]);
            }
          }
          ++issued;
          if (++slot == NS_STAGES) { slot = 0; lap ^= 1u; }
        }
      }
      // Behind an error: no copy is under way when the block ends.
      if (!ok)
        for (uint32_t i = 0; i < NS_STAGES && i < issued; ++i) {
          if (slot == 0) { slot = NS_STAGES; lap ^= 1u; }
          --slot;
          mbar_wait(&full[slot], lap, p.status, p.tag);
        }
    }
    __syncwarp();
  } else if (go && warp == 1) {
    uint32_t slot = 0, lap = 0, set = 0, set_lap = 0, used = 0;
    int k = 0;
    bool ok = true;
    // Shared-memory descriptors: rows along the result (groups of eight 1024 bytes apart, 32 bytes a step of 16 terms), or along the sum (2048
    // bytes a step, column blocks 8 KB apart).
    constexpr uint32_t HI = (1024u >> 4) | (1u << 14) | (2u << 29);
    constexpr uint32_t A_LO = (16u >> 4) << 16, B_LO = ((SYM ? 16u : NS_PART / 2) >> 4) << 16;
    constexpr uint32_t A_STEP = 32u >> 4, B_STEP = (SYM ? 32u : 2048u) >> 4;
    constexpr uint32_t IDESC = (1u << 4) | (SYM ? 0u : (1u << 16)) | ((uint32_t)(TILE_M >> 4) << 24);
    for (int u = u0; u < units && ok; u += step) {
      const NsUnit w = ns_unit<MODE>(p, u, k);
      const bool same = SYM && w.i == w.j;
      const int halves = SYM ? 2 : min(2, x_cols(*w.e) - 2 * w.j);
      const uint32_t idesc = IDESC | ((uint32_t)(halves * 64 >> 3) << 17);
      const int s0 = w.stages * rank / p.cs, s1 = w.stages * (rank + 1) / p.cs;
      for (int s = s0; s < s1; ++s) {
        if (!mbar_wait_warp(&full[slot], lap, p.status, p.tag)) { ok = false; break; }
        if (used >= NS_SETS && !mbar_wait_warp(&acc_empty[set], set_lap ^ 1u, p.status, p.tag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t at = (smem + slot * NS_STAGE) & 0x3FFFFu;      // (in a cluster an address has the CTA's rank above these bits)
        const uint32_t a = A_LO | (at >> 4), b = B_LO | ((at + (same ? 0u : NS_OPERAND)) >> 4), d = tmem + set * 128;
        constexpr uint32_t L = NS_PART >> 4;
#pragma unroll
        for (int t = 0; t < 4; ++t) umma_warp(d, a + L + t * A_STEP, HI, b + t * B_STEP, HI, idesc, t > 0);
#pragma unroll
        for (int t = 0; t < 4; ++t) umma_warp(d, a + t * A_STEP, HI, b + L + t * B_STEP, HI, idesc, 1u);
#pragma unroll
        for (int t = 0; t < 4; ++t) umma_warp(d, a + t * A_STEP, HI, b + t * B_STEP, HI, idesc, 1u);
        umma_commit_warp(&empty[slot]);
        umma_commit_warp(&acc_full[set]);
        ++used;
        if (++slot == NS_STAGES) { slot = 0; lap ^= 1u; }
        if (++set == NS_SETS) { set = 0; set_lap ^= 1u; }
      }
    }
    // Behind an error: no MMA is under way when its tensor memory is given back.
    if (!ok)
      for (uint32_t i = 0; i < NS_SETS && i < used; ++i) {
        if (set == 0) { set = NS_SETS; set_lap ^= 1u; }
        --set;
        mbar_wait_warp(&acc_full[set], set_lap, p.status, p.tag);
      }
  } else if (go) {
    const int quadrant = warp & 3, half = (warp - 2) >> 2, row = quadrant * 32 + lane;
    uint32_t set = 0, set_lap = 0;
    int k = 0;
    bool ok = true;
    for (int u = u0; u < units && ok; u += step) {
      const NsUnit w = ns_unit<MODE>(p, u, k);
      float sum[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) sum[i] = 0.f;
      const int s0 = w.stages * rank / p.cs, s1 = w.stages * (rank + 1) / p.cs;
      for (int s = s0; s < s1; ++s) {
        if (!mbar_wait_warp(&acc_full[set], set_lap, p.status, p.tag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t from = tmem + set * 128 + half * 64 + ((uint32_t)(quadrant * 32) << 16);
        if (SYM || half == 0 || 2 * w.j + 1 < x_cols(*w.e)) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t x[16], y[16];
            tmem_ld16_issue(from + q * 32, x);
            tmem_ld16_issue(from + q * 32 + 16, y);
            tmem_ld_wait(x); tmem_ld_wait(y);
#pragma unroll
            for (int i = 0; i < 16; ++i) { sum[q * 32 + i] += __uint_as_float(x[i]); sum[q * 32 + 16 + i] += __uint_as_float(y[i]); }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&acc_empty[set]);
        if (++set == NS_SETS) { set = 0; set_lap ^= 1u; }
      }
      if (!ok) break;
      if (p.cs == 1) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = sum[q * 8 + i];
          ns_emit<MODE>(p, w, row, half * 8 + q, v);
        }
      } else {
        // (one unit a cluster: every stage of this CTA has been multiplied, and the ring's memory is free)
#pragma unroll
        for (int q = 0; q < 16; ++q)
          asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(smem + (uint32_t)(((half * 16 + q) * 128 + row) * 16)), "f"(sum[4 * q]), "f"(sum[4 * q + 1]),
                       "f"(sum[4 * q + 2]), "f"(sum[4 * q + 3]) : "memory");
      }
    }
  }
  if (p.cs > 1) {
    __syncwarp();
    cluster_sync();
    if (go && warp >= 2 && u0 < units) {
      int k = 0;
      const NsUnit w = ns_unit<MODE>(p, u0, k);
      const int t = threadIdx.x - 64, row = t & 127, per = 16 / p.cs;      // this CTA's groups of eight columns
      for (int g = t >> 7; g < per; g += 2) {
        const int q8 = rank * per + g;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
        for (int c = 0; c < p.cs; ++c) {
          const float4 x = ld_cluster_f4(smem + (uint32_t)((2 * q8 * 128 + row) * 16), (uint32_t)c);
          const float4 y = ld_cluster_f4(smem + (uint32_t)(((2 * q8 + 1) * 128 + row) * 16), (uint32_t)c);
          v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w; v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
        }
        ns_emit<MODE>(p, w, row, q8, v);
      }
    }
    __syncwarp();
    cluster_sync();                                  // (no CTA ends while its sums are read)
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, 512);
}

template <int MODE>
cudaError_t launch_product(NsArgs& p, cudaStream_t st) {
  constexpr bool SYM = MODE == NS_GRAM || MODE == NS_SQUARE;
  constexpr size_t smem = NS_STAGES * NS_STAGE + 1024;
  const int units = SYM ? p.t.syms : p.t.prods;
  // A cluster's CTAs have a stage each at least where the longest sum has that many.
  int stages = 1;
  for (int k = 0; k < p.t.entries; ++k) stages = std::max(stages, MODE == NS_GRAM ? x_cols(p.t.e[k]) : a_cols(p.t.e[k]));
  p.cs = 1;
  while (p.cs < 8 && units * p.cs * 2 <= NS_SMS && p.cs * 2 <= stages) p.cs *= 2;
  cudaError_t e = cudaFuncSetAttribute(ns_product_kernel<MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.cs > 1 ? units * p.cs : std::min(units, NS_SMS)));
  cfg.blockDim = dim3(NS_THREADS);
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
  return cudaLaunchKernelEx(&cfg, ns_product_kernel<MODE>, p);
}

size_t sums_bytes(const NsTable& t) { return ((size_t)t.chunks * sizeof(double) + 1023) / 1024 * 1024; }

}  // namespace

size_t ns_blocks_of(long rows, long cols) {
  const long n = std::min(rows, cols), m = std::max(rows, cols);
  const size_t nt = (size_t)((n + NS_ROWS - 1) / NS_ROWS);
  return 2 * nt * (size_t)((m + NS_COLS - 1) / NS_COLS) + 2 * nt * (size_t)((n + NS_COLS - 1) / NS_COLS);
}

void ns_add(NsTable* t, NsEntry e) {
  e.n = std::min(e.rows, e.cols);
  e.m = std::max(e.rows, e.cols);
  const int nt = row_blocks(e);
  const uint32_t x = (uint32_t)e.count * nt * x_cols(e), a = (uint32_t)e.count * nt * a_cols(e);
  e.x0 = t->ws_blocks; e.x1 = e.x0 + x; e.a = e.x1 + x; e.b = e.a + a;
  t->ws_blocks = e.b + a;
  e.chunk0 = t->chunks; e.block0 = t->blocks; e.sym0 = t->syms; e.prod0 = t->prods;
  t->chunks += e.count * chunks_of(e);
  t->blocks += (int)x;
  t->syms += e.count * (nt * (nt + 1) / 2);
  t->prods += e.count * nt * ((x_cols(e) + 1) / 2);
  t->e[t->entries++] = e;
}

size_t ns_bytes(const NsTable& t) { return sums_bytes(t) + t.ws_blocks * NS_BLOCK; }

cudaError_t launch_newton_schulz(const NsTable& t, const NsOptions& o, void* ws, unsigned tag, cudaStream_t st, int* launches) {
  NsArgs p = {};
  p.t = t;
  p.status = static_cast<unsigned*>(ws);
  p.tag = tag;
  p.sums = reinterpret_cast<double*>(static_cast<char*>(ws) + NS_HEADER);
  p.blocks = static_cast<char*>(ws) + NS_HEADER + sums_bytes(t);
  p.a = o.a; p.b = o.b; p.c = o.c; p.eps = o.eps; p.momentum = o.momentum; p.keep = o.keep; p.muon = o.muon; p.nesterov = o.nesterov;
  cudaError_t e = launch_pdl(ns_squares_kernel, dim3((unsigned)t.chunks), dim3(256), 0, st, p);
  if (e != cudaSuccess) return e;
  ++*launches;
  e = launch_pdl(ns_blocks_kernel, dim3((unsigned)t.blocks), dim3(256), 0, st, p);
  if (e != cudaSuccess) return e;
  ++*launches;
  for (int s = 0; s < o.steps; ++s) {
    p.which = s & 1;
    if ((e = launch_product<NS_GRAM>(p, st)) != cudaSuccess) return e;
    ++*launches;
    if ((e = launch_product<NS_SQUARE>(p, st)) != cudaSuccess) return e;
    ++*launches;
    if ((e = s + 1 < o.steps ? launch_product<NS_APPLY>(p, st) : launch_product<NS_LAST>(p, st)) != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

}  // namespace xconv
