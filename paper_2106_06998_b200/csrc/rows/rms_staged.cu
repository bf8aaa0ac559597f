// RMS norm and its gradients of dense rows that do not begin on 16-byte boundaries (formulas: rms_norm.cu, rms_backward.cu).
//
// Too few warps bound it: 16 an SM or fewer, which fill 62 to 64 % of the issue slots (a row's pairs take the registers of more).  Measured (B200; replayed from a graph): 47250 x 97 float16 with
// residual and dropout 17 to 18 us (floor of bytes 5.6), by octets cut out in registers 23; gradients
// with dh 21.5 us (floor 7.0), 31; 164948 x 97 bf16 without dropout 39 us (floor 19.5), 59, with it 54, 67; 8192 x 4097 bf16 100 us, gradients 124 (floors 40.9).  Masks drawn into shared memory by all threads before a run's
// rows: 58 instead of 53.
#include "eight_bits.cuh"
#include "rms.h"
#include "staged.cuh"

namespace xconv {

namespace {

struct StagedArgs {
  Staged s;
  const void *in[3];               // forward: x, residual; backward: h, dy, dh
  void *out[2];                    // over the first and the second of them: y, h; dx, dr
  const void* weight;
  int weight_f32;
  int q;                           // forward: y in 8 bits, a scale a row
  float* scales;
  float* rstd;                     // (read by the backward pass)
  float* part;
  float eps, inv_c;
};

template <typename T, int V, bool BACK>
__global__ void __launch_bounds__(512, V <= 4 ? 2 : 1) rms_staged_kernel(const StagedArgs a) {
  extern __shared__ uint4 ring[];
  __shared__ float sums[2][32], most[2][32];
  constexpr int PER = 16 / sizeof(T);
  char* const base = reinterpret_cast<char*>(ring);
  const Staged& s = a.s;
  const int group = s.group, lane = group <= 32 ? threadIdx.x & (group - 1) : threadIdx.x, own = group <= 32 ? threadIdx.x / group : 0;
  const int bytes = s.slots * s.slot;                          // of a stage
  const bool drops = s.drop.how != DROP_NONE;
  pdl_wait();
  const uint2 key = s.drop.how == DROP_DEVICE ? s.drop.key<DROP_DEVICE>() : s.drop.key<DROP_HOST>();
  const auto fetch = [&](long run, int stage) {
    if (run < s.runs) {
      const Run r = Run::of<PER>(s, run);
#pragma unroll
      for (int i = 0; i < (BACK ? 3 : 2); ++i)
        if (a.in[i]) run_in<T>(s, r, base + stage * bytes + i * s.slot, static_cast<const T*>(a.in[i]));
    }
    copies_commit();
  };
  for (int i = 0; i < s.stages - 1; ++i) fetch(blockIdx.x + (long)i * gridDim.x, i);
  const Pairs<T, V> pairs(lane, group, s.C, s.C & 1 ? (int)((long)blockIdx.x * s.run + own) & 1 : 0);
  float w[V][2], dw[V][2];
  if (sizeof(T) == 4 || a.weight_f32) pairs.template weights<float>(a.weight, w);
  else pairs.template weights<T>(a.weight, w);
#pragma unroll
  for (int v = 0; v < V; ++v) dw[v][0] = dw[v][1] = 0.f;
  int stage = 0, turn = 0;
  PairMask<V> mask;
  for (long run = blockIdx.x; run < s.runs; run += gridDim.x) {
    const Run here = Run::of<PER>(s, run);
    if (s.stages == 3) copies_wait<1>();
    else copies_wait<0>();
    __syncthreads();
    // (the stage before this one was written out before the barrier)
    fetch(run + (long)(s.stages - 1) * gridDim.x, stage == 0 ? s.stages - 1 : stage - 1);
    T* const at = reinterpret_cast<T*>(base + stage * bytes) + here.shift;
    const int apart = s.slot / (int)sizeof(T);
    unsigned char* const codes = reinterpret_cast<unsigned char*>(base + s.stages * bytes);
    const Run eight = Run::of<16>(s, run);                     // (of a tensor of bytes)
    for (int r = own; r < s.run; r += s.groups, turn ^= 1) {
      const bool in = r < here.rows;                           // (of a row that is not there memory holds whatever: nothing of it is kept)
      const long row = run * s.run + r;
      T* const x = at + r * s.C;
      if (drops) mask.draw(s, key, lane, pairs.odd, s.drop.per((uint32_t)min(row, s.rows - 1)));
      if constexpr (!BACK) {
        float h[V][2], f[V][2], ss = 0.f;
        pairs.read(x, h);
        if (a.in[1]) pairs.read(x + apart, f);
        else
#pragma unroll
          for (int v = 0; v < V; ++v) f[v][0] = f[v][1] = 0.f;
        if (drops) {
          bool gone[V][2];
          mask.gone(s, lane, gone);
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int k = 0; k < 2; ++k) h[v][k] = gone[v][k] ? f[v][k] : fmaf(h[v][k], s.drop.scale, f[v][k]);
        } else {
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int k = 0; k < 2; ++k) h[v][k] += f[v][k];
        }
        if (a.out[1] && in) pairs.write(x + apart, h);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int k = 0; k < 2; ++k) ss = fmaf(h[v][k], h[v][k], ss);
        ss = row_sum(ss, group, sums[turn]);
        const float rstd = rsqrtf(fmaf(ss, a.inv_c, a.eps));
        if (in && lane == 0 && a.rstd) a.rstd[row] = rstd;
        const Root root = root_of(rstd);
        const float by = a.q ? root.power : rstd;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int k = 0; k < 2; ++k) h[v][k] *= by * w[v][k];
        if (!a.q) {
          if (in) pairs.write(x, h);
        } else {
          float m = 0.f;
#pragma unroll
          for (int v = 0; v < V; ++v) m = most_of(m, most_of(fabsf(h[v][0]), fabsf(h[v][1])));
          const Scale f = q_scale(row_most(m, group, most[turn]), root, a.q);
          if (in && lane == 0) a.scales[row] = f.scale;
          unsigned char* const to = codes + eight.shift + r * s.C + pairs.column;
          if (in)
#pragma unroll
            for (int v = 0; v < V; ++v) {
              const float2 t = q_of(h[v][0], h[v][1], f);
              const uint32_t b = a.q == XCONV_Q_E4M3 ? e4m3x2(t) : int8x2(t);
              if (pairs.has(v, 0)) to[2 * v * group] = (unsigned char)b;
              if (pairs.has(v, 1)) to[2 * v * group + 1] = (unsigned char)(b >> 8);
            }
        }
      } else {
        float xh[V][2], g[V][2], t = 0.f;
        const float rstd = in ? a.rstd[row] : 0.f;
        pairs.read(x, xh);
        pairs.read(x + apart, g);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            xh[v][k] *= rstd;
            if (in) dw[v][k] = fmaf(g[v][k], xh[v][k], dw[v][k]);
            g[v][k] *= w[v][k];
            t = fmaf(g[v][k], xh[v][k], t);
          }
        const float mean = row_sum(t, group, sums[turn]) * a.inv_c;
        if (a.in[2]) {
          float d[V][2];
          pairs.read(x + 2 * apart, d);
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int k = 0; k < 2; ++k) g[v][k] = fmaf(rstd, fmaf(-xh[v][k], mean, g[v][k]), d[v][k]);
        } else {
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int k = 0; k < 2; ++k) g[v][k] = rstd * fmaf(-xh[v][k], mean, g[v][k]);
        }
        if (a.out[1] && in) pairs.write(x + apart, g);
        if (a.out[0]) {
          if (drops) {
            bool gone[V][2];
            mask.gone(s, lane, gone);
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
              for (int k = 0; k < 2; ++k) g[v][k] = gone[v][k] ? 0.f : g[v][k] * s.drop.scale;
          }
          if (in) pairs.write(x, g);
        }
      }
    }
    __syncthreads();
    if (!BACK && a.q) run_out<unsigned char>(eight, reinterpret_cast<const char*>(codes), static_cast<unsigned char*>(a.out[0]));
#pragma unroll
    for (int i = !BACK && a.q ? 1 : 0; i < 2; ++i)
      if (a.out[i]) run_out<T>(here, base + stage * bytes + i * s.slot, static_cast<T*>(a.out[i]));
    stage = stage == s.stages - 1 ? 0 : stage + 1;
  }
  if (!BACK || !a.part) return;
  pdl_trigger();
  // The block's sums of dw: every group's side by side in shared memory, then column by column in order.
  copies_wait<0>();
  __syncthreads();
  float* const cols = reinterpret_cast<float*>(ring);
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (pairs.has(v, k)) cols[(size_t)own * s.C + pairs.column + 2 * v * group + k] = dw[v][k];
  __syncthreads();
  for (int c = threadIdx.x; c < s.C; c += blockDim.x) {
    float t = cols[c];
    for (int i = 1; i < s.groups; ++i) t += cols[(size_t)i * s.C + c];
    a.part[(size_t)blockIdx.x * s.C + c] = t;
  }
}

template <bool BACK>
cudaError_t launch(const xconv_rows_desc* d, const StagedPlan& p, const StagedArgs& a, cudaStream_t st) {
  return with_type(d->dtype, [&](auto t) {
    using T = decltype(t);
    void (*kernel)(const StagedArgs) = nullptr;
#define XC_STAGED(N) if (p.V == N) kernel = rms_staged_kernel<T, N, BACK>;
    XC_STAGED(1) XC_STAGED(2) XC_STAGED(3) XC_STAGED(4) XC_STAGED(5) XC_STAGED(6) XC_STAGED(7) XC_STAGED(8)
#undef XC_STAGED
    if (!kernel) return cudaErrorInvalidValue;
    if (p.smem > 40 * 1024) {
      // (the same for every size, so that no other thread finds it lowered)
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, STAGED_SMEM);
      if (e != cudaSuccess) return e;
    }
    return launch_pdl(kernel, dim3((unsigned)p.blocks), dim3(p.threads), p.smem, st, a);
  });
}

// (rows of whole pieces never come here, whatever their pointers: the scratch memory of a call is known by its sizes)
bool is_odd(const xconv_rows_desc* d) { return d->C % (d->dtype == XCONV_F32 ? 4 : 8) != 0; }
bool is_dense(const xconv_rows_desc* d, const void* p, int64_t stride) { return !p || (stride == d->C && at(p, 16)); }

}  // namespace

bool rms_staged_forward(const xconv_rows_desc* d, const void* X, const void* residual, const void* weight, void* H, void* Y, float* scales, float* rstd, cudaStream_t st, cudaError_t* e) {
  if (d->q_type && d->q_group > 0 && d->q_group < d->C) return false;
  if (!is_odd(d) || !is_dense(d, X, d->x_stride) || !is_dense(d, residual, d->r_stride) || !is_dense(d, H, d->h_stride) || !is_dense(d, Y, d->y_stride)) return false;
  StagedArgs a = {};
  a.s.drop = drop_of(d);
  const StagedPlan p = staged_plan(d, residual || H ? 2 : 1, false, d->q_type != 0, &a.s);
  if (!p.threads) return false;
  a.in[0] = X; a.in[1] = residual; a.out[0] = Y; a.out[1] = H; a.q = d->q_type; a.scales = scales;
  a.weight = weight; a.weight_f32 = d->param_dtype == XCONV_F32; a.rstd = rstd; a.eps = d->eps; a.inv_c = 1.f / (float)d->C;
  *e = launch<false>(d, p, a, st);
  return true;
}

long rms_staged_backward_parts(const xconv_rows_desc* d) {
  Staged s = {};
  long most = 0;
  if (!is_odd(d)) return 0;
  // (fewer tensors need less memory, so that more blocks fit)
  for (int slots = 2; slots <= 3; ++slots) {
    const StagedPlan p = staged_plan(d, slots, true, false, &s);
    if (p.threads) most = std::max(most, p.blocks);
  }
  return most;
}

bool rms_staged_backward(const xconv_rows_desc* d, const void* dY, const void* H, const float* rstd, const void* weight, const void* dH, void* dX, void* dR, float* part, long* parts,
                         cudaStream_t st, cudaError_t* e) {
  if (!is_odd(d) || !is_dense(d, dY, d->y_stride) || !is_dense(d, H, d->h_stride) || !is_dense(d, dH, d->dh_stride) || !is_dense(d, dX, d->x_stride) || !is_dense(d, dR, d->r_stride)) return false;
  StagedArgs a = {};
  if (dX) a.s.drop = drop_of(d);
  const StagedPlan p = staged_plan(d, dH ? 3 : 2, true, false, &a.s);
  if (!p.threads) return false;
  a.in[0] = H; a.in[1] = dY; a.in[2] = dH; a.out[0] = dX; a.out[1] = dR;
  a.weight = weight; a.weight_f32 = d->param_dtype == XCONV_F32; a.rstd = const_cast<float*>(rstd); a.part = part; a.inv_c = 1.f / (float)d->C;
  *parts = p.blocks;
  *e = launch<true>(d, p, a, st);
  return true;
}

}  // namespace xconv
