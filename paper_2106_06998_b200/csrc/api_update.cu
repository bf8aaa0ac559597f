// C ABI of the weights' update: argument checks, planning and dispatch (kernels: update/newton_schulz.cu).
#include "../../include/xconv.h"

#include <algorithm>
#include <cmath>
#include <vector>

#include "api_state.h"
#include "update/newton_schulz.h"

namespace xconv {

namespace {

const size_t UPDATE_HEADER = 256;
// Matrices that go through the launches together hold at most this much scratch memory (a larger matrix goes alone): beyond it every launch fills the GPU
// many times over, and more matrices a launch save nothing.
const size_t UPDATE_BLOCKS = 65536;              // 2 GB
const size_t UPDATE_MOST = 4u << 20;             // of one matrix: 128 GB

inline size_t size_of(int dtype) { return dtype == XCONV_F32 ? 4 : 2; }
inline bool is_dtype(int d) { return d == XCONV_F32 || d == XCONV_BF16 || d == XCONV_F16; }

// What |x| <= bound becomes under a x + b x^3 + c x^5, and the largest |a + b x^2 + c x^4| there.
void step_bounds(const xconv_update_desc* d, double bound, double* out, double* factor) {
  const double a = d->a, b = d->b, c = d->c;
  double top = 0.0, q = std::fabs(a);
  const auto p = [&](double x) { const double s = x * x; return std::fabs(x * (a + s * (b + s * c))); };
  const auto f = [&](double s) { return std::fabs(a + s * (b + s * c)); };
  top = p(bound);
  q = std::max(q, f(bound * bound));
  if (c != 0.0) {
    const double s = -b / (2.0 * c);
    if (s > 0.0 && s < bound * bound) q = std::max(q, f(s));
    const double disc = 9.0 * b * b - 20.0 * a * c;          // of a + 3 b s + 5 c s^2, whose zeros are where the polynomial turns
    if (disc >= 0.0)
      for (const double sign : {-1.0, 1.0}) {
        const double t = (-3.0 * b + sign * std::sqrt(disc)) / (10.0 * c);
        if (t > 0.0 && t < bound * bound) top = std::max(top, p(std::sqrt(t)));
      }
  } else if (b != 0.0) {
    const double t = -a / (3.0 * b);
    if (t > 0.0 && t < bound * bound) top = std::max(top, p(std::sqrt(t)));
  }
  *out = top;
  *factor = q;
}

// The matrices' operands are held as float16 parts times 2^13: singular values stay below 1.9 from step to step, the factors of a step below 7.5.
xconv_status validate_update(const xconv_update_desc* d) {
  if (!d || d->steps < 1 || d->steps > 64 || !(d->eps >= 0.f) || !std::isfinite(d->a) || !std::isfinite(d->b) || !std::isfinite(d->c)) return XCONV_ERR_INVALID_ARG;
  double bound = 1.0 + 1e-4;
  for (int s = 0; s < d->steps; ++s) {
    double next, factor;
    step_bounds(d, bound, &next, &factor);
    if (!(factor <= 7.5) || !(next <= 1.9)) return XCONV_ERR_UNSUPPORTED;
    next = std::max(next, 0.0) + 1e-4;
    if (std::fabs(next - bound) < 1e-12) break;
    bound = next;
  }
  return XCONV_OK;
}

struct Range { uintptr_t from, to; };

xconv_status validate_items(const xconv_matrices* items, int count, bool muon) {
  if (!items || count <= 0 || count > 65536) return XCONV_ERR_INVALID_ARG;
  for (int k = 0; k < count; ++k) {
    const xconv_matrices& m = items[k];
    if (!m.G || !m.O || (muon && !m.M) || m.rows <= 0 || m.cols <= 0 || m.batch <= 0 || !is_dtype(m.g_dtype) || !is_dtype(m.o_dtype)) return XCONV_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(m.G) % 16 || reinterpret_cast<uintptr_t>(m.O) % 16 || (muon && reinterpret_cast<uintptr_t>(m.M) % 16)) return XCONV_ERR_ALIGNMENT;
    if (m.rows > (1 << 24) || m.cols > (1 << 24) || ns_blocks_of(m.rows, m.cols) > UPDATE_MOST) return XCONV_ERR_UNSUPPORTED;
  }
  // What is written overlaps nothing else: the matrices of a call are worked on at the same time.
  std::vector<Range> written, read;
  const auto range = [](const void* p, const xconv_matrices& m, size_t es) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    return Range{at, at + (size_t)m.rows * m.cols * m.batch * es};
  };
  written.reserve(2 * (size_t)count);
  for (int k = 0; k < count; ++k) {
    written.push_back(range(items[k].O, items[k], size_of(items[k].o_dtype)));
    if (muon) written.push_back(range(items[k].M, items[k], 4));
  }
  std::sort(written.begin(), written.end(), [](const Range& x, const Range& y) { return x.from < y.from; });
  for (size_t i = 1; i < written.size(); ++i)
    if (written[i].from < written[i - 1].to) return XCONV_ERR_INVALID_ARG;
  for (int k = 0; k < count; ++k) {
    const Range r = range(items[k].G, items[k], size_of(items[k].g_dtype));
    const auto at = std::lower_bound(written.begin(), written.end(), r.to, [](const Range& x, uintptr_t v) { return x.from < v; });
    if (at != written.begin() && (at - 1)->to > r.from) return XCONV_ERR_INVALID_ARG;
  }
  return XCONV_OK;
}

double scale_of(const xconv_update_desc* d, const xconv_matrices& m) {
  if (d->adjust == XCONV_ADJUST_RMS) return 0.2 * std::sqrt((double)std::max(m.rows, m.cols));
  return std::sqrt(std::max(1.0, (double)m.rows / (double)m.cols));
}

// f(table) for the tables that the call's matrices go into, in order; stops at the first status that is not XCONV_OK.
template <class F>
xconv_status for_tables(const xconv_update_desc* d, const xconv_matrices* items, int count, bool muon, F&& f) {
  static thread_local NsTable t;
  t = NsTable{};
  // The longest sides first: launches share the longest sums (those of X X^T, at least) between their blocks of threads, and end with the short ones.
  std::vector<int> order((size_t)count);
  for (int k = 0; k < count; ++k) order[k] = k;
  std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return std::max(items[x].rows, items[x].cols) > std::max(items[y].rows, items[y].cols); });
  for (const int k : order) {
    const xconv_matrices& m = items[k];
    const size_t each = ns_blocks_of(m.rows, m.cols), values = (size_t)m.rows * m.cols;
    for (int done = 0; done < m.batch;) {
      size_t room = t.ws_blocks < UPDATE_BLOCKS ? (UPDATE_BLOCKS - t.ws_blocks) / each : 0;
      if (t.entries == NS_MOST || (room == 0 && t.entries > 0)) {
        const xconv_status s = f(t);
        if (s != XCONV_OK) return s;
        t = NsTable{};
        continue;
      }
      NsEntry e = {};
      e.count = (int)std::min<size_t>(std::max<size_t>(room, 1), (size_t)(m.batch - done));
      const size_t at = (size_t)done * values;
      e.g = static_cast<const char*>(m.G) + at * size_of(m.g_dtype);
      e.mom = muon ? m.M + at : nullptr;
      e.out = static_cast<char*>(m.O) + at * size_of(m.o_dtype);
      e.rows = m.rows; e.cols = m.cols; e.g_dtype = m.g_dtype; e.out_dtype = m.o_dtype;
      e.scale = muon ? (float)(d->lr * scale_of(d, m)) : 0.f;
      ns_add(&t, e);
      done += e.count;
    }
  }
  return t.entries ? f(t) : XCONV_OK;
}

xconv_status update(const xconv_update_desc* d, const xconv_matrices* items, int count, bool muon, void* ws, size_t ws_bytes, void* cuda_stream) {
  xconv_status s = validate_update(d);
  if (s != XCONV_OK) return s;
  if (muon && (!std::isfinite(d->lr) || !std::isfinite(d->weight_decay) || !(d->momentum >= 0.f && d->momentum <= 1.f) || (d->nesterov != 0 && d->nesterov != 1) ||
               (d->adjust != XCONV_ADJUST_SPECTRAL && d->adjust != XCONV_ADJUST_RMS)))
    return XCONV_ERR_INVALID_ARG;
  s = validate_items(items, count, muon);
  if (s != XCONV_OK) return s;
  size_t need = 0;
  for_tables(d, items, count, muon, [&](const NsTable& t) { need = std::max(need, ns_bytes(t)); return XCONV_OK; });
  if (!ws || ws_bytes < UPDATE_HEADER + need) return XCONV_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) % 16) return XCONV_ERR_ALIGNMENT;
  NsOptions o = {};
  o.a = d->a; o.b = d->b; o.c = d->c; o.steps = d->steps; o.eps = d->eps; o.muon = muon;
  if (muon) { o.nesterov = d->nesterov != 0; o.momentum = d->momentum; o.keep = (float)(1.0 - (double)d->lr * (double)d->weight_decay); }
  new_call();
  int launches = 0;
  s = for_tables(d, items, count, muon, [&](const NsTable& t) {
    const cudaError_t e = launch_newton_schulz(t, o, ws, call_tag(), static_cast<cudaStream_t>(cuda_stream), &launches);
    if (e == cudaSuccess) return XCONV_OK;
    g_last_cuda_error = (int)e;
    return XCONV_ERR_CUDA;
  });
  g_launches = launches;
  return s;
}

}  // namespace

}  // namespace xconv

using namespace xconv;

extern "C" {

size_t xconv_update_workspace_bytes(const xconv_matrices* items, int count) try {
  if (!items || count <= 0 || count > 65536) return 0;
  for (int k = 0; k < count; ++k)
    if (items[k].rows <= 0 || items[k].cols <= 0 || items[k].batch <= 0 || items[k].rows > (1 << 24) || items[k].cols > (1 << 24) ||
        ns_blocks_of(items[k].rows, items[k].cols) > UPDATE_MOST)
      return 0;
  size_t need = 0;
  for_tables(nullptr, items, count, false, [&](const NsTable& t) { need = std::max(need, ns_bytes(t)); return XCONV_OK; });
  return UPDATE_HEADER + need;
} catch (...) {
  return 0;
}

xconv_status xconv_orthogonalize(const xconv_update_desc* desc, const xconv_matrices* items, int count, void* ws, size_t ws_bytes, void* cuda_stream) try {
  return update(desc, items, count, false, ws, ws_bytes, cuda_stream);
} catch (...) {                                      // (host memory)
  return XCONV_ERR_INVALID_ARG;
}

xconv_status xconv_muon_step(const xconv_update_desc* desc, const xconv_matrices* items, int count, void* ws, size_t ws_bytes, void* cuda_stream) try {
  return update(desc, items, count, true, ws, ws_bytes, cuda_stream);
} catch (...) {
  return XCONV_ERR_INVALID_ARG;
}

}  // extern "C"
