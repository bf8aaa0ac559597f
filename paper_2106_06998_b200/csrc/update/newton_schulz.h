// Orthogonalisation of matrices by Newton-Schulz products, and the step of weights by orthogonalised momenta (newton_schulz.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../../include/xconv.h"

namespace xconv {

// Matrices of one shape that lie behind one another, as the kernels see them: n = min, m = max of rows and columns.
struct NsEntry {
  const void* g;                     // gradients
  float* mom;                        // momenta, or null
  void* out;                         // what the last product goes to: the orthogonalised matrices, or the weights
  uint32_t x0, x1, a, b;             // first blocks of X (two buffers), A and B in the scratch memory
  int n, m, rows, cols, count;
  int chunk0, block0, sym0, prod0;   // first unit of the entry in each kernel
  int g_dtype, out_dtype;
  float scale;                       // of the orthogonalised matrix in the update
};
constexpr int NS_MOST = 64;          // entries of a launch

struct NsTable {
  NsEntry e[NS_MOST];
  int entries, chunks, blocks, syms, prods;
  uint32_t ws_blocks;                // blocks of 32 KB
};

struct NsOptions {
  float a, b, c;                     // a step: X <- (a I + b A + c A A) X, A = X X^T
  int steps;
  double eps;
  bool muon, nesterov;
  float momentum, keep;              // weights <- keep * weights - scale * O
};

constexpr int NS_ROWS = 128, NS_COLS = 64;                          // of a block
constexpr size_t NS_BLOCK = (size_t)NS_ROWS * NS_COLS * 2 * 2;      // two float16 parts of every value
constexpr int NS_CHUNK = 8192;                                      // values of a matrix that a block of threads squares

// Blocks of scratch memory that a matrix needs; `count` matrices of an entry added to a table that has room for it (its pointers, shape and types given).
size_t ns_blocks_of(long rows, long cols);
void ns_add(NsTable* t, NsEntry e);
// Bytes behind the scratch memory's header that a table needs: partial sums, then blocks.
size_t ns_bytes(const NsTable& t);
// Enqueues everything; *launches counts.  ws: the header (256 bytes) and ns_bytes(t).
cudaError_t launch_newton_schulz(const NsTable& t, const NsOptions& o, void* ws, unsigned tag, cudaStream_t st, int* launches);

}  // namespace xconv
