// Host-side launch interface of the layer kernels: 8-bit codes and their products, dropout.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tng.h"

namespace tng {

// Streams of the generator (the low byte of a counter's last word; the site is above it).  0 to 2 belong to the coder,
// the minibatches and the Rosenbrock noise.
constexpr uint32_t kStreamDropout = 3u;
constexpr uint32_t kStreamRounding = 4u;

// Elements of workers x rows x cols, a row's contiguous; ld and pitch in elements.
struct View {
  void* p;
  uint64_t ld, pitch;
};

struct DropArgs {
  uint32_t k0, k1, iter, word;  // key; counter words 2 and 3
  uint32_t threshold;           // ceil(p 2^24) 2^8: an element is kept if its word is no less, which says the same of its 24-bit draw; 0: nothing is drawn
  float scale;                  // 1 / (1 - p)
  int relu;
};

struct Extent {
  uint32_t workers;
  uint64_t rows, cols;
};

// y = residual + keep f(x) scale; residual.p may be null.
hipError_t launch_dropout(tng_type type, const Extent& n, const DropArgs& drop, const View& x, const View& residual,
                          const View& y, hipStream_t s);
// dx = keep f'(x) dy scale; x is read only with relu.
hipError_t launch_dropout_grad(tng_type type, const Extent& n, const DropArgs& drop, const View& x, const View& dy,
                               const View& dx, hipStream_t s);

// Codes of rows, rounded to nearest: scale[worker][row], q as x lies, qt (p may be null) the same codes as [worker][col][row].
hipError_t launch_quantize_rows(tng_type type, const Extent& n, const DropArgs* drop, const View& x, const View& q,
                                float* scale, const View& qt, hipStream_t s);

// Codes of dy for the two products of a backward pass, rounded by draws.  Scratch: quantize_grad_floats() floats.
size_t quantize_grad_floats(const Extent& n);
hipError_t launch_quantize_grad(tng_type type, const Extent& n, const DropArgs& key, const View& dy, const float* col_scale,
                                const float* row_scale, const View& q, float* q_scale, const View& qt, float* qt_scale,
                                float* col_sum, float* scratch, hipStream_t s);

// y[m][t][n] = a_scale[m][t] b_scale[n] sum_k a[m][t][k] b[n][k] + bias[n], times keep f'(x) scale of drop where drop is not null.
struct Product {
  uint32_t workers;
  uint64_t rows, channels, depth;  // rows of a, rows of b, columns of both
  View a, b;                       // b.pitch 0: one b for all workers
  const float *a_scale, *b_scale, *bias;
  uint64_t b_scale_pitch;
  View y;
  tng_type type;
  const DropArgs* drop;
  View x;  // of y's type, read only with relu
  uint64_t rows_of_worker;  // set by launch_product
};
size_t product_scratch_bytes(const Product& p);
hipError_t launch_product(const Product& p, void* scratch, hipStream_t s);
// The same with rows of a that are the codes of x (of y's type), which the kernel makes itself; a and a_scale are not looked at.
bool coded_product_applies(const Product& p, const View& x);
hipError_t launch_coded_product(const Product& p, const View& x, hipStream_t s);

}  // namespace tng
