// Host-side launchers of the first-order operators (internal to the library): layer
// normalisation, and Newton-Schulz orthogonalisation with the Muon update.
#pragma once

#include <cstdint>

#include <cuda.h>
#include <cuda_runtime.h>

namespace zo {

// ---- layer normalisation (zo_layernorm.cu) ------------------------------------------
struct LayerNormArgs {
  // forward: x (+ r) -> h = rnd(x + r) (only with r), y, mean, rstd (either may be null)
  // backward: dy, x (= h), mean, rstd (+ dr) -> dx, dweight, dbias
  const void *x, *r, *dy;
  const void *weight, *bias;      // null: 1 and 0
  void *y, *h, *dx;
  float *mean, *rstd;
  void *dweight, *dbias;          // null: not wanted
  float* partial;                 // backward: layernorm_partial_rows() x 2 x cols sums
  int64_t rows, cols;
  int64_t ldx, ldr, lddy, ldy, ldh, lddx;
  int32_t dtype, wdtype;          // of x, r, y, h, dy, dx, dr; of weight, bias, dweight, dbias
  float eps;
};

cudaError_t launch_layernorm_forward(const LayerNormArgs& a, cudaStream_t s);
// CTAs of the backward pass: rows of the partial sums of dweight and of dbias
int64_t layernorm_partial_rows(int64_t rows, int64_t cols, int32_t sms);
cudaError_t launch_layernorm_backward(const LayerNormArgs& a, int32_t sms, cudaStream_t s);

}  // namespace zo
