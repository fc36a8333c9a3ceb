// C ABI of the first-order operators (declared in include/zo.h): layer normalisation.
#include <cmath>

#include "../../include/zo.h"
#include "zo_host.h"
#include "zo_ops.h"

namespace {

using namespace zo::host;

// Set by a layer norm kernel whose wait for its rows has run out; one per device.
__device__ uint32_t g_layernorm_status;

bool known_dtype(int32_t d) { return d == ZO_F32 || d == ZO_BF16; }
int32_t elem_bytes(int32_t d) { return d == ZO_BF16 ? 2 : 4; }

// whether p is aligned to its elements
bool elem_aligned(const void* p, int32_t dtype) {
  return reinterpret_cast<uintptr_t>(p) % elem_bytes(dtype) == 0;
}

constexpr int64_t kMaxExtent = int64_t(1) << 31;

// the current device's status word, or null
uint32_t* status_word() {
  static uint32_t* word[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
  if (word[dev] == nullptr) {
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_layernorm_status) != cudaSuccess) return nullptr;
    word[dev] = static_cast<uint32_t*>(p);
  }
  return word[dev];
}

zo_status check_rows(int64_t rows, int64_t cols, int32_t dtype, int32_t wdtype) {
  if (!known_dtype(dtype) || !known_dtype(wdtype)) return refuse(ZO_ERR_DTYPE, "unknown dtype");
  if (rows < 0 || rows >= kMaxExtent || cols < 1 || cols >= kMaxExtent)
    return refuse(ZO_ERR_SHAPE, "layer norm: need 0 <= rows < 2^31 and 1 <= cols < 2^31");
  return ZO_OK;
}

}  // namespace

extern "C" {

zo_status zo_layernorm_forward(const void* X, int64_t ldx, const void* R, int64_t ldr, int64_t rows,
                               int64_t cols, int32_t dtype, const void* weight, const void* bias,
                               int32_t wdtype, float eps, void* Y, int64_t ldy, void* H,
                               int64_t ldh, float* mean, float* rstd, void* stream) {
  const zo_status st = check_rows(rows, cols, dtype, wdtype);
  if (st != ZO_OK) return st;
  if (!(eps >= 0.0f) || !std::isfinite(eps) || (R == nullptr) != (H == nullptr))
    return refuse(ZO_ERR_INVALID_ARG,
                  "zo_layernorm_forward: need a finite eps >= 0, and H exactly where R is given");
  if (ldx < cols || ldy < cols || (R && (ldr < cols || ldh < cols)))
    return refuse(ZO_ERR_SHAPE, "zo_layernorm_forward: a row stride is smaller than cols");
  if (rows == 0) return ZO_OK;
  if (!X || !Y) return refuse(ZO_ERR_INVALID_ARG, "zo_layernorm_forward: null X or Y");
  if (!elem_aligned(X, dtype) || !elem_aligned(Y, dtype) || !elem_aligned(R, dtype) ||
      !elem_aligned(H, dtype) || !elem_aligned(weight, wdtype) || !elem_aligned(bias, wdtype) ||
      !elem_aligned(mean, ZO_F32) || !elem_aligned(rstd, ZO_F32))
    return refuse(ZO_ERR_ALIGN, "zo_layernorm_forward: a buffer is not aligned to its elements");
  zo::LayerNormArgs a{};
  a.x = X;
  a.r = R;
  a.weight = weight;
  a.bias = bias;
  a.y = Y;
  a.h = H;
  a.mean = mean;
  a.rstd = rstd;
  a.rows = rows;
  a.cols = cols;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldy = ldy;
  a.ldh = ldh;
  a.dtype = dtype;
  a.wdtype = wdtype;
  a.eps = eps;
  const int32_t sms = sm_count();
  a.status = status_word();
  if (sms <= 0 || !a.status) return refuse(ZO_ERR_CUDA, "zo_layernorm_forward: no usable CUDA device");
  ZO_CUDA(zo::launch_layernorm_forward(a, sms, reinterpret_cast<cudaStream_t>(stream)),
          "layer norm forward kernel");
  return ZO_OK;
}

int64_t zo_layernorm_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || rows >= kMaxExtent || cols < 1 || cols >= kMaxExtent) return 0;
  const int32_t sms = sm_count();
  if (sms <= 0) return 0;
  return zo::layernorm_partial_rows(rows, cols, sms) * 2 * cols * (int64_t)sizeof(float);
}

zo_status zo_layernorm_backward(const void* dY, int64_t lddy, const void* X, int64_t ldx,
                                const void* dR, int64_t lddr, int64_t rows, int64_t cols,
                                int32_t dtype, const void* weight, int32_t wdtype,
                                const float* mean, const float* rstd, void* dX, int64_t lddx,
                                void* dweight, void* dbias, void* workspace,
                                int64_t workspace_bytes, void* stream) {
  const zo_status st = check_rows(rows, cols, dtype, wdtype);
  if (st != ZO_OK) return st;
  if (lddy < cols || ldx < cols || lddx < cols || (dR && lddr < cols))
    return refuse(ZO_ERR_SHAPE, "zo_layernorm_backward: a row stride is smaller than cols");
  if (rows > 0 && (!dY || !X || !mean || !rstd || !dX))
    return refuse(ZO_ERR_INVALID_ARG, "zo_layernorm_backward: null dY, X, mean, rstd or dX");
  if (!elem_aligned(dY, dtype) || !elem_aligned(X, dtype) || !elem_aligned(dR, dtype) ||
      !elem_aligned(dX, dtype) || !elem_aligned(weight, wdtype) || !elem_aligned(dweight, wdtype) ||
      !elem_aligned(dbias, wdtype) || !elem_aligned(mean, ZO_F32) || !elem_aligned(rstd, ZO_F32) ||
      !aligned16(workspace))
    return refuse(ZO_ERR_ALIGN, "zo_layernorm_backward: a buffer is not aligned to its elements "
                                "(the workspace: to 16 bytes)");
  const bool sums = dweight || dbias;
  if (rows == 0 && !sums) return ZO_OK;
  const int32_t sms = sm_count();
  if (sms <= 0) return refuse(ZO_ERR_CUDA, "zo_layernorm_backward: no usable CUDA device");
  if (sums && rows > 0 &&
      (!workspace || workspace_bytes < zo_layernorm_workspace(rows, cols)))
    return refuse(ZO_ERR_INVALID_ARG,
                  "zo_layernorm_backward: the workspace is missing or smaller than "
                  "zo_layernorm_workspace(rows, cols)");
  zo::LayerNormArgs a{};
  a.status = status_word();
  if (!a.status) return refuse(ZO_ERR_CUDA, "zo_layernorm_backward: no usable CUDA device");
  a.dy = dY;
  a.x = X;
  a.r = dR;
  a.weight = weight;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dx = dX;
  a.dweight = dweight;
  a.dbias = dbias;
  a.partial = sums ? static_cast<float*>(workspace) : nullptr;
  a.rows = rows;
  a.cols = cols;
  a.lddy = lddy;
  a.ldx = ldx;
  a.ldr = lddr;
  a.lddx = lddx;
  a.dtype = dtype;
  a.wdtype = wdtype;
  ZO_CUDA(zo::launch_layernorm_backward(a, sms, reinterpret_cast<cudaStream_t>(stream)),
          "layer norm backward kernels");
  return ZO_OK;
}

zo_status zo_layernorm_sync_status(void* stream) {
  const auto s = reinterpret_cast<cudaStream_t>(stream);
  uint32_t* word = status_word();
  if (!word) return refuse(ZO_ERR_CUDA, "zo_layernorm_sync_status: no usable CUDA device");
  uint32_t status = 0;
  ZO_CUDA(cudaMemcpyAsync(&status, word, sizeof(status), cudaMemcpyDeviceToHost, s), "read status");
  ZO_CUDA(cudaStreamSynchronize(s), "stream synchronize");
  if (status != 0) {
    ZO_CUDA(cudaMemsetAsync(word, 0, sizeof(status), s), "clear status");
    ZO_CUDA(cudaStreamSynchronize(s), "stream synchronize");
    return refuse(ZO_ERR_TIMEOUT, "layer norm: a device-side wait ran out");
  }
  return ZO_OK;
}

}  // extern "C"
