// Host-side helpers shared by the entry points: error reporting, the context's device, and
// tensor-map descriptors.
#pragma once

#include <cstdint>
#include <string>

#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>

#include "../../include/zo.h"

namespace zo {

// Text returned by zo_last_error (zo_api.cu); thread-local.
void set_last_error(const char* msg);

namespace host {

inline zo_status cuda_fail(cudaError_t e, const char* what) {
  set_last_error((std::string(what) + ": " + cudaGetErrorString(e)).c_str());
  return ZO_ERR_CUDA;
}
inline zo_status refuse(zo_status st, const char* why) {
  set_last_error(why);
  return st;
}

#define ZO_CUDA(call, what)                                         \
  do {                                                              \
    cudaError_t _e = (call);                                        \
    if (_e != cudaSuccess) return zo::host::cuda_fail(_e, what);    \
  } while (0)

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Makes a context's device current for the length of a call and gives the caller's back:
// every kernel of a context runs on the device it was created on, whatever device the
// calling thread has selected since.
struct DeviceGuard {
  int prev = -1;
  bool switched = false;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) == cudaSuccess && prev != dev && cudaSetDevice(dev) == cudaSuccess)
      switched = true;
  }
  ~DeviceGuard() {
    if (switched) cudaSetDevice(prev);
  }
};

inline PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  if (!fn) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  }
  return fn;
}

// 2-D tensor map of 16-bit elements (bf16, or fp16 with f16 = true): `cols` contiguous
// elements per row, `rows` rows `row_bytes` apart, boxes of box_cols x box_rows with the
// 128-byte swizzle.
inline bool encode_16b_2d(CUtensorMap* tm, void* base, uint64_t cols, uint64_t rows,
                          uint64_t row_bytes, uint32_t box_cols, uint32_t box_rows, bool f16,
                          CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
  auto enc = tensor_map_encoder();
  if (!enc) return false;
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {row_bytes};
  const cuuint32_t box[2] = {box_cols, box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return enc(tm, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base,
             dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
inline bool encode_bf16_2d(CUtensorMap* tm, void* base, uint64_t cols, uint64_t rows,
                           uint64_t row_bytes, uint32_t box_cols, uint32_t box_rows,
                           CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
  return encode_16b_2d(tm, base, cols, rows, row_bytes, box_cols, box_rows, false, swizzle);
}
inline bool encode_f16_2d(CUtensorMap* tm, void* base, uint64_t cols, uint64_t rows,
                          uint64_t row_bytes, uint32_t box_cols, uint32_t box_rows) {
  return encode_16b_2d(tm, base, cols, rows, row_bytes, box_cols, box_rows, true);
}

}  // namespace host
}  // namespace zo
