// Before the products of a Newton-Schulz orthogonalisation (zo_ortho_gemm.cu): the Muon
// update's momentum, the Frobenius norm of U, and X_0 = U / (||U|| + eps).
//
// Iterates are held as fp16 values of x 2^e: every entry of X_k, A and B is bounded by its
// spectral norm, which the host follows through the steps, so e puts the bound just below
// fp16's 65504 and 2^-29 of it is still a normal number.
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "zo_launch.cuh"
#include "zo_ops.h"
#include "zo_tc_common.cuh"

namespace zo {
namespace {

using tc::exp2i;

__device__ __forceinline__ float element(const void* p, int bf16, int64_t at) {
  return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at])
              : static_cast<const float*>(p)[at];
}
// x = hi + lo in fp16
__device__ __forceinline__ void split(float x, uint16_t& hi, uint16_t& lo) {
  const __half h = __float2half_rn(x);
  const __half l = __float2half_rn(x - __half2float(h));
  hi = *reinterpret_cast<const uint16_t*>(&h);
  lo = *reinterpret_cast<const uint16_t*>(&l);
}

constexpr int kUnitThreads = 256;
static_assert(kOrthoUnitCols == kUnitThreads, "a column per thread");

// U of one element, and with `write` the new momentum
template <bool kWrite>
__device__ __forceinline__ float update_of(const OrthoMat& mt, const OrthoUpdate& u, int64_t i,
                                           int64_t j) {
  const float g = element(mt.G, mt.grad_bf16, i * mt.ldg + j);
  if (!u.step || mt.M == nullptr) return g;
  float* m = mt.M + i * mt.n + j;
  float mom = *m;
  if constexpr (kWrite) {
    mom = fmaf(u.momentum, mom, g);
    *m = mom;
  }
  return u.nesterov ? fmaf(u.momentum, mom, g) : mom;
}

// M <- momentum M + G, and the sum of U^2 over each unit
__global__ void __launch_bounds__(kUnitThreads)
momentum_kernel(const OrthoMat* __restrict__ mats, const int4* __restrict__ units,
                const OrthoUpdate u, float* __restrict__ partial) {
  __shared__ float sums[kUnitThreads / 32];
  const int4 un = units[blockIdx.x];
  const OrthoMat mt = mats[un.x];
  pdl_wait();
  pdl_trigger();
  const int64_t j = (int64_t)un.z + threadIdx.x;
  const int64_t end = min((int64_t)un.y + kOrthoUnitRows, mt.m);
  float s = 0.0f;
  if (j < mt.n)
    for (int64_t i = un.y; i < end; ++i) {
      const float v = update_of<true>(mt, u, i, j);
      s = fmaf(v, v, s);
    }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0f;
    for (int w = 0; w < kUnitThreads / 32; ++w) s += sums[w];
    partial[un.w] = s;
  }
}

// X_0 = U / (||U|| + eps)
__global__ void __launch_bounds__(kUnitThreads)
scale_kernel(const OrthoMat* __restrict__ mats, const int4* __restrict__ units,
             const OrthoUpdate u, int ex, const float* __restrict__ partial) {
  __shared__ float tile[64][65];
  __shared__ double sums[kUnitThreads / 32];
  const int4 un = units[blockIdx.x];
  const OrthoMat mt = mats[un.x];
  pdl_wait();
  pdl_trigger();
  double s = 0.0;
  for (int k = threadIdx.x; k < mt.n_units; k += kUnitThreads) s += (double)partial[mt.unit0 + k];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < kUnitThreads / 32; ++w) s += sums[w];
  const float norm = (float)sqrt(s) + u.eps;
  const float inv = norm == 0.0f ? 0.0f : exp2i(ex) / norm;
  const int64_t i0 = un.y;
  for (int64_t j0 = un.z; j0 < min((int64_t)un.z + kOrthoUnitCols, mt.n); j0 += 64) {
    __syncthreads();
    for (int e = threadIdx.x; e < 64 * 64; e += kUnitThreads) {
      const int64_t i = i0 + e / 64, j = j0 + e % 64;
      if (i < mt.m && j < mt.n) tile[e / 64][e % 64] = update_of<false>(mt, u, i, j) * inv;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 64 * 64; e += kUnitThreads) {
      // X's row and column; TMA moves whole 16-byte chunks, so a row's last one ends in zeros
      const int64_t row = (mt.tall ? j0 : i0) + e / 64, col = (mt.tall ? i0 : j0) + e % 64;
      if (row >= mt.p || col >= (mt.c + 7) / 8 * 8) continue;
      const float x = col >= mt.c ? 0.0f : mt.tall ? tile[e % 64][e / 64] : tile[e / 64][e % 64];
      split(x, mt.xh[0][row * mt.ldx + col], mt.xl[0][row * mt.ldx + col]);
    }
  }
}

}  // namespace

cudaError_t launch_ortho_momentum(const OrthoMat* mats, const int4* units, int32_t n_units,
                                  const OrthoUpdate& u, float* partial, cudaStream_t s) {
  return launch_dependent(momentum_kernel, (unsigned)n_units, kUnitThreads, 0, s, 1, true, mats,
                          units, u, partial);
}
cudaError_t launch_ortho_scale(const OrthoMat* mats, const int4* units, int32_t n_units,
                               const OrthoUpdate& u, int32_t ex, const float* partial,
                               cudaStream_t s) {
  return launch_dependent(scale_kernel, (unsigned)n_units, kUnitThreads, 0, s, 1, true, mats, units,
                          u, ex, partial);
}

}  // namespace zo
