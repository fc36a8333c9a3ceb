// Before the products of a Newton-Schulz orthogonalisation (zo_ortho_gemm.cu): the Muon
// update's momentum, the Frobenius norm of U, and X_0 = U / (||U|| + eps).
//
// Iterates are held as fp16 values of x 2^e: every entry of X_k, A and B is bounded by its
// spectral norm, which the host follows through the steps, so e puts the bound just below
// fp16's 65504 and 2^-29 of it is still a normal number.
//
// Bound by HBM: the first kernel reads G and M and writes M, the second, which needs the norm,
// reads both again and writes X's hi and lo parts.  A unit of 32 x 256 elements per CTA, four
// elements a load where the caller's rows allow it; X is written from shared memory, by rows or,
// where U is taller than wide, by columns.  A CTA is a chain of loads, a sum or a tile, and
// stores, so four share an SM, with half of a thread's loads under way at once: for a Muon step's
// 62 M bf16 weights the two kernels took 448 us with two CTAs and all loads at once, 294 us so
// (1.24 GB: 186 us at the copy rate); six CTAs with a quarter of the loads are 25 us faster there
// and 13 us slower at 1001 x 333.
// The norm: each unit's sum of squares, and the last of a matrix's units to finish adds them
// up, in their order.  Where a unit's squares leave fp32, the unit is read again and scaled by a
// power of two; where the norm does, U is scaled before it is divided by it.
#include <algorithm>

#include <cuda_fp16.h>

#include "zo_launch.cuh"
#include "zo_ops.h"
#include "zo_ortho_io.cuh"
#include "zo_tc_common.cuh"

namespace zo {
namespace {

using tc::exp2i;

constexpr int kRows = kOrthoUnitRows, kCols = kOrthoUnitCols;
constexpr int kThreads = 256;
constexpr int kResident = 4;                  // CTAs of an SM
constexpr int kPitch = kCols + 4;             // of a tile in shared memory, in floats
static_assert(kCols == kThreads && kRows % 8 == 0, "a column per thread, or four rows of fours");

// U of this thread's elements: f(row of the unit, column, kV values).  With kWrite the new
// momentum is stored.
template <bool kWrite, int kV, typename F>
__device__ __forceinline__ void for_unit(const OrthoMat& mt, const OrthoUpdate& u, const int4& un, F f) {
  constexpr int kPass = kThreads * kV / kCols;                  // rows at a time: 1 or 4
  constexpr int kBatch = kV == 4 ? 4 : 8;                       // rows under way at once
  const int r0 = (int)threadIdx.x / (kCols / kV), c = (int)threadIdx.x % (kCols / kV) * kV;
  const int64_t j = (int64_t)un.z + c;
  const bool moving = u.step && mt.M != nullptr;
  if (j >= mt.n) return;
  for (int b = 0; b < kRows; b += kPass * kBatch) {
    float g[kBatch][kV], m[kBatch][kV];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int64_t i = (int64_t)un.y + b + k * kPass + r0;
      if (i < mt.m) ortho::load_values<kV>(mt.G, mt.grad_bf16, i * mt.ldg + j, g[k]);
    }
    if (moving) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int64_t i = (int64_t)un.y + b + k * kPass + r0;
        if (i < mt.m) ortho::load_values<kV>(mt.M, 0, i * mt.n + j, m[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int64_t i = (int64_t)un.y + b + k * kPass + r0;
      if (i >= mt.m) continue;
      if (moving) {
        if constexpr (kWrite) {
#pragma unroll
          for (int e = 0; e < kV; ++e) m[k][e] = fmaf(u.momentum, m[k][e], g[k][e]);
          ortho::store_values<kV>(mt.M, 0, i * mt.n + j, m[k]);
        }
#pragma unroll
        for (int e = 0; e < kV; ++e)
          g[k][e] = u.nesterov ? fmaf(u.momentum, m[k][e], g[k][e]) : m[k][e];
      }
      f(b + k * kPass + r0, c, g[k]);
    }
  }
}
template <bool kWrite, typename F>
__device__ __forceinline__ void for_unit(const OrthoMat& mt, const OrthoUpdate& u, const int4& un, F f) {
  if (ortho::by_fours(mt.G, mt.ldg, mt.grad_bf16, mt.n) &&
      (mt.M == nullptr || !u.step || ortho::by_fours(mt.M, mt.n, 0, mt.n)))
    for_unit<kWrite, 4>(mt, u, un, f);
  else
    for_unit<kWrite, 1>(mt, u, un, f);
}

__device__ __forceinline__ double block_sum(double s, double* sums) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) s += sums[w];
  __syncthreads();
  return s;
}

// the sum of U^2 over a unit whose squares are beyond fp32, where its values are not
__device__ __noinline__ double scaled_squares(const OrthoMat* mats, const OrthoUpdate& u, int4 un,
                                              double total, double* sums, uint32_t* mosts) {
  const OrthoMat mt = mats[un.x];
  uint32_t most = 0;
  for_unit<false>(mt, u, un, [&](int, int, const auto& v) {
#pragma unroll
    for (int e = 0; e < (int)(sizeof(v) / sizeof(float)); ++e)
      most = max(most, __float_as_uint(v[e]) & 0x7FFFFFFFu);
  });
  most = __reduce_max_sync(0xffffffffu, most);
  if ((threadIdx.x & 31) == 0) mosts[threadIdx.x >> 5] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) most = max(most, mosts[w]);
  if (!ortho::plain_value(most)) return total;                  // zero, or not finite: as it is
  const int e = ortho::square_exponent(most);
  const float scale = exp2i(-e);
  float s = 0.0f;
  for_unit<false>(mt, u, un, [&](int, int, const auto& v) {
#pragma unroll
    for (int k = 0; k < (int)(sizeof(v) / sizeof(float)); ++k) s = fmaf(v[k] * scale, v[k] * scale, s);
  });
  return block_sum((double)s, sums) * __hiloint2double((1023 + 2 * e) << 20, 0);     // 4^e
}

// M <- momentum M + G, the sum of U^2 over each unit, and of each matrix 2^-e and
// 2^e / (||U|| + eps), e = 0 unless the norm is far from 1
__global__ void __launch_bounds__(kThreads, kResident)
momentum_kernel(const OrthoMat* __restrict__ mats, const int4* __restrict__ units,
                const OrthoUpdate u, double* __restrict__ partial, uint32_t* __restrict__ counter,
                float2* __restrict__ inverse) {
  __shared__ double sums[kThreads / 32];
  __shared__ uint32_t mosts[kThreads / 32];
  __shared__ bool last;
  const int4 un = units[blockIdx.x];
  const OrthoMat mt = mats[un.x];
  pdl_wait();
  pdl_trigger();
  float s = 0.0f;
  for_unit<true>(mt, u, un, [&](int, int, const auto& v) {
#pragma unroll
    for (int e = 0; e < (int)(sizeof(v) / sizeof(float)); ++e) s = fmaf(v[e], v[e], s);
  });
  double total = block_sum((double)s, sums);
  total = ortho::squares_hold(total) ? (double)(float)total
                                     : scaled_squares(mats, u, un, total, sums, mosts);
  if (threadIdx.x == 0) {
    partial[un.w] = total;
    __threadfence();
    last = atomicAdd(&counter[un.x], 1u) == (uint32_t)mt.n_units - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double all = 0.0;
  for (int k = threadIdx.x; k < mt.n_units; k += kThreads)
    all += __ldcg(&partial[mt.unit0 + k]);
  all = block_sum(all, sums);
  if (threadIdx.x == 0) {
    const double root = sqrt(all);
    float scale = 1.0f;
    if (root > 0.0 && root < 0x1p-50) scale = 0x1p126f;
    else if (root > 0x1p60 && root < 0x1p200) scale = 0x1p-126f;  // (more is an infinity)
    const float norm = (float)(root * (double)scale) + u.eps * scale;
    inverse[un.x] = make_float2(scale, norm == 0.0f ? 0.0f : 1.0f / norm);
    counter[un.x] = 0;                                          // for the next call
  }
}

// X_0 = U / (||U|| + eps)
__global__ void __launch_bounds__(kThreads, kResident)
scale_kernel(const OrthoMat* __restrict__ mats, const int4* __restrict__ units,
             const OrthoUpdate u, int ex, const float2* __restrict__ inverse) {
  __shared__ __align__(16) float tile[kRows * kPitch];
  const int4 un = units[blockIdx.x];
  const OrthoMat mt = mats[un.x];
  // TMA moves whole 16-byte chunks, so a row of X ends in zeros up to a multiple of eight: what
  // lies outside U is zero here
  for (int e = threadIdx.x; e < kRows * kPitch / 4; e += kThreads)
    reinterpret_cast<float4*>(tile)[e] = make_float4(0.f, 0.f, 0.f, 0.f);
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const float2 inv = inverse[un.x];
  const float scale = exp2i(ex);
  for_unit<false>(mt, u, un, [&](int r, int c, const auto& v) {
#pragma unroll
    for (int e = 0; e < (int)(sizeof(v) / sizeof(float)); ++e) tile[r * kPitch + c + e] = v[e] * inv.x * inv.y;
  });
  __syncthreads();
  const int64_t width = (mt.c + 7) / 8 * 8;
  for (int e = threadIdx.x; e < kRows * kCols / 4; e += kThreads) {
    // four neighbours of a row of X
    float4 v;
    int64_t row, col;
    if (mt.tall) {
      const int c = e / (kRows / 4), r = e % (kRows / 4) * 4;
      const float* t = tile + r * kPitch + c;
      v = make_float4(t[0], t[kPitch], t[2 * kPitch], t[3 * kPitch]);
      row = (int64_t)un.z + c;
      col = (int64_t)un.y + r;
    } else {
      const int r = e / (kCols / 4), c = e % (kCols / 4) * 4;
      v = *reinterpret_cast<const float4*>(tile + r * kPitch + c);
      row = (int64_t)un.y + r;
      col = (int64_t)un.z + c;
    }
    if (row >= mt.p || col >= width) continue;
    uint2 hi, lo;
    tc::split4_f16(v, scale, hi, lo);
    *reinterpret_cast<uint2*>(mt.xh[0] + row * mt.ldx + col) = hi;
    *reinterpret_cast<uint2*>(mt.xl[0] + row * mt.ldx + col) = lo;
  }
}

}  // namespace

cudaError_t launch_ortho_momentum(const OrthoMat* mats, const int4* units, int32_t n_units,
                                  const OrthoUpdate& u, double* partial, uint32_t* counter,
                                  float2* inverse, cudaStream_t s) {
  return launch_dependent(momentum_kernel, (unsigned)n_units, kThreads, 0, s, 1, true, mats, units,
                          u, partial, counter, inverse);
}
cudaError_t launch_ortho_scale(const OrthoMat* mats, const int4* units, int32_t n_units,
                               const OrthoUpdate& u, int32_t ex, const float2* inverse,
                               cudaStream_t s) {
  return launch_dependent(scale_kernel, (unsigned)n_units, kThreads, 0, s, 1, true, mats, units, u,
                          ex, inverse);
}

}  // namespace zo
