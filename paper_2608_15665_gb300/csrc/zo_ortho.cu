// Newton-Schulz orthogonalisation: X <- a X + (b A + c A A) X with A = X X^T, and the Muon
// update around it (declared in include/zo.h).
//
// A step is three products over all matrices of a group: A = X X^T and B = b A + c A A, both
// symmetric (only tiles on or below the diagonal are computed, and written twice), and
// X' = a X + B X.  Iterates are held as fp16 values of x 2^e: every entry of X_k, A and B is
// bounded by its spectral norm, which the host follows through the steps, so e puts the bound
// just below fp16's 65504 and 2^-29 of it is still a normal number.
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
__device__ __forceinline__ float f16_value(const uint16_t* p) {
  return __half2float(*reinterpret_cast<const __half*>(p));
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
      const int r = mt.tall ? e % 64 : e / 64, c = mt.tall ? e / 64 : e % 64;
      const int64_t i = i0 + r, j = j0 + c;
      if (i >= mt.m || j >= mt.n) continue;
      const int64_t at = mt.tall ? j * mt.ldx + i : i * mt.ldx + j;
      split(tile[r][c], mt.xh[0][at], mt.xl[0][at]);
    }
  }
}

// one element of a product: D = the accumulated sum
__device__ __forceinline__ void finish(const OrthoMat& mt, int phase, const OrthoStep& st,
                                       const OrthoUpdate& u, int64_t i, int64_t j, float d) {
  uint16_t hi, lo;
  if (phase == kOrthoApply) {
    const int64_t at = i * mt.ldx + j;
    const float x = f16_value(mt.xh[st.k & 1] + at) + f16_value(mt.xl[st.k & 1] + at);
    const float v = st.a * x * exp2i(-st.ex) + d * exp2i(-st.ex - st.eb);
    if (!st.last) {
      split(v * exp2i(st.ex_next), hi, lo);
      mt.xh[(st.k & 1) ^ 1][at] = hi;
      mt.xl[(st.k & 1) ^ 1][at] = lo;
      return;
    }
    const int64_t w = mt.tall ? j * mt.ldw + i : i * mt.ldw + j;
    float out = v;
    if (u.step) {
      const float m = (float)mt.m, n = (float)mt.n;
      const float s = u.adjust == 1 ? sqrtf(fmaxf(1.0f, m / n))
                                    : u.adjust == 2 ? 0.2f * sqrtf(fmaxf(m, n)) : 1.0f;
      out = fmaf(-u.lr * s, v, u.keep * element(mt.W, mt.bf16, w));
    }
    if (mt.bf16) static_cast<__nv_bfloat16*>(mt.W)[w] = __float2bfloat16_rn(out);
    else static_cast<float*>(mt.W)[w] = out;
    return;
  }
  if (i < j) return;                                      // a diagonal tile's upper half
  const int64_t at = i * mt.ldp + j, mirror = j * mt.ldp + i;
  if (phase == kOrthoGram) {
    split(d * exp2i(st.ea - 2 * st.ex), hi, lo);
    mt.ah[at] = mt.ah[mirror] = hi;
    if (mt.pairs) mt.al[at] = mt.al[mirror] = lo;
  } else {
    float a = f16_value(mt.ah + at);
    if (mt.pairs) a += f16_value(mt.al + at);
    split((st.b * a * exp2i(-st.ea) + st.c * d * exp2i(-2 * st.ea)) * exp2i(st.eb), hi, lo);
    mt.bh[at] = mt.bh[mirror] = hi;
    if (mt.pairs) mt.bl[at] = mt.bl[mirror] = lo;
  }
}

// 64 x 64 of a product, 16 of K at a time, 4 x 4 per thread
__global__ void __launch_bounds__(256)
product_kernel(const OrthoMat* __restrict__ mats, const int4* __restrict__ tiles, int phase,
               const OrthoStep st, const OrthoUpdate u) {
  __shared__ float as[16][65], bs[16][65];
  const int4 t = tiles[blockIdx.x];
  const OrthoMat mt = mats[t.x];
  pdl_wait();
  pdl_trigger();
  const int64_t i0 = t.y, j0 = t.z;
  const int64_t K = phase == kOrthoGram ? mt.c : mt.p;
  const int64_t rows_b = phase == kOrthoApply ? mt.c : mt.p;
  const uint16_t* xh = mt.xh[st.k & 1];
  const uint16_t* xl = mt.xl[st.k & 1];
  const uint16_t* ah = phase == kOrthoGram ? xh : phase == kOrthoPoly ? mt.ah : mt.bh;
  const uint16_t* al = phase == kOrthoGram ? xl : phase == kOrthoPoly ? mt.al : mt.bl;
  const uint16_t* bh = phase == kOrthoPoly ? mt.ah : xh;
  const uint16_t* bl = phase == kOrthoPoly ? mt.al : xl;
  const int64_t lda = phase == kOrthoGram ? mt.ldx : mt.ldp;
  const int64_t ldb = phase == kOrthoPoly ? mt.ldp : mt.ldx;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float acc[4][4] = {};
  for (int64_t k0 = 0; k0 < K; k0 += 16) {
    for (int e = threadIdx.x; e < 64 * 16; e += 256) {
      const int r = e / 16, kk = e % 16;
      const int64_t i = i0 + r, k = k0 + kk;
      float v = 0.0f;
      if (i < mt.p && k < K) {
        v = f16_value(ah + i * lda + k);
        if (mt.pairs) v += f16_value(al + i * lda + k);
      }
      as[kk][r] = v;
    }
    for (int e = threadIdx.x; e < 64 * 16; e += 256) {
      // B's rows are X's columns in the last product
      const int r = phase == kOrthoApply ? e % 64 : e / 16, kk = phase == kOrthoApply ? e / 64 : e % 16;
      const int64_t j = j0 + r, k = k0 + kk;
      float v = 0.0f;
      if (j < rows_b && k < K) {
        const int64_t at = phase == kOrthoApply ? k * ldb + j : j * ldb + k;
        v = f16_value(bh + at);
        if (mt.pairs) v += f16_value(bl + at);
      }
      bs[kk][r] = v;
    }
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < 16; ++kk)
#pragma unroll
      for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[a][b] = fmaf(as[kk][ty * 4 + a], bs[kk][tx * 4 + b], acc[a][b]);
    __syncthreads();
  }
  for (int a = 0; a < 4; ++a)
    for (int b = 0; b < 4; ++b) {
      const int64_t i = i0 + ty * 4 + a, j = j0 + tx * 4 + b;
      if (i < mt.p && j < rows_b) finish(mt, phase, st, u, i, j, acc[a][b]);
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
cudaError_t launch_ortho_product(const OrthoMat* mats, const int4* tiles, int32_t n_tiles,
                                 OrthoPhase phase, const OrthoStep& st, const OrthoUpdate& u,
                                 cudaStream_t s) {
  return launch_dependent(product_kernel, (unsigned)n_tiles, 256, 0, s, 1, true, mats, tiles,
                          (int)phase, st, u);
}

}  // namespace zo
