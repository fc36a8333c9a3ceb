// What the one-launch orthogonalisation kernels (zo_ortho_mma.cu, zo_ortho_small.cu) share: a
// CTA's walk over its columns of the caller's matrices, and a cluster's sum of one value.
#pragma once

#include <cuda_bf16.h>

#include "zo_cluster.cuh"
#include "zo_ops.h"
#include "zo_tc_common.cuh"

namespace zo {
namespace ortho {

// One lane of a warp that is here as a whole.  Under elect.sync the compiler keeps addresses and
// descriptors in uniform registers: a tcgen05.mma is issued every ~40 cycles, against ~66 (~85
// in a product's loop) from a branch on the lane's number.
__device__ __forceinline__ bool elected() {
  uint32_t e;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(e));
  return e != 0;
}

// (kThreads: threads of the CTA)

// kV consecutive values of a bf16 or fp32 buffer
template <int kV>
__device__ __forceinline__ void load_values(const void* p, int bf16, int64_t at, float (&v)[kV]) {
  if constexpr (kV == 4) {
    if (bf16) {
      const uint2 q = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(p) + at);
      v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xFFFF0000u);
      v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xFFFF0000u);
    } else {
      const float4 q = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
      v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    }
  } else {
    v[0] = bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at])
                : static_cast<const float*>(p)[at];
  }
}
template <int kV>
__device__ __forceinline__ void store_values(void* p, int bf16, int64_t at, const float (&v)[kV]) {
  if constexpr (kV == 4) {
    if (bf16) {
      const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p) + at) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    } else {
      *reinterpret_cast<float4*>(static_cast<float*>(p) + at) = make_float4(v[0], v[1], v[2], v[3]);
    }
  } else {
    if (bf16) static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v[0]);
    else static_cast<float*>(p)[at] = v[0];
  }
}

// whether rows of a buffer with `ld` elements between them can be read four at a time
__device__ __forceinline__ bool by_fours(const void* p, int64_t ld, int bf16, int64_t n) {
  return n % 4 == 0 && ld % 4 == 0 && reinterpret_cast<uintptr_t>(p) % (bf16 ? 8 : 16) == 0;
}

// This CTA's share of a matrix: X's columns c0 .. c0 + cols - 1, i.e. rows of the caller's
// matrix where it is tall.  Calls f(x_row, x_col, row, col) for the first element of every run
// of kV elements that are neighbours in the caller's rows, four runs of a thread at a time
// through `batch`, which loads before it computes.
template <int kThreads, int kV, typename F>
__device__ __forceinline__ void for_runs(const OrthoMat& mt, int64_t c0, int cols, F batch) {
  const int rows = mt.tall ? cols : (int)mt.p;              // of the caller's matrix
  const int runs = (mt.tall ? (int)mt.p : cols) / kV;       // in each (kV divides it)
  if (rows == 0 || runs == 0) return;
  int r = (int)threadIdx.x / runs, q = (int)threadIdx.x - r * runs;
  const int dr = kThreads / runs, dq = kThreads - dr * runs;
  while (r < rows) {
    int rr[4], qq[4], n = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      rr[k] = r;
      qq[k] = q * kV;
      if (r < rows) {
        n = k + 1;
        r += dr;
        q += dq;
        if (q >= runs) {
          q -= runs;
          ++r;
        }
      }
    }
    batch(rr, qq, n);
  }
}

// M <- momentum M + G and U, of every run: f(x_row, x_col, values) stores them.  Returns this
// thread's sum of U^2.
template <int kThreads, int kV, typename F>
__device__ __forceinline__ float load_update(const OrthoMat& mt, const OrthoUpdate& u, int64_t c0,
                                             int cols, F f) {
  const bool moving = u.step && mt.M != nullptr;
  const int64_t r0 = mt.tall ? c0 : 0, k0 = mt.tall ? 0 : c0;
  float sq = 0.0f;
  for_runs<kThreads, kV>(mt, c0, cols, [&](const int (&r)[4], const int (&q)[4], int n) {
    float g[4][kV], m[4][kV];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < n) load_values<kV>(mt.G, mt.grad_bf16, (r0 + r[k]) * mt.ldg + k0 + q[k], g[k]);
    if (moving) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < n) load_values<kV>(mt.M, 0, (r0 + r[k]) * mt.n + k0 + q[k], m[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k >= n) continue;
      if (moving) {
#pragma unroll
        for (int e = 0; e < kV; ++e) m[k][e] = fmaf(u.momentum, m[k][e], g[k][e]);
        store_values<kV>(mt.M, 0, (r0 + r[k]) * mt.n + k0 + q[k], m[k]);
#pragma unroll
        for (int e = 0; e < kV; ++e)
          g[k][e] = u.nesterov ? fmaf(u.momentum, m[k][e], g[k][e]) : m[k][e];
      }
#pragma unroll
      for (int e = 0; e < kV; ++e) sq = fmaf(g[k][e], g[k][e], sq);
      f(mt.tall ? q[k] : r[k], mt.tall ? r[k] : q[k], g[k]);
    }
  });
  return sq;
}

// W <- keep W - lr s O, or W <- O: f(x_row, x_col, values) fetches O's run.
template <int kThreads, int kV, typename F>
__device__ __forceinline__ void store_result(const OrthoMat& mt, const OrthoUpdate& u, int64_t c0,
                                             int cols, F f) {
  const int64_t r0 = mt.tall ? c0 : 0, k0 = mt.tall ? 0 : c0;
  const float fm = (float)mt.m, fn = (float)mt.n;
  const float rate = u.lr * (u.adjust == 1 ? sqrtf(fmaxf(1.0f, fm / fn))
                             : u.adjust == 2 ? 0.2f * sqrtf(fmaxf(fm, fn)) : 1.0f);
  for_runs<kThreads, kV>(mt, c0, cols, [&](const int (&r)[4], const int (&q)[4], int n) {
    float w[4][kV];
    if (u.step) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < n) load_values<kV>(mt.W, mt.bf16, (r0 + r[k]) * mt.ldw + k0 + q[k], w[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k >= n) continue;
      float o[kV];
      f(mt.tall ? q[k] : r[k], mt.tall ? r[k] : q[k], o);
      if (u.step) {
#pragma unroll
        for (int e = 0; e < kV; ++e) o[e] = fmaf(-rate, o[e], u.keep * w[k][e]);
      }
      store_values<kV>(mt.W, mt.bf16, (r0 + r[k]) * mt.ldw + k0 + q[k], o);
    }
  });
}

struct SumShared {
  float warp[32];
  float cta;
  uint32_t warp_most[32];
  uint32_t cta_most;
};
// Sum of the threads' values (in warp, then rank order); every CTA of the cluster gets the same.
// A barrier of the CTA's threads lies between earlier and later work.
template <int kThreads>
__device__ __forceinline__ float cluster_sum(float v, int cluster, SumShared& sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) sh.warp[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0f;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) v += sh.warp[w];
  if (cluster > 1) {
    if (threadIdx.x == 0) sh.cta = v;
    cta2::cluster_sync_all();
    v = 0.0f;
    for (int r = 0; r < cluster; ++r) {
      float q;
      asm volatile("ld.shared::cluster.f32 %0, [%1];"
                   : "=f"(q) : "r"(cta2::map_to(&sh.cta, (uint32_t)r)) : "memory");
      v += q;
    }
  }
  return v;
}
// the largest of the threads' values
template <int kThreads>
__device__ __forceinline__ uint32_t cluster_most(uint32_t v, int cluster, SumShared& sh) {
  v = __reduce_max_sync(0xffffffffu, v);
  if ((threadIdx.x & 31) == 0) sh.warp_most[threadIdx.x >> 5] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) v = max(v, sh.warp_most[w]);
  if (cluster > 1) {
    if (threadIdx.x == 0) sh.cta_most = v;
    cta2::cluster_sync_all();
    for (int r = 0; r < cluster; ++r) {
      uint32_t q;
      asm volatile("ld.shared::cluster.u32 %0, [%1];"
                   : "=r"(q) : "r"(cta2::map_to(&sh.cta_most, (uint32_t)r)) : "memory");
      v = max(v, q);
    }
  }
  return v;
}

// Sums of squares in this range are exact to fp32: none overflowed, and what a square below fp32's
// smallest numbers lost is no part of the sum's digits.
template <typename T>
__device__ __forceinline__ bool squares_hold(T sum) { return sum >= (T)0x1p-100 && sum <= (T)0x1p120; }
// The exponent by which values of at most `most` (an fp32 value's bits) are scaled for their
// squares: 2^-e most lies in [1, 4), or is subnormal where most is.
__device__ __forceinline__ int square_exponent(uint32_t most) {
  return min(max((int)(most >> 23) - 127, -126), 126);
}
// whether bits of |v| are those of a finite value other than zero
__device__ __forceinline__ bool plain_value(uint32_t bits) { return bits - 1u < 0x7F800000u - 1u; }

// fp32 values as their upper and lower halves, two to a word
__device__ __forceinline__ uint32_t upper2(float a, float b) {
  return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
}
__device__ __forceinline__ uint32_t lower2(float a, float b) {
  return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x5410);
}
__device__ __forceinline__ float first_of(uint32_t up, uint32_t low) {
  return __uint_as_float(__byte_perm(low, up, 0x5410));
}
__device__ __forceinline__ float second_of(uint32_t up, uint32_t low) {
  return __uint_as_float(__byte_perm(low, up, 0x7632));
}

// A CTA's values of U in shared memory: `chunks` times eight, their upper and lower halves.
struct Planes {
  uint4 *up, *low;
  int chunks;
};
// f(v) for every value, which it may change
template <int kThreads, typename F>
__device__ __forceinline__ void for_values(const Planes& x, F f) {
  for (int c = threadIdx.x; c < x.chunks; c += kThreads) {
    uint32_t up[4] = {x.up[c].x, x.up[c].y, x.up[c].z, x.up[c].w};
    uint32_t low[4] = {x.low[c].x, x.low[c].y, x.low[c].z, x.low[c].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float a = first_of(up[k], low[k]), b = second_of(up[k], low[k]);
      f(a);
      f(b);
      up[k] = upper2(a, b);
      low[k] = lower2(a, b);
    }
    x.up[c] = make_uint4(up[0], up[1], up[2], up[3]);
    x.low[c] = make_uint4(low[0], low[1], low[2], low[3]);
  }
}
// U scaled by a power of two to squares within fp32: their sum, and the power of two in `scale`.
// (Not inlined: in place, forty 8 x 5120 Muon steps took 26.8 us instead of 26.5; without it 26.1.)
template <int kThreads>
__device__ __noinline__ float scaled_squares(Planes x, float sum, int cluster, SumShared& sh, float& scale) {
  uint32_t most = 0;
  for_values<kThreads>(x, [&](float& v) { most = max(most, __float_as_uint(v) & 0x7FFFFFFFu); });
  most = cluster_most<kThreads>(most, cluster, sh);
  if (!plain_value(most)) return sum;              // zero, or not finite: as it is
  const float s = tc::exp2i(-square_exponent(most));
  scale = s;
  sum = 0.0f;
  for_values<kThreads>(x, [&](float& v) {
    v *= s;
    sum = fmaf(v, v, sum);
  });
  return cluster_sum<kThreads>(sum, cluster, sh);
}

// 1 / (||U|| + eps) from the threads' sums of squares; every CTA of the cluster gets the same.
// Where ||U||^2 is beyond fp32 (||U|| above 2^60 or below 2^-50), U is scaled first.
template <int kThreads>
__device__ __forceinline__ float inverse_norm(float sq, float eps, int cluster, SumShared& sh,
                                              const Planes& x) {
  sq = cluster_sum<kThreads>(sq, cluster, sh);
  if (!squares_hold(sq)) {
    float scale = 1.0f;
    sq = scaled_squares<kThreads>(x, sq, cluster, sh, scale);
    eps *= scale;
  }
  const float norm = sqrtf(sq) + eps;
  return norm == 0.0f ? 0.0f : 1.0f / norm;
}

}  // namespace ortho
}  // namespace zo
