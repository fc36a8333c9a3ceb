// Newton-Schulz orthogonalisation of matrices of at most 32 rows in one launch, in fp32.
//
// A matrix is a cluster of C CTAs, each with its share of X's columns in shared memory.  A
// step:  Gram   the CTA's X X^T, K dealt to its eight warps (each lane a P/4 x P/8 tile of the
//               P x P sums), added up in warp order, then over the cluster in rank order: every
//               CTA reads all the partial sums through distributed shared memory, so one
//               cluster barrier a step is enough;
//        Poly   B = b A + c A A, by every CTA for itself, four values per thread;
//        Apply  X' = a X + B X in place, 4 x 4 (or, in few columns, 4 x 1) per thread.
//
// Latency-bound: at 32 x 32 a product is a few hundred cycles of multiply-adds, less than a
// round trip through the tensor cores (~1000 cycles to issue, commit and wait), which the
// wider matrices of zo_ortho_small.cu make up by their size.
#include <algorithm>

#include "zo_launch.cuh"
#include "zo_ops.h"
#include "zo_ortho_io.cuh"

namespace zo {
namespace {

using namespace ortho;

constexpr int kThreads = 256;
constexpr int kMaxCluster = 8;
constexpr int kWarps = kThreads / 32;
constexpr int kSmemMax = 227 * 1024;

__host__ __device__ constexpr int fma_rows(int64_t p) { return p <= 8 ? 8 : p <= 16 ? 16 : 32; }
// columns of a CTA, a multiple of 32
__host__ __device__ inline int fma_cols(int64_t c, int cluster) {
  return (int)(((c + cluster - 1) / cluster + 31) / 32 * 32);
}
__host__ __device__ constexpr int fma_floats(int P, int cs) {
  return P * (cs + 4) + 2 * P * (P + 4) + 2 * P * P + kWarps * P * P;
}

struct Coeffs {
  float a[kOrthoMaxSteps], b[kOrthoMaxSteps], c[kOrthoMaxSteps];
  int n;
};

// X' of kC neighbouring columns and four rows per thread, a sweep of columns at a time; all
// rows of a column fall in one sweep, which reads before it writes.
template <int P, int kC>
__device__ __forceinline__ void apply(float* X, const float* B, int ld, int cs, float a) {
  constexpr int kGroups = kThreads / (P / 4);               // column groups of a sweep
  const int i0 = (int)threadIdx.x / kGroups * 4;
  for (int s = 0; s < cs; s += kGroups * kC) {
    const int j = s + (int)threadIdx.x % kGroups * kC;
    float v[4][kC] = {};
    if (j < cs) {
#pragma unroll 8
      for (int k = 0; k < P; ++k) {
        const float4 b = *reinterpret_cast<const float4*>(B + k * (P + 4) + i0);
        float x[kC];
        if constexpr (kC == 4) {
          const float4 q = *reinterpret_cast<const float4*>(X + k * ld + j);
          x[0] = q.x; x[1] = q.y; x[2] = q.z; x[3] = q.w;
        } else {
          x[0] = X[k * ld + j];
        }
#pragma unroll
        for (int e = 0; e < kC; ++e) {
          v[0][e] = fmaf(b.x, x[e], v[0][e]);
          v[1][e] = fmaf(b.y, x[e], v[1][e]);
          v[2][e] = fmaf(b.z, x[e], v[2][e]);
          v[3][e] = fmaf(b.w, x[e], v[3][e]);
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < kC; ++e) v[r][e] = fmaf(a, X[(i0 + r) * ld + j + e], v[r][e]);
    }
    __syncthreads();
    if (j < cs) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (kC == 4)
          *reinterpret_cast<float4*>(X + (i0 + r) * ld + j) =
              make_float4(v[r][0], v[r][1], v[r][2], v[r][3]);
        else
          X[(i0 + r) * ld + j] = v[r][0];
      }
    }
  }
  __syncthreads();
}

template <int P>
__global__ void __launch_bounds__(kThreads)
ortho_fma_kernel(const OrthoMat* __restrict__ mats, const int* __restrict__ which, int cluster,
                 const __grid_constant__ Coeffs co, const OrthoUpdate u) {
  extern __shared__ float4 smem4[];
  __shared__ SumShared sums;
  const OrthoMat mt = mats[which[blockIdx.x / cluster]];
  const int rank = (int)(blockIdx.x % cluster);
  const int cs = fma_cols(mt.c, cluster), ld = cs + 4;
  float* X = reinterpret_cast<float*>(smem4);
  float* A = X + P * ld;
  float* B = A + P * (P + 4);
  float* red = B + P * (P + 4);
  float* part = red + 2 * P * P;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t c0 = (int64_t)rank * cs;
  const int cols = (int)max((int64_t)0, min((int64_t)cs, mt.c - c0));

  for (int e = tid; e < P * ld / 4; e += kThreads) smem4[e] = make_float4(0.f, 0.f, 0.f, 0.f);
  __syncthreads();
  pdl_wait();
  pdl_trigger();

  // ---------------------------------------------------------------- U, scaled by its norm
  const int64_t n = mt.tall ? mt.p : cols;
  const bool fours = by_fours(mt.G, mt.ldg, mt.grad_bf16, n) &&
                     (mt.M == nullptr || !u.step || by_fours(mt.M, mt.n, 0, n));
  float sq;
  if (fours) {
    sq = load_update<kThreads, 4>(mt, u, c0, cols, [&](int i, int j, const float (&v)[4]) {
      if (mt.tall) {
#pragma unroll
        for (int e = 0; e < 4; ++e) X[(i + e) * ld + j] = v[e];
      } else {
        *reinterpret_cast<float4*>(X + i * ld + j) = make_float4(v[0], v[1], v[2], v[3]);
      }
    });
  } else {
    sq = load_update<kThreads, 1>(mt, u, c0, cols,
                        [&](int i, int j, const float (&v)[1]) { X[i * ld + j] = v[0]; });
  }
  const float inv = inverse_norm<kThreads>(sq, u.eps, cluster, sums);
  for (int e = tid; e < P * ld / 4; e += kThreads) {
    float4 v = smem4[e];
    smem4[e] = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
  }
  __syncthreads();

  // ---------------------------------------------------------------- the steps
  constexpr int kTy = P / 4, kTx = P / 8;
  const int ly = lane >> 3, lx = lane & 7;
  for (int k = 0; k < co.n; ++k) {
    float acc[kTy][kTx] = {};
    for (int k4 = warp * 4; k4 < cs; k4 += 4 * kWarps) {
      float4 xa[kTy], xb[kTx];
#pragma unroll
      for (int a = 0; a < kTy; ++a) xa[a] = *reinterpret_cast<const float4*>(X + (ly + 4 * a) * ld + k4);
#pragma unroll
      for (int b = 0; b < kTx; ++b) xb[b] = *reinterpret_cast<const float4*>(X + (lx + 8 * b) * ld + k4);
#pragma unroll
      for (int a = 0; a < kTy; ++a)
#pragma unroll
        for (int b = 0; b < kTx; ++b) {
          acc[a][b] = fmaf(xa[a].x, xb[b].x, acc[a][b]);
          acc[a][b] = fmaf(xa[a].y, xb[b].y, acc[a][b]);
          acc[a][b] = fmaf(xa[a].z, xb[b].z, acc[a][b]);
          acc[a][b] = fmaf(xa[a].w, xb[b].w, acc[a][b]);
        }
    }
#pragma unroll
    for (int a = 0; a < kTy; ++a)
#pragma unroll
      for (int b = 0; b < kTx; ++b) part[warp * P * P + (ly + 4 * a) * P + lx + 8 * b] = acc[a][b];
    __syncthreads();
    // the partial sums alternate between two buffers: those of the step before the last have
    // been read by every CTA once the last step's barrier is passed
    float* mine = red + (k & 1) * P * P;
    for (int e = tid; e < P * P; e += kThreads) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) s += part[w * P * P + e];
      if (cluster > 1) mine[e] = s;
      else A[e / P * (P + 4) + e % P] = s;
    }
    if (cluster > 1) {
      cta2::cluster_sync_all();
      for (int e = tid; e < P * P; e += kThreads) {
        float v[kMaxCluster];
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r)
          if (r < cluster)
            asm volatile("ld.shared::cluster.f32 %0, [%1];"
                         : "=f"(v[r]) : "r"(cta2::map_to(mine + e, (uint32_t)r)) : "memory");
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r)
          if (r < cluster) s += v[r];
        A[e / P * (P + 4) + e % P] = s;
      }
    }
    __syncthreads();
    if (tid < P * P / 4) {
      const int i = tid / (P / 4), j = tid % (P / 4) * 4;
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
      for (int q = 0; q < P; ++q) {
        const float a = A[i * (P + 4) + q];
        const float4 r = *reinterpret_cast<const float4*>(A + q * (P + 4) + j);
        s.x = fmaf(a, r.x, s.x); s.y = fmaf(a, r.y, s.y);
        s.z = fmaf(a, r.z, s.z); s.w = fmaf(a, r.w, s.w);
      }
      const float4 r = *reinterpret_cast<const float4*>(A + i * (P + 4) + j);
      const float b = co.b[k], c = co.c[k];
      *reinterpret_cast<float4*>(B + i * (P + 4) + j) =
          make_float4(fmaf(b, r.x, c * s.x), fmaf(b, r.y, c * s.y), fmaf(b, r.z, c * s.z),
                      fmaf(b, r.w, c * s.w));
    }
    __syncthreads();
    // one column a thread where that already takes half of the threads
    if (P / 4 * cs <= 2 * kThreads) apply<P, 1>(X, B, ld, cs, co.a[k]);
    else apply<P, 4>(X, B, ld, cs, co.a[k]);
  }

  // ---------------------------------------------------------------- the result
  if (by_fours(mt.W, mt.ldw, mt.bf16, n)) {
    store_result<kThreads, 4>(mt, u, c0, cols, [&](int i, int j, float (&v)[4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = mt.tall ? X[(i + e) * ld + j] : X[i * ld + j + e];
    });
  } else {
    store_result<kThreads, 1>(mt, u, c0, cols, [&](int i, int j, float (&v)[1]) { v[0] = X[i * ld + j]; });
  }
  if (cluster > 1) cta2::cluster_sync_all();     // the peers have read this CTA's sums
}

template <int P>
cudaError_t launch(const OrthoMat* mats, const int* which, int32_t n, int32_t cluster, int32_t smem,
                   const Coeffs& co, const OrthoUpdate& u, cudaStream_t s) {
  const cudaError_t e = cudaFuncSetAttribute(
      ortho_fma_kernel<P>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax - 1024);
  if (e != cudaSuccess) return e;
  return launch_dependent(ortho_fma_kernel<P>, (unsigned)n * (unsigned)cluster, kThreads,
                          (size_t)smem, s, (unsigned)cluster, true, mats, which, cluster, co, u);
}

}  // namespace

int32_t ortho_fma_rows(int64_t p) { return p <= 32 ? fma_rows(p) : 0; }
int32_t ortho_fma_cluster(int64_t p, int64_t c) {
  if (p > 32) return 0;
  const int P = fma_rows(p);
  for (int cl = 1; cl <= kMaxCluster; cl *= 2) {
    if (c > (int64_t)cl << 16) continue;
    const int cs = fma_cols(c, cl);
    // a CTA takes 10240 elements while the cluster can still grow: 8 x 5120 on four
    if (cl < kMaxCluster && P * cs > 10240) continue;
    if (4 * (int64_t)fma_floats(P, cs) <= kSmemMax - 1024) return cl;
  }
  return 0;
}
int32_t ortho_fma_smem(int64_t p, int64_t c, int32_t cluster) {
  return 4 * fma_floats(fma_rows(p), fma_cols(c, cluster));
}

cudaError_t launch_ortho_fma(const OrthoMat* mats, const int* which, int32_t n, int32_t rows,
                             int32_t cluster, int32_t smem, const OrthoStep* steps,
                             int32_t n_steps, const OrthoUpdate& u, cudaStream_t s) {
  if (n <= 0) return cudaSuccess;
  if (n_steps > kOrthoMaxSteps || smem > kSmemMax - 1024) return cudaErrorInvalidValue;
  Coeffs co{};
  co.n = n_steps;
  for (int32_t k = 0; k < n_steps; ++k) {
    co.a[k] = steps[k].a;
    co.b[k] = steps[k].b;
    co.c[k] = steps[k].c;
  }
  switch (rows) {
    case 8: return launch<8>(mats, which, n, cluster, smem, co, u, s);
    case 16: return launch<16>(mats, which, n, cluster, smem, co, u, s);
    case 32: return launch<32>(mats, which, n, cluster, smem, co, u, s);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace zo
