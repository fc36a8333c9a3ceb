// Newton-Schulz orthogonalisation of matrices of at most 128 rows in one launch: momentum,
// norm, every step and the update of W, with X in shared memory throughout.
//
// A matrix is a cluster of C CTAs, each with X's columns [rank cs, rank cs + cs).  A step:
//   Gram   each CTA's X X^T on its columns, summed over the cluster through distributed
//          shared memory (CTA r sums the rows of its share and writes them into every CTA);
//   Poly   B = b A + c A A, by every CTA for itself;
//   Apply  the columns' X' = a X + B X, computed as X'^T = X^T B (B is symmetric), so that the
//          128 rows of an MMA are X's columns and no Tensor Memory lane idles at p = 8 or 16.
// All three are M = 128 tcgen05.mma on fp16 hi + lo pairs (hi.lo, lo.hi, then hi.hi), fp32
// accumulators.  X lies in shared memory once, as 128-byte swizzled panels of 64 columns: the
// Gram product reads them as a K-major operand, Apply as an MN-major one.  Rows are padded
// with zeros to a multiple of 16; where an operand has fewer than an MMA's 128 rows, the
// rest of it is whatever follows in shared memory, and those rows of the result are not read.
// The Gram product's K is dealt to up to four accumulators, since the tensor cores' sums
// round towards zero (zo_ortho_gemm.cu).
//
// Latency-bound: three MMA round trips and their epilogues per step (~1 us each), whatever
// the width, and everything else once.  The same matrices by the launches of the SM-pair
// kernel cost 17 launches, each with little work.
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "zo_cluster.cuh"
#include "zo_launch.cuh"
#include "zo_ops.h"
#include "zo_sm100.cuh"
#include "zo_tc_common.cuh"

namespace zo {
namespace {

using namespace sm100;
using tc::exp2i;

constexpr int kThreads = 256;
constexpr int kMaxCluster = 8;
constexpr long long kWait = 4000000000LL;               // ~2 s at 2 GHz
constexpr int kSmemMax = 227 * 1024;

struct Geometry {
  int p16, cs, panels;            // padded rows; columns of a CTA; 64-column panels of X
  int a_panels;                   // 64-column panels of A
  int x_bytes, a_bytes;           // of a hi (or lo) part
  int red_bytes;                  // the cluster's partial Gram sums
  int splits, chunks;             // Gram accumulators; 128-column chunks of Apply
  int tmem_cols;
  int smem;
};
__host__ __device__ inline Geometry geometry(int p, int64_t c, int cluster) {
  Geometry g{};
  g.p16 = (p + 15) / 16 * 16;
  const int64_t share = (c + cluster - 1) / cluster;
  g.cs = (int)((share + 63) / 64 * 64);
  g.panels = g.cs / 64;
  g.a_panels = (g.p16 + 63) / 64;
  g.x_bytes = g.panels * g.p16 * 128;
  g.a_bytes = g.a_panels * g.p16 * 128;
  g.red_bytes = cluster > 1 ? g.p16 * g.p16 * 4 : 0;
  // K steps of 16 to an accumulator: at least 4
  g.splits = g.panels >= 4 ? 4 : g.panels >= 2 ? 2 : 1;
  g.chunks = (g.cs + 127) / 128;
  const int cols = (g.splits > g.chunks ? g.splits : g.chunks) * g.p16;
  g.tmem_cols = 32;
  while (g.tmem_cols < cols) g.tmem_cols *= 2;
  // an operand's last rows: up to 128 of them from any 8-row group on; Apply reads a second
  // panel where there is one only
  const int over = 16 * 1024;
  const int need = 2 * g.x_bytes + 2 * g.a_bytes + (g.red_bytes > over ? g.red_bytes : over) +
                   1024 /*barrier, sums*/ + 1024 /*align*/;
  // A CTA must never wait for another's Tensor Memory: clusters of two launches could then
  // wait for one another.  So each takes at least its columns' share of the SM's 228 KB (1 KB
  // of them the system's), and CTAs that fit together have their columns too.
  const int least = g.tmem_cols * (228 * 1024 / 512) - 1024;
  g.smem = need > least ? need : least;
  return g;
}

struct Shared {
  uint64_t done;
  uint32_t tmem_base;
  float warp_sum[kThreads / 32];
  float cta_sum;
};

// byte offset of element (row, col) in panels of `rows` rows, 128-byte swizzle
__device__ __forceinline__ int swizzled(int rows, int row, int col) {
  return (col >> 6) * rows * 128 + row * 128 + ((((col >> 3) & 7) ^ (row & 7)) << 4) + (col & 7) * 2;
}

__device__ __forceinline__ uint64_t sdesc(uint32_t saddr, uint32_t leading) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>((leading >> 4) & 0x3FFFu) << 16;
  d |= static_cast<uint64_t>(1024u >> 4) << 32;
  d |= static_cast<uint64_t>(1u) << 46;
  d |= static_cast<uint64_t>(2u) << 61;
  return d;
}
constexpr uint32_t kMnMajorA = 1u << 15;

__device__ __forceinline__ void tmem_ld_x8(uint32_t taddr, uint32_t (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]),
                 "=r"(v[6]), "=r"(v[7])
               : "r"(taddr));
}
__device__ __forceinline__ float f16(const uint8_t* p) {
  return __half2float(*reinterpret_cast<const __half*>(p));
}
__device__ __forceinline__ void split(float x, uint16_t& hi, uint16_t& lo) {
  const __half h = __float2half_rn(x);
  const __half l = __float2half_rn(x - __half2float(h));
  hi = __half_as_ushort(h);
  lo = __half_as_ushort(l);
}
__device__ __forceinline__ float element(const void* p, int bf16, int64_t at) {
  return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at])
              : static_cast<const float*>(p)[at];
}

struct Steps {
  OrthoStep s[kOrthoMaxSteps];
  int n;
};

__global__ void __launch_bounds__(kThreads)
ortho_small_kernel(const OrthoMat* __restrict__ mats, const int* __restrict__ which, int cluster,
                   const __grid_constant__ Steps steps, const OrthoUpdate u,
                   uint32_t* __restrict__ status) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  const OrthoMat mt = mats[which[blockIdx.x / cluster]];
  const int rank = (int)(blockIdx.x % cluster);
  const int p = (int)mt.p;
  const Geometry geo = geometry(p, mt.c, cluster);
  const int p16 = geo.p16;
  uint8_t* xh = smem + 1024;
  uint8_t* xl = xh + geo.x_bytes;
  uint8_t* ah = xl + geo.x_bytes;
  uint8_t* al = ah + geo.a_bytes;
  float* red = reinterpret_cast<float*>(al + geo.a_bytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t c0 = (int64_t)rank * geo.cs;
  const int cols = (int)max((int64_t)0, min((int64_t)geo.cs, mt.c - c0));   // of this CTA

  if (tid == 0) {
    mbar_init(&sh.done, 1);
    fence_mbar_init();
  }
  if (warp == 0) {
    tmem_alloc(&sh.tmem_base, (uint32_t)geo.tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;
  pdl_wait();
  pdl_trigger();

  // ---------------------------------------------------------------- U and its norm
  // element e of this CTA's share: (row i, column j) with the caller's rows contiguous
  const int n_el = p * cols;
  const auto place = [&](int e, int& i, int& j) {
    if (mt.tall) { j = e / p; i = e - j * p; }
    else { i = e / cols; j = e - i * cols; }
  };
  const auto update_of = [&](int i, int j, bool write) {
    const int64_t r = mt.tall ? c0 + j : i, c = mt.tall ? i : c0 + j;
    const float g = element(mt.G, mt.grad_bf16, r * mt.ldg + c);
    if (!u.step || mt.M == nullptr) return g;
    float* m = mt.M + r * mt.n + c;
    float mom = *m;
    if (write) {
      mom = fmaf(u.momentum, mom, g);
      *m = mom;
    }
    return u.nesterov ? fmaf(u.momentum, mom, g) : mom;
  };
  float sq = 0.0f;
#pragma unroll 4
  for (int e = tid; e < n_el; e += kThreads) {
    int i, j;
    place(e, i, j);
    const float v = update_of(i, j, true);
    sq = fmaf(v, v, sq);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
  if (lane == 0) sh.warp_sum[warp] = sq;
  // zero both parts of X: the padding rows and columns stay so
  for (int b = tid * 16; b < 2 * geo.x_bytes; b += kThreads * 16)
    *reinterpret_cast<uint4*>(xh + b) = make_uint4(0, 0, 0, 0);
  __syncthreads();
  sq = 0.0f;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) sq += sh.warp_sum[w];
  double total = (double)sq;
  if (cluster > 1) {
    if (tid == 0) sh.cta_sum = sq;
    cta2::cluster_sync_all();
    total = 0.0;
    for (int r = 0; r < cluster; ++r) {
      float v;
      asm volatile("ld.shared::cluster.f32 %0, [%1];"
                   : "=f"(v) : "r"(cta2::map_to(&sh.cta_sum, (uint32_t)r)) : "memory");
      total += (double)v;
    }
  }
  const float norm = (float)sqrt(total) + u.eps;
  const float inv = norm == 0.0f ? 0.0f : exp2i(steps.s[0].ex) / norm;
#pragma unroll 4
  for (int e = tid; e < n_el; e += kThreads) {
    int i, j;
    place(e, i, j);
    uint16_t hi, lo;
    split(update_of(i, j, false) * inv, hi, lo);
    const int at = swizzled(p16, i, j);
    *reinterpret_cast<uint16_t*>(xh + at) = hi;
    *reinterpret_cast<uint16_t*>(xl + at) = lo;
  }

  // ---------------------------------------------------------------- the steps
  const uint32_t idesc = idesc_f16_f32(128, p16);
  uint32_t parity = 0;
  const auto before_mma = [&]() {              // every thread's shared-memory writes are done
    fence_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
  };
  const auto wait_mma = [&]() {
    if (!mbar_wait_bounded(&sh.done, parity, nullptr, kWait) && lane == 0) atomicOr(status, 1u);
    parity ^= 1u;
    __syncwarp();
    tc_fence_after();
  };
  const int g4 = warp & 3, half = warp >> 2;   // TMEM lane group; half of the columns
  const uint32_t lanes = (uint32_t)(32 * g4) << 16;
  const int row = 32 * g4 + lane;
  const uint32_t xh_s = smem_u32(xh), xl_s = smem_u32(xl), ah_s = smem_u32(ah), al_s = smem_u32(al);

  for (int k = 0; k < steps.n; ++k) {
    const OrthoStep st = steps.s[k];
    // ---- A = X X^T over this CTA's columns
    before_mma();
    if (tid == 0) {
      const int per = (geo.panels + geo.splits - 1) / geo.splits;
      for (int s = 0; s < geo.splits; ++s)
        for (int prod = 0; prod < 3; ++prod) {
          const uint32_t a = prod == 1 ? xl_s : xh_s, b = prod == 0 ? xl_s : xh_s;
          for (int q = s * per; q < min(geo.panels, (s + 1) * per); ++q)
            for (int kk = 0; kk < 4; ++kk) {
              const uint32_t off = (uint32_t)(q * p16 * 128 + 32 * kk);
              mma_f16(tmem + (uint32_t)(s * p16), sdesc(a + off, 16), sdesc(b + off, 16), idesc,
                      (prod > 0 || q > s * per || kk > 0) ? 1u : 0u);
            }
        }
      mma_commit(&sh.done);
    }
    wait_mma();
    const float sa = exp2i(st.ea - 2 * st.ex);
    if (32 * g4 < p16) {
      for (int j = half * (p16 / 2); j < (half + 1) * (p16 / 2); j += 8) {
        uint32_t r[8];
        float v[8];
        tmem_ld_x8(tmem + lanes + (uint32_t)j, r);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(r[e]);
        const int per = (geo.panels + geo.splits - 1) / geo.splits;
        for (int s = 1; s < geo.splits && s * per < geo.panels; ++s) {
          tmem_ld_x8(tmem + lanes + (uint32_t)(s * p16 + j), r);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += __uint_as_float(r[e]);
        }
        if (row < p16) {
          if (cluster > 1) {
            float* to = red + row * p16 + j;
            *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(to + 4) = make_float4(v[4], v[5], v[6], v[7]);
          } else {
            uint4 hi, lo;
            tc::split8_f16(v, sa, hi, lo);
            const int at = swizzled(p16, row, j);
            *reinterpret_cast<uint4*>(ah + at) = hi;
            *reinterpret_cast<uint4*>(al + at) = lo;
          }
        }
        __syncwarp();
      }
    }
    if (cluster > 1) {
      // CTA r sums the 8-column pieces r, r + C, ... in rank order and writes them to all
      cta2::cluster_sync_all();
      const int pieces = p16 * p16 / 8;
      for (int q = rank + cluster * tid; q < pieces; q += cluster * kThreads) {
        const int i = q / (p16 / 8), j = q % (p16 / 8) * 8;
        float v[8] = {};
        for (int r = 0; r < cluster; ++r) {
          const uint32_t from = cta2::map_to(red + i * p16 + j, (uint32_t)r);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float4 f;
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w) : "r"(from + 16 * h) : "memory");
            v[4 * h] += f.x; v[4 * h + 1] += f.y; v[4 * h + 2] += f.z; v[4 * h + 3] += f.w;
          }
        }
        uint4 hi, lo;
        tc::split8_f16(v, sa, hi, lo);
        const int at = swizzled(p16, i, j);
        for (int r = 0; r < cluster; ++r) {
          asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                           cta2::map_to(ah + at, (uint32_t)r)),
                       "r"(hi.x), "r"(hi.y), "r"(hi.z), "r"(hi.w) : "memory");
          asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                           cta2::map_to(al + at, (uint32_t)r)),
                       "r"(lo.x), "r"(lo.y), "r"(lo.z), "r"(lo.w) : "memory");
        }
      }
      asm volatile("fence.proxy.async;" ::: "memory");
      cta2::cluster_sync_all();
    }
    // ---- B = b A + c A A, in A's place
    before_mma();
    if (tid == 0) {
      for (int prod = 0; prod < 3; ++prod) {
        const uint32_t a = prod == 1 ? al_s : ah_s, b = prod == 0 ? al_s : ah_s;
        for (int kk = 0; kk < p16 / 16; ++kk) {
          const uint32_t off = (uint32_t)((kk / 4) * p16 * 128 + 32 * (kk % 4));
          mma_f16(tmem, sdesc(a + off, 16), sdesc(b + off, 16), idesc, (prod > 0 || kk > 0) ? 1u : 0u);
        }
      }
      mma_commit(&sh.done);
    }
    wait_mma();
    if (32 * g4 < p16) {
      const float s0 = st.b * exp2i(st.eb - st.ea), s1 = st.c * exp2i(st.eb - 2 * st.ea);
      for (int j = half * (p16 / 2); j < (half + 1) * (p16 / 2); j += 8) {
        uint32_t r[8];
        tmem_ld_x8(tmem + lanes + (uint32_t)j, r);
        tmem_ld_wait();
        if (row < p16) {
          const int at = swizzled(p16, row, j);
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            v[e] = fmaf(s0, f16(ah + at + 2 * e) + f16(al + at + 2 * e), s1 * __uint_as_float(r[e]));
          uint4 hi, lo;
          tc::split8_f16(v, 1.0f, hi, lo);
          *reinterpret_cast<uint4*>(ah + at) = hi;
          *reinterpret_cast<uint4*>(al + at) = lo;
        }
        __syncwarp();
      }
    }
    // ---- X'^T = a X^T + X^T B, 128 columns of X at a time
    before_mma();
    if (tid == 0) {
      const uint32_t panel = (uint32_t)(p16 * 128);
      for (int q = 0; q < geo.chunks; ++q)
        for (int prod = 0; prod < 3; ++prod) {
          const uint32_t a = (prod == 1 ? xl_s : xh_s) + 2 * q * panel;
          const uint32_t b = prod == 0 ? al_s : ah_s;
          for (int kk = 0; kk < p16 / 16; ++kk) {
            const uint32_t off = (uint32_t)((kk / 4) * p16 * 128 + 32 * (kk % 4));
            mma_f16(tmem + (uint32_t)(q * p16), sdesc(a + 2048 * kk, panel), sdesc(b + off, 16),
                    idesc | kMnMajorA, (prod > 0 || kk > 0) ? 1u : 0u);
          }
        }
      mma_commit(&sh.done);
    }
    wait_mma();
    const float s0 = st.a * exp2i(st.last ? -st.ex : st.ex_next - st.ex);
    const float s1 = exp2i((st.last ? 0 : st.ex_next) - st.ex - st.eb);
    const float fm = (float)mt.m, fn = (float)mt.n;
    const float rate = u.lr * (u.adjust == 1 ? sqrtf(fmaxf(1.0f, fm / fn))
                               : u.adjust == 2 ? 0.2f * sqrtf(fmaxf(fm, fn)) : 1.0f);
    for (int q = 0; q < geo.chunks; ++q) {
      const int j = 128 * q + row;             // this thread's column of X
      for (int i0 = half * (p16 / 2); i0 < (half + 1) * (p16 / 2); i0 += 8) {
        uint32_t r[8];
        tmem_ld_x8(tmem + lanes + (uint32_t)(q * p16 + i0), r);
        tmem_ld_wait();
        if (j < cols) {
          float v[8], old[8];
          int64_t w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int at = swizzled(p16, i0 + e, j);
            v[e] = fmaf(s0, f16(xh + at) + f16(xl + at), s1 * __uint_as_float(r[e]));
          }
          if (!st.last) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int at = swizzled(p16, i0 + e, j);
              uint16_t hi, lo;
              split(v[e], hi, lo);
              *reinterpret_cast<uint16_t*>(xh + at) = hi;
              *reinterpret_cast<uint16_t*>(xl + at) = lo;
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int64_t i = i0 + e;
              w[e] = mt.tall ? (c0 + j) * mt.ldw + i : i * mt.ldw + c0 + j;
              old[e] = u.step && i < p ? element(mt.W, mt.bf16, w[e]) : 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              if (i0 + e >= p) continue;
              const float o = u.step ? fmaf(-rate, v[e], u.keep * old[e]) : v[e];
              if (mt.bf16) static_cast<__nv_bfloat16*>(mt.W)[w[e]] = __float2bfloat16_rn(o);
              else static_cast<float*>(mt.W)[w[e]] = o;
            }
          }
        }
        __syncwarp();
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, (uint32_t)geo.tmem_cols);
  }
}

}  // namespace

int32_t ortho_small_cluster(int64_t p, int64_t c) {
  if (p > 128) return 0;
  for (int cl = 1; cl <= kMaxCluster; cl *= 2) {
    // a CTA's columns: at most 256 where the cluster can still grow
    if (cl < kMaxCluster && c > 256 * (int64_t)cl) continue;
    if (c > (int64_t)cl * 8192) return 0;
    const Geometry g = geometry((int)p, c, cl);
    if (g.smem <= kSmemMax && g.tmem_cols <= 512) return cl;
  }
  return 0;
}
int32_t ortho_small_smem(int64_t p, int64_t c, int32_t cluster) {
  return geometry((int)p, c, cluster).smem;
}

cudaError_t launch_ortho_small(const OrthoMat* mats, const int* which, int32_t n, int32_t cluster,
                               int32_t smem, const OrthoStep* steps, int32_t n_steps,
                               const OrthoUpdate& u, uint32_t* status, cudaStream_t s) {
  if (n <= 0) return cudaSuccess;
  if (n_steps > kOrthoMaxSteps || smem > kSmemMax) return cudaErrorInvalidValue;
  cudaError_t e = cudaFuncSetAttribute(ortho_small_kernel,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax);
  if (e != cudaSuccess) return e;
  Steps st{};
  st.n = n_steps;
  std::copy(steps, steps + n_steps, st.s);
  return launch_dependent(ortho_small_kernel, (unsigned)n * (unsigned)cluster, kThreads,
                          (size_t)smem, s, (unsigned)cluster, true, mats, which, cluster, st, u,
                          status);
}

}  // namespace zo
