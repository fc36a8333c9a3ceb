// Newton-Schulz orthogonalisation of matrices of 65 to 128 rows in one launch: momentum, norm,
// every step and the update of W, with X in shared memory throughout.  (At most 64 rows:
// zo_ortho_mma.cu.)
//
// A matrix is a cluster of C CTAs, each with X's columns [rank cs, rank cs + cs).  A step:
//   Gram   each CTA's X X^T on its columns, summed over the cluster through distributed
//          shared memory (CTA r sums its share of the elements and writes them into every CTA);
//   Poly   B = b A + c A A, by every CTA for itself;
//   Apply  the columns' X' = a X + B X.
// All three are M = 128 tcgen05.mma on fp16 hi + lo pairs (hi.lo, lo.hi, then hi.hi), fp32
// accumulators.  X lies in shared memory once, as 128-byte swizzled panels of 64 columns: the
// Gram product reads them as a K-major operand, Apply as an MN-major one.  Rows are padded
// with zeros to a multiple of 16; where an operand has fewer than an MMA's 128 rows, the
// rest of it is whatever follows in shared memory, and those rows of the result are not read.
// One accumulator a product: dealing the K steps to four in turn took the MMAs of 128 x 128 no
// less time, and adding them up in the epilogues doubled a step's (75 K cycles for five steps,
// 187 K with four).  The small products come first, so that few of the sums that the tensor
// cores round towards zero (zo_ortho_gemm.cu) are large ones: errors of 0.5 to 1.25 times an fp32
// evaluation's for gradients, up to 2 times for Gaussian matrices of 70 rows (70 x 1000: 3.4e-6).
// Gram's hi.hi in an accumulator for every 64 columns left 3.3e-6 there, at 4% of the time.
// Between load and scaling, and between the last step and the update of W, the two fp16 planes
// of X hold the upper and lower halves of fp32 values, so that the caller's matrices are read
// and written once, in their own order.
//
// Bound by latency and the epilogues: a product's MMAs take 1.9-2.1 K cycles and its epilogue
// 1.3-2.2 K, about half of that at shared memory's rate, one after the other.  224 matrices of
// 128 x 128 fp32: 74 us, two waves of a CTA per SM; one matrix 36 us.
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "zo_cluster.cuh"
#include "zo_launch.cuh"
#include "zo_ops.h"
#include "zo_ortho_io.cuh"
#include "zo_sm100.cuh"
#include "zo_tc_common.cuh"

namespace zo {
namespace {

using namespace sm100;
using ortho::first_of;
using ortho::lower2;
using ortho::second_of;
using ortho::upper2;
using tc::exp2i;

constexpr int kMaxCluster = 8;
constexpr long long kWait = 4000000000LL;               // ~2 s at 2 GHz
constexpr int kSmemMax = 227 * 1024;

struct Geometry {
  int p16, cs, panels;            // padded rows; columns of a CTA; 64-column panels of X
  int a_panels;                   // 64-column panels of A
  int x_bytes, a_bytes;           // of a hi (or lo) part
  int red_bytes;                  // the cluster's partial Gram sums
  int tmem_cols;                  // an accumulator: p16 columns, or in Apply cs
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
  // (16 bytes past a row's end: a warp stores 32 rows' at once, each in its own banks)
  g.red_bytes = cluster > 1 ? g.p16 * (g.p16 + 4) * 4 : 0;
  // an operand's last rows: up to 128 of them from any 8-row group on
  const int over = 16 * 1024;
  const int need = 2 * g.x_bytes + 2 * g.a_bytes + (g.red_bytes > over ? g.red_bytes : over) +
                   1024 /*barrier, sums*/ + 1024 /*align*/;
  g.tmem_cols = 32;
  while (g.tmem_cols < g.p16 || g.tmem_cols < g.cs) g.tmem_cols *= 2;
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
  ortho::SumShared sums;
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
constexpr uint32_t kMnMajorB = 1u << 16;

__device__ __forceinline__ void tmem_ld_x8(uint32_t taddr, uint32_t (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]),
                 "=r"(v[6]), "=r"(v[7])
               : "r"(taddr));
}
// eight columns of an accumulator
__device__ __forceinline__ void sums8(uint32_t taddr, float (&v)[8]) {
  uint32_t r[8];
  tmem_ld_x8(taddr, r);
  tmem_ld_wait();
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(r[e]);
}
// hi + lo of eight neighbouring fp16 pairs
__device__ __forceinline__ void pairs8(const uint8_t* hi, const uint8_t* lo, float (&v)[8]) {
  const uint4 h = *reinterpret_cast<const uint4*>(hi), l = *reinterpret_cast<const uint4*>(lo);
  const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&hw[k]));
    const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&lw[k]));
    v[2 * k] = x.x + y.x;
    v[2 * k + 1] = x.y + y.y;
  }
}
struct Steps {
  OrthoStep s[kOrthoMaxSteps];
  int n;
};

template <int kThreads>
__global__ void __launch_bounds__(kThreads, 512 / kThreads)
ortho_small_kernel(const OrthoMat* __restrict__ mats, const int* __restrict__ which, int cluster,
                   const __grid_constant__ Steps steps, const OrthoUpdate u,
                   uint32_t* __restrict__ status) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  const OrthoMat mt = mats[which[blockIdx.x / cluster]];
  const int rank = (int)(blockIdx.x % cluster);
  const Geometry geo = geometry((int)mt.p, mt.c, cluster);
  const int p16 = geo.p16, cs = geo.cs;
  uint8_t* xh = smem + 1024;
  uint8_t* xl = xh + geo.x_bytes;
  uint8_t* ah = xl + geo.x_bytes;
  uint8_t* al = ah + geo.a_bytes;
  float* red = reinterpret_cast<float*>(al + geo.a_bytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t c0 = (int64_t)rank * cs;
  const int cols = (int)max((int64_t)0, min((int64_t)cs, mt.c - c0));   // of this CTA

  if (tid == 0) {
    mbar_init(&sh.done, 1);
    fence_mbar_init();
  }
  if (warp == 0) {
    tmem_alloc(&sh.tmem_base, (uint32_t)geo.tmem_cols);
    tmem_relinquish();
  }
  // both parts of X: the padding rows and columns stay zero
  for (int b = tid * 16; b < 2 * geo.x_bytes; b += kThreads * 16)
    *reinterpret_cast<uint4*>(xh + b) = make_uint4(0, 0, 0, 0);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;
  pdl_wait();
  pdl_trigger();

  // ---------------------------------------------------------------- U, scaled by its norm
  const auto put = [&](int i, int j, float v) {
    const int at = swizzled(p16, i, j);
    *reinterpret_cast<uint16_t*>(xh + at) = (uint16_t)(__float_as_uint(v) >> 16);
    *reinterpret_cast<uint16_t*>(xl + at) = (uint16_t)__float_as_uint(v);
  };
  const auto get = [&](int i, int j) {
    const int at = swizzled(p16, i, j);
    return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(xh + at) << 16 |
                           *reinterpret_cast<const uint16_t*>(xl + at));
  };
  const int64_t n = mt.tall ? mt.p : cols;
  float sq;
  if (ortho::by_fours(mt.G, mt.ldg, mt.grad_bf16, n) &&
      (mt.M == nullptr || !u.step || ortho::by_fours(mt.M, mt.n, 0, n))) {
    sq = ortho::load_update<kThreads, 4>(mt, u, c0, cols, [&](int i, int j, const float (&v)[4]) {
      if (mt.tall) {
#pragma unroll
        for (int e = 0; e < 4; ++e) put(i + e, j, v[e]);
      } else {
        const int at = swizzled(p16, i, j);
        *reinterpret_cast<uint2*>(xh + at) = make_uint2(upper2(v[0], v[1]), upper2(v[2], v[3]));
        *reinterpret_cast<uint2*>(xl + at) = make_uint2(lower2(v[0], v[1]), lower2(v[2], v[3]));
      }
    });
  } else {
    sq = ortho::load_update<kThreads, 1>(mt, u, c0, cols,
                                         [&](int i, int j, const float (&v)[1]) { put(i, j, v[0]); });
  }
  const ortho::Planes planes{reinterpret_cast<uint4*>(xh), reinterpret_cast<uint4*>(xl), geo.x_bytes / 16};
  const float inv = ortho::inverse_norm<kThreads>(sq, u.eps, cluster, sh.sums, planes);
  const float s_in = exp2i(steps.s[0].ex);
  for (int b = tid * 16; b < geo.x_bytes; b += kThreads * 16) {
    uint4* ph = reinterpret_cast<uint4*>(xh + b);
    uint4* pl = reinterpret_cast<uint4*>(xl + b);
    const uint4 h = *ph, l = *pl;
    const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
    float v[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = first_of(hw[k], lw[k]) * inv;
      v[2 * k + 1] = second_of(hw[k], lw[k]) * inv;
    }
    tc::split8_f16(v, s_in, *ph, *pl);
  }

  // ---------------------------------------------------------------- the steps
  uint32_t parity = 0;
  const auto before_mma = [&]() {              // every thread's shared-memory writes are done
    fence_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
  };
  const auto wait_mma = [&]() {
    __syncwarp();
    if (!mbar_wait_bounded(&sh.done, parity, nullptr, kWait) && lane == 0) atomicOr(status, 1u);
    parity ^= 1u;
    __syncwarp();
    tc_fence_after();
  };
  constexpr int kGroups = kThreads / 128;      // warps that share a TMEM lane group
  const int g4 = warp & 3, group = warp >> 2;
  const uint32_t lanes = (uint32_t)(32 * g4) << 16;
  const int row = 32 * g4 + lane;
  const bool active = 32 * g4 < p16;           // (a whole warp)
  const uint32_t xh_s = smem_u32(xh), xl_s = smem_u32(xl), ah_s = smem_u32(ah), al_s = smem_u32(al);
  const uint32_t panel = (uint32_t)(p16 * 128);
  const auto k_major = [&](int s) { return (uint32_t)(s >> 2) * panel + 32u * (uint32_t)(s & 3); };
  const auto mn_major = [&](int s) { return 2048u * (uint32_t)s; };
  // D = sum over K steps of A B^T: K step s of 16 lies at step(s) of either operand's bytes
  const auto product = [&](int n_k, uint32_t idesc, uint32_t hi_a, uint32_t lo_a, uint32_t hi_b,
                           uint32_t lo_b, auto step_b, uint32_t lead_b, uint32_t col) {
    for (int prod = 0; prod < 3; ++prod) {
      const uint32_t a = prod == 1 ? lo_a : hi_a, b = prod == 0 ? lo_b : hi_b;
      for (int s = 0; s < n_k; ++s)
        mma_f16(tmem + col, sdesc(a + k_major(s), 16), sdesc(b + step_b(s), lead_b), idesc,
                prod > 0 || s > 0 ? 1u : 0u);
    }
  };
  const uint32_t idesc_sym = idesc_f16_f32(128, p16);

  for (int k = 0; k < steps.n; ++k) {
    const OrthoStep st = steps.s[k];
    // ---- A = X X^T over this CTA's columns
    before_mma();
    if (warp == 0 && ortho::elected()) {
      product(4 * geo.panels, idesc_sym, xh_s, xl_s, xh_s, xl_s, k_major, 16, 0);
      mma_commit(&sh.done);
    }
    wait_mma();
    const float sa = exp2i(st.ea - 2 * st.ex);
    if (active) {
      for (int j = 8 * group; j < p16; j += 8 * kGroups) {
        float v[8];
        sums8(tmem + lanes + (uint32_t)j, v);
        if (row < p16) {
          if (cluster > 1) {
            float* to = red + row * (p16 + 4) + j;
            *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(to + 4) = make_float4(v[4], v[5], v[6], v[7]);
          } else {
            const int at = swizzled(p16, row, j);
            tc::split8_f16(v, sa, *reinterpret_cast<uint4*>(ah + at), *reinterpret_cast<uint4*>(al + at));
          }
        }
        __syncwarp();
      }
    }
    if (cluster > 1) {
      // CTA r sums its run of the 8-column pieces in rank order and writes them to all.  A warp's
      // pieces are neighbours: dealt out one at a time, 128 x 1000 took 117 us instead of 79.
      cta2::cluster_sync_all();
      const int pieces = p16 * p16 / 8, share = (pieces + cluster - 1) / cluster;
      const int q_end = min(pieces, (rank + 1) * share);
      for (int q = rank * share + tid; q < q_end; q += kThreads) {
        const int i = q / (p16 / 8), j = q % (p16 / 8) * 8;
        float v[8] = {};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float4 f[kMaxCluster];
#pragma unroll
          for (int r = 0; r < kMaxCluster; ++r)
            if (r < cluster)
              asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                           : "=f"(f[r].x), "=f"(f[r].y), "=f"(f[r].z), "=f"(f[r].w)
                           : "r"(cta2::map_to(red + i * (p16 + 4) + j + 4 * half, (uint32_t)r))
                           : "memory");
#pragma unroll
          for (int r = 0; r < kMaxCluster; ++r)
            if (r < cluster) {
              v[4 * half] += f[r].x; v[4 * half + 1] += f[r].y;
              v[4 * half + 2] += f[r].z; v[4 * half + 3] += f[r].w;
            }
        }
        uint4 hi, lo;
        tc::split8_f16(v, sa, hi, lo);
        const int at = swizzled(p16, i, j);
        for (int r = 0; r < cluster; ++r) {
          asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                           cta2::map_to(ah + at, (uint32_t)r)), "r"(hi.x), "r"(hi.y), "r"(hi.z), "r"(hi.w)
                       : "memory");
          asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                           cta2::map_to(al + at, (uint32_t)r)), "r"(lo.x), "r"(lo.y), "r"(lo.z), "r"(lo.w)
                       : "memory");
        }
      }
      asm volatile("fence.proxy.async;" ::: "memory");
      cta2::cluster_sync_all();
    }
    // ---- B = b A + c A A, in A's place
    before_mma();
    if (warp == 0 && ortho::elected()) {
      product(p16 / 16, idesc_sym, ah_s, al_s, ah_s, al_s, k_major, 16, 0);
      mma_commit(&sh.done);
    }
    wait_mma();
    if (active) {
      const float s0 = st.b * exp2i(st.eb - st.ea), s1 = st.c * exp2i(st.eb - 2 * st.ea);
      for (int j = 8 * group; j < p16; j += 8 * kGroups) {
        float v[8];
        sums8(tmem + lanes + (uint32_t)j, v);
        if (row < p16) {
          const int at = swizzled(p16, row, j);
          float x[8];
          pairs8(ah + at, al + at, x);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = fmaf(s0, x[e], s1 * v[e]);
          tc::split8_f16(v, 1.0f, *reinterpret_cast<uint4*>(ah + at), *reinterpret_cast<uint4*>(al + at));
        }
        __syncwarp();
      }
    }
    // ---- X' = a X + B X, at most 256 columns an MMA
    before_mma();
    if (warp == 0 && ortho::elected()) {
      for (int q = 0; q < geo.panels; q += 4) {
        const int width = 64 * min(4, geo.panels - q);
        product(p16 / 16, idesc_f16_f32(128, width) | kMnMajorB, ah_s, al_s, xh_s + q * panel,
                xl_s + q * panel, mn_major, panel, (uint32_t)(64 * q));
      }
      mma_commit(&sh.done);
    }
    wait_mma();
    if (active) {
      const float s0 = st.a * exp2i(st.last ? -st.ex : st.ex_next - st.ex);
      const float s1 = exp2i((st.last ? 0 : st.ex_next) - st.ex - st.eb);
      for (int j = 8 * group; j < cs; j += 8 * kGroups) {
        float v[8];
        sums8(tmem + lanes + (uint32_t)j, v);
        if (row < p16) {
          const int at = swizzled(p16, row, j);
          uint4* ph = reinterpret_cast<uint4*>(xh + at);
          uint4* pl = reinterpret_cast<uint4*>(xl + at);
          float x[8];
          pairs8(xh + at, xl + at, x);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = fmaf(s0, x[e], s1 * v[e]);
          if (st.last) {
            *ph = make_uint4(upper2(v[0], v[1]), upper2(v[2], v[3]), upper2(v[4], v[5]), upper2(v[6], v[7]));
            *pl = make_uint4(lower2(v[0], v[1]), lower2(v[2], v[3]), lower2(v[4], v[5]), lower2(v[6], v[7]));
          } else {
            tc::split8_f16(v, 1.0f, *ph, *pl);
          }
        }
        __syncwarp();
      }
    }
  }

  // ---------------------------------------------------------------- the result
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, (uint32_t)geo.tmem_cols);
  }
  if (ortho::by_fours(mt.W, mt.ldw, mt.bf16, n)) {
    ortho::store_result<kThreads, 4>(mt, u, c0, cols, [&](int i, int j, float (&v)[4]) {
      if (mt.tall) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = get(i + e, j);
      } else {
        const int at = swizzled(p16, i, j);
        const uint2 h = *reinterpret_cast<const uint2*>(xh + at);
        const uint2 l = *reinterpret_cast<const uint2*>(xl + at);
        v[0] = first_of(h.x, l.x);
        v[1] = second_of(h.x, l.x);
        v[2] = first_of(h.y, l.y);
        v[3] = second_of(h.y, l.y);
      }
    });
  } else {
    ortho::store_result<kThreads, 1>(mt, u, c0, cols,
                                     [&](int i, int j, float (&v)[1]) { v[0] = get(i, j); });
  }
}

template <int kThreads>
cudaError_t launch(const OrthoMat* mats, const int* which, int32_t n, int32_t cluster, int32_t smem,
                   const Steps& st, const OrthoUpdate& u, uint32_t* status, cudaStream_t s) {
  const cudaError_t e = cudaFuncSetAttribute(ortho_small_kernel<kThreads>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax);
  if (e != cudaSuccess) return e;
  return launch_dependent(ortho_small_kernel<kThreads>, (unsigned)n * (unsigned)cluster, kThreads,
                          (size_t)smem, s, (unsigned)cluster, true, mats, which, cluster, st, u,
                          status);
}

}  // namespace

int32_t ortho_small_cluster(int64_t p, int64_t c) {
  if (p <= 64 || p > 128) return 0;
  for (int cl = 1; cl <= kMaxCluster; cl *= 2) {
    // a CTA's columns: at most 256 where the cluster can still grow
    if (cl < kMaxCluster && c > 256 * (int64_t)cl) continue;
    if (c > 512 * (int64_t)cl) return 0;                 // a column of Tensor Memory each
    const Geometry g = geometry((int)p, c, cl);
    if (g.smem <= kSmemMax) return cl;
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
  Steps st{};
  st.n = n_steps;
  std::copy(steps, steps + n_steps, st.s);
  // sixteen warps for the epilogues where a CTA has its SM to itself
  return smem > 113 * 1024 ? launch<512>(mats, which, n, cluster, smem, st, u, status, s)
                           : launch<256>(mats, which, n, cluster, smem, st, u, status, s);
}

}  // namespace zo
