// Newton-Schulz orthogonalisation of matrices of at most 64 rows in one launch: momentum, norm,
// every step and the update of W, with X in shared memory throughout.
//
// A matrix is a cluster of C CTAs, each with its share of X's columns as a hi and a lo plane of
// fp16 values of x 2^e.  A step:
//   Gram   the CTA's X X^T: 16 rows of the result per warp, K dealt to the warps that are left;
//          their fp32 sums are added up in warp order, then over the cluster in rank order (every
//          CTA reads all the partial sums through distributed shared memory, so one cluster
//          barrier a step is enough);
//   Poly   B = b A + c A A, by every CTA for itself;
//   Apply  X' = a X + B X in place: a warp takes all rows of eight or sixteen columns.
// Products are hi.lo + lo.hi + hi.hi with fp32 sums (to 32 rows lo.lo too in Poly and Apply), by
// warp-wide m16n8k16 MMAs on registers: at these sizes a step is a chain of short latencies, and
// the round trip of a tcgen05.mma (issue, commit, wait, Tensor Memory to registers: ~2.5 K cycles
// a product at 64 x 64, against ~1 K here) would be most of it; from 65 rows on the larger MMAs
// win (zo_ortho_small.cu).
// An MMA's fp32 sum rounds towards zero, which few singular directions do not average out.  At 64
// rows hi.hi is therefore summed apart from the small products, 16 of K at a time, to nearest;
// at 16 rows so is X X^T, whose K is long.  Mean errors of sets so, and in one sum without lo.lo
// (fp32 evaluation): 112 of 64 x 64 7.2e-7, 1.31e-6 (1.19e-6); 30 of 64 x 256 1.32e-6, 2.56e-6
// (1.49e-6); 100 of 32 x 64 1.35e-6, 1.65e-6 (1.13e-6); 448 of 8 x 8 6.9e-7, 8.6e-7 (7.5e-7); 20 of
// 8 x 8000 7.5e-7, 1.43e-6 (8.3e-7).  It takes 8 to 11% of the time at 64 rows, 4% at 32, 1 to 4% at
// 16, and none where X is in registers.
// Between load and scaling, and between the last step and the update of W, the planes hold the
// upper and lower halves of fp32 values, so that the caller's matrices are read and written
// once, in their own order.
// Bound by the chain's latencies.  224 matrices of 32 x 32 fp32 9.8 us; Muon steps of forty 8 x
// 5120 26 us: five steps of 6 K cycles, half of them the cluster's sums, and 14 K of load, norm
// and store.
#include <algorithm>

#include <cuda_fp16.h>

#include "zo_launch.cuh"
#include "zo_ops.h"
#include "zo_ortho_io.cuh"
#include "zo_sm100.cuh"
#include "zo_tc_common.cuh"

namespace zo {
namespace {

using namespace ortho;
using sm100::smem_u32;
using tc::exp2i;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kSmemMax = 227 * 1024 - 1024;

__host__ __device__ constexpr int mma_rows(int64_t p) { return p <= 16 ? 16 : p <= 32 ? 32 : 64; }
// columns of a CTA, a multiple of 16, and the planes' row pitch in halves: 16 bytes past a
// multiple of 128, so that eight rows' 16 bytes lie in different banks
__host__ __device__ inline int mma_cols(int64_t c, int cluster) {
  return (int)(((c + cluster - 1) / cluster + 15) / 16 * 16);
}
__host__ __device__ constexpr int pitch_of(int cs) { return (cs + 63) / 64 * 64 + 8; }

template <int P>
struct Shape {
  static constexpr int kM = P / 16;                    // tiles of 16 rows
  static constexpr int kSplits = P == 16 ? 8 : P == 32 ? 4 : 1;   // of Gram's K
  static constexpr int kN = P == 64 ? P / 16 : P / 8;  // Gram: tiles of 8 columns per warp
  static constexpr int kPitch = P + 8;                 // of A, B (halves) and of sums (floats)
  static constexpr int kSumFloats = P * kPitch;
  static_assert(kM * kSplits * (P / 8 / kN) == kWarps, "a Gram task per warp");
  static __host__ __device__ int smem(int cs, int cluster) {
    return 2 * 2 * P * pitch_of(cs) + 4 * 2 * P * kPitch +
           4 * (kSplits + (cluster > 1 ? 2 : 0)) * kSumFloats;
  }
};

__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
// D += A B, m16n8k16, fp16 operands, fp32 sums
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// an 8 x 8 matrix of halves, a row's pair per lane, transposed
__device__ __forceinline__ uint32_t transposed(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ float2 pair2(const __half* hi, const __half* lo) {
  const float2 h = __half22float2(*reinterpret_cast<const __half2*>(hi));
  const float2 l = __half22float2(*reinterpret_cast<const __half2*>(lo));
  return make_float2(h.x + l.x, h.y + l.y);
}
__device__ __forceinline__ void split2(float a, float b, __half* hi, __half* lo) {
  const __half2 h = __floats2half2_rn(a, b);
  const float2 f = __half22float2(h);
  *reinterpret_cast<__half2*>(hi) = h;
  *reinterpret_cast<__half2*>(lo) = __floats2half2_rn(a - f.x, b - f.y);
}
struct Steps {
  OrthoStep s[kOrthoMaxSteps];
  int n;
};

// X' = a X + B X in kNb x 8 columns from j0 on, by one warp: X's columns are in registers
// before any of them is written, and the sums of all rows and columns run side by side (an MMA
// waits for the one before it on the same sums).  At 64 rows hi.hi comes after all the others, for
// which B_hi is read twice: its sums beside theirs would not fit the registers.
template <int P, int kNb>
__device__ __forceinline__ void apply(__half* xh, __half* xl, const __half* bh, const __half* bl,
                                      int pitch, int j0, float s0, float s1, bool last) {
  constexpr int kK = P / 16, kBp = Shape<P>::kPitch, kX = (kNb + 1) / 2;
  const int lane = threadIdx.x & 31;
  uint32_t x[2][kK][kX][4];                            // hi, lo; 16 rows x 16 columns each
#pragma unroll
  for (int k = 0; k < kK; ++k)
#pragma unroll
    for (int q = 0; q < kX; ++q) {
      // matrices: rows 16 k + 0..7 and + 8..15 of columns j.. and (kNb > 1) j + 8..
      const int at = (16 * k + (lane & 15)) * pitch + j0 + 16 * q + (kNb > 1 ? (lane >> 4) * 8 : 0);
      ldmatrix_x4_trans(x[0][k][q], smem_u32(xh + at));
      ldmatrix_x4_trans(x[1][k][q], smem_u32(xl + at));
    }
  const int own = (lane >> 2) * pitch + j0 + (lane & 3) * 2;     // of a sum's first two values
  float2 v[kK][kNb][2];
#pragma unroll
  for (int m = 0; m < kK; ++m)
#pragma unroll
    for (int n = 0; n < kNb; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = own + (16 * m + 8 * h) * pitch + 8 * n;
        v[m][n][h] = pair2(xh + at, xl + at);
      }
  float d[kK][kNb][4] = {};
#pragma unroll
  for (int k = 0; k < kK; ++k)
#pragma unroll
    for (int m = 0; m < kK; ++m) {
      uint32_t b[2][4];
      const int at = (16 * m + (lane & 15)) * kBp + 16 * k + (lane >> 4) * 8;
      ldmatrix_x4(b[0], smem_u32(bh + at));
      ldmatrix_x4(b[1], smem_u32(bl + at));
      if constexpr (P <= 32) {
#pragma unroll
        for (int n = 0; n < kNb; ++n)
          mma(d[m][n], b[1], x[1][k][n / 2][n % 2 * 2], x[1][k][n / 2][n % 2 * 2 + 1]);
      }
#pragma unroll
      for (int n = 0; n < kNb; ++n)
        mma(d[m][n], b[0], x[1][k][n / 2][n % 2 * 2], x[1][k][n / 2][n % 2 * 2 + 1]);
#pragma unroll
      for (int n = 0; n < kNb; ++n)
        mma(d[m][n], b[1], x[0][k][n / 2][n % 2 * 2], x[0][k][n / 2][n % 2 * 2 + 1]);
      if constexpr (P != 64) {
#pragma unroll
        for (int n = 0; n < kNb; ++n)
          mma(d[m][n], b[0], x[0][k][n / 2][n % 2 * 2], x[0][k][n / 2][n % 2 * 2 + 1]);
      }
    }
  if constexpr (P == 64) {
#pragma unroll
    for (int m = 0; m < kK; ++m)
#pragma unroll
      for (int k = 0; k < kK; ++k) {
        uint32_t b[4];
        ldmatrix_x4(b, smem_u32(bh + (16 * m + (lane & 15)) * kBp + 16 * k + (lane >> 4) * 8));
#pragma unroll
        for (int n = 0; n < kNb; ++n) {
          float g[4] = {};
          mma(g, b, x[0][k][n / 2][n % 2 * 2], x[0][k][n / 2][n % 2 * 2 + 1]);
#pragma unroll
          for (int e = 0; e < 4; ++e) d[m][n][e] += g[e];
        }
      }
  }
  __syncwarp();
#pragma unroll
  for (int m = 0; m < kK; ++m)
#pragma unroll
    for (int n = 0; n < kNb; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = own + (16 * m + 8 * h) * pitch + 8 * n;
        const float a = fmaf(s0, v[m][n][h].x, s1 * d[m][n][2 * h]);
        const float b = fmaf(s0, v[m][n][h].y, s1 * d[m][n][2 * h + 1]);
        if (last) {
          *reinterpret_cast<uint32_t*>(xh + at) = upper2(a, b);
          *reinterpret_cast<uint32_t*>(xl + at) = lower2(a, b);
        } else {
          split2(a, b, xh + at, xl + at);
        }
      }
}

// X of at most eight rows in registers: a warp's kTiles x 16 columns (tile warp + 8 i), as the A
// operand of X'^T = a X^T + X^T B: lane (g, t) holds rows 2 t, 2 t + 1 of columns g and g + 8.
// That is also how the product's sums lie, so Apply reads nothing but B; Gram's operands are the
// same 8 x 8 blocks transposed.  (Sixteen rows would take twice the registers: three CTAs an SM,
// 80 registers a thread, spilled and were slower than shared memory.  Five tiles, 5120 columns of
// a cluster of eight, are what the registers hold beside the rest: with eight, spills take 7% of
// 224 of 8 x 8 and 3% of forty 8 x 5120, 26.4 -> 27.3 us; forty 8 x 5136 would take 28 us there,
// 39 from shared memory.)
constexpr int kTiles = 5;
struct Columns {
  uint32_t hi[kTiles][2], lo[kTiles][2];
};
__device__ __forceinline__ int tile_col(int i) { return 16 * ((int)(threadIdx.x >> 5) + kWarps * i); }
// from the planes' fp32 values
__device__ __forceinline__ void take(Columns& x, const __half* xh, const __half* xl, int pitch, int cs,
                                     float inv, float scale) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    if (tile_col(i) >= cs) break;
    uint32_t up[4], low[4];                           // (rows 8 .. 15 are not used)
    const int at = (lane & 15) * pitch + tile_col(i) + (lane >> 4) * 8;
    ldmatrix_x4_trans(up, smem_u32(xh + at));
    ldmatrix_x4_trans(low, smem_u32(xl + at));
#pragma unroll
    for (int q = 0; q < 2; ++q)
      split2(first_of(up[2 * q], low[2 * q]) * inv * scale, second_of(up[2 * q], low[2 * q]) * inv * scale,
             reinterpret_cast<__half*>(&x.hi[i][q]), reinterpret_cast<__half*>(&x.lo[i][q]));
  }
}
// the warp's share of X X^T: hi above lo, eight rows each, so that an MMA is two products, and every
// 16 columns added up to nearest
__device__ __forceinline__ void gram(const Columns& x, int cs, float* to) {
  constexpr int kPitch = Shape<16>::kPitch;
  const int lane = threadIdx.x & 31;
  float2 small = make_float2(0.f, 0.f), large = small;
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    if (tile_col(i) >= cs) break;
    const uint32_t h0 = transposed(x.hi[i][0]), h1 = transposed(x.hi[i][1]);
    const uint32_t l0 = transposed(x.lo[i][0]), l1 = transposed(x.lo[i][1]);
    const uint32_t both[4] = {h0, l0, h1, l1};
    float p[4] = {}, q[4] = {};                       // hi.hi over lo.hi, hi.lo over lo.lo
    mma(p, both, h0, h1);
    mma(q, both, l0, l1);
    large.x += p[0];
    large.y += p[1];
    small.x += p[2] + (q[0] + q[2]);
    small.y += p[3] + (q[1] + q[3]);
  }
  const float2 v = make_float2(small.x + large.x, small.y + large.y);
  float* at = to + (lane >> 2) * kPitch + (lane & 3) * 2;
#pragma unroll
  for (int q = 0; q < 4; ++q)                         // the rest of 16 x 16 is zero
    *reinterpret_cast<float2*>(at + (q & 1) * 8 + (q >> 1) * 8 * kPitch) = q == 0 ? v : make_float2(0.f, 0.f);
}
// X' = a X + B X; the last step's fp32 values go to the planes
__device__ __forceinline__ void apply(Columns& x, int cs, const __half* bh, const __half* bl, __half* xh,
                                      __half* xl, int pitch, float s0, float s1, bool last) {
  const int lane = threadIdx.x & 31;
  const int own = (lane >> 2) * Shape<16>::kPitch + (lane & 3) * 2;
  const uint32_t b_hi = *reinterpret_cast<const uint32_t*>(bh + own);
  const uint32_t b_lo = *reinterpret_cast<const uint32_t*>(bl + own);
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    if (tile_col(i) >= cs) break;
    // hi beside lo: one MMA is (hi + lo) B_lo, the other (hi + lo) B_hi
    const uint32_t both[4] = {x.hi[i][0], x.hi[i][1], x.lo[i][0], x.lo[i][1]};
    float d[4] = {};
    mma(d, both, b_lo, b_lo);
    mma(d, both, b_hi, b_hi);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const float2 o = pair2(reinterpret_cast<const __half*>(&x.hi[i][q]),
                             reinterpret_cast<const __half*>(&x.lo[i][q]));
      const float v0 = fmaf(s0, o.x, s1 * d[2 * q]), v1 = fmaf(s0, o.y, s1 * d[2 * q + 1]);
      if (last) {
        const int at = (lane >> 2) * pitch + tile_col(i) + 8 * q + (lane & 3) * 2;
        *reinterpret_cast<uint32_t*>(xh + at) = transposed(upper2(v0, v1));
        *reinterpret_cast<uint32_t*>(xl + at) = transposed(lower2(v0, v1));
      } else {
        split2(v0, v1, reinterpret_cast<__half*>(&x.hi[i][q]), reinterpret_cast<__half*>(&x.lo[i][q]));
      }
    }
  }
}

template <int P>
__global__ void __launch_bounds__(kThreads, P == 16 ? 3 : 2)
ortho_mma_kernel(const OrthoMat* __restrict__ mats, const int* __restrict__ which, int cluster,
                 const __grid_constant__ Steps steps, const OrthoUpdate u) {
  using S = Shape<P>;
  constexpr int kPitch = S::kPitch;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ SumShared sums;
  const OrthoMat mt = mats[which[blockIdx.x / cluster]];
  const int rank = (int)(blockIdx.x % cluster);
  const int cs = mma_cols(mt.c, cluster), pitch = pitch_of(cs);
  __half* xh = reinterpret_cast<__half*>(smem);
  __half* xl = xh + P * pitch;
  __half* ah = xl + P * pitch;
  __half* al = ah + P * kPitch;
  __half* bh = al + P * kPitch;
  __half* bl = bh + P * kPitch;
  float* part = reinterpret_cast<float*>(bl + P * kPitch);
  float* red = part + S::kSplits * S::kSumFloats;      // two of them, for a cluster's sums
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t c0 = (int64_t)rank * cs;
  const int cols = (int)max((int64_t)0, min((int64_t)cs, mt.c - c0));

  // both planes: the padding rows and columns stay zero
  for (int e = tid; e < 2 * P * pitch / 8; e += kThreads)
    reinterpret_cast<uint4*>(xh)[e] = make_uint4(0, 0, 0, 0);
  __syncthreads();
  pdl_wait();
  pdl_trigger();

  // ---------------------------------------------------------------- U, scaled by its norm
  const auto put = [&](int i, int j, float v) {
    reinterpret_cast<uint16_t*>(xh)[i * pitch + j] = (uint16_t)(__float_as_uint(v) >> 16);
    reinterpret_cast<uint16_t*>(xl)[i * pitch + j] = (uint16_t)__float_as_uint(v);
  };
  const auto get = [&](int i, int j) {
    return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(xh)[i * pitch + j] << 16 |
                           reinterpret_cast<const uint16_t*>(xl)[i * pitch + j]);
  };
  const int64_t n = mt.tall ? mt.p : cols;
  float sq;
  if (by_fours(mt.G, mt.ldg, mt.grad_bf16, n) &&
      (mt.M == nullptr || !u.step || by_fours(mt.M, mt.n, 0, n))) {
    sq = load_update<kThreads, 4>(mt, u, c0, cols, [&](int i, int j, const float (&v)[4]) {
      if (mt.tall) {
#pragma unroll
        for (int e = 0; e < 4; ++e) put(i + e, j, v[e]);
      } else {
        *reinterpret_cast<uint2*>(xh + i * pitch + j) = make_uint2(upper2(v[0], v[1]), upper2(v[2], v[3]));
        *reinterpret_cast<uint2*>(xl + i * pitch + j) = make_uint2(lower2(v[0], v[1]), lower2(v[2], v[3]));
      }
    });
  } else {
    sq = load_update<kThreads, 1>(mt, u, c0, cols,
                                  [&](int i, int j, const float (&v)[1]) { put(i, j, v[0]); });
  }
  const Planes planes{reinterpret_cast<uint4*>(xh), reinterpret_cast<uint4*>(xl), P * pitch / 8};
  const float inv = inverse_norm<kThreads>(sq, u.eps, cluster, sums, planes);
  const float s_in = exp2i(steps.s[0].ex);
  const bool in_registers = P == 16 && mt.p <= 8 && cs <= 16 * kTiles * kWarps;
  Columns x;
  if (in_registers) {
    take(x, xh, xl, pitch, cs, inv, s_in);
  } else {
    for (int e = tid; e < P * pitch / 8; e += kThreads) {
      uint4* ph = reinterpret_cast<uint4*>(xh) + e;
      uint4* pl = reinterpret_cast<uint4*>(xl) + e;
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
    __syncthreads();
  }

  // ---------------------------------------------------------------- the steps
  const int row = lane >> 2, col = (lane & 3) * 2;     // of a sum's first two values
  for (int k = 0; k < steps.n; ++k) {
    const OrthoStep st = steps.s[k];
    if (in_registers) {
      gram(x, cs, part + warp * S::kSumFloats);
    } else {
      // ---- X X^T: rows 16 m, columns 8 (kN n0 ..), K tiles split, split + kSplits, ...
      const int m = warp % S::kM, split = warp / S::kM % S::kSplits, n0 = warp / (S::kM * S::kSplits) * S::kN;
      // hi.hi of 16 columns at a time is added up here, to nearest; not at 32 rows, where K is dealt
      // to four warps and that took 6% of the time for a tenth of the error.  (lo.lo made no
      // difference to the error.)
      constexpr bool kNearest = P != 32;
      float d[S::kN][4] = {}, small[kNearest ? S::kN : 1][4] = {};
      for (int kt = split; kt < cs / 16; kt += S::kSplits) {
        uint32_t a[2][4];
        const int at = (16 * m + (lane & 15)) * pitch + 16 * kt + (lane >> 4) * 8;
        ldmatrix_x4(a[0], smem_u32(xh + at));
        ldmatrix_x4(a[1], smem_u32(xl + at));
#pragma unroll
        for (int q = 0; q < S::kN; q += 2) {           // two tiles of 8 columns: 16 rows of X
          uint32_t b[2][4];
          const int bt = (8 * (n0 + q) + (lane & 15)) * pitch + 16 * kt + (lane >> 4) * 8;
          ldmatrix_x4(b[0], smem_u32(xh + bt));
          ldmatrix_x4(b[1], smem_u32(xl + bt));
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if constexpr (kNearest) {
              float large[4] = {};
              mma(small[q + h], a[0], b[1][h], b[1][h + 2]);
              mma(large, a[0], b[0][h], b[0][h + 2]);
              mma(small[q + h], a[1], b[0][h], b[0][h + 2]);
#pragma unroll
              for (int e = 0; e < 4; ++e) d[q + h][e] += large[e];
            } else {
              mma(d[q + h], a[0], b[1][h], b[1][h + 2]);
              mma(d[q + h], a[1], b[0][h], b[0][h + 2]);
              mma(d[q + h], a[0], b[0][h], b[0][h + 2]);
            }
          }
        }
      }
      if constexpr (kNearest) {
#pragma unroll
        for (int q = 0; q < S::kN; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e) d[q][e] += small[q][e];
      }
      float* to = part + split * S::kSumFloats;
#pragma unroll
      for (int q = 0; q < S::kN; ++q)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<float2*>(to + (16 * m + row + 8 * h) * kPitch + 8 * (n0 + q) + col) =
              make_float2(d[q][2 * h], d[q][2 * h + 1]);
    }
    __syncthreads();
    // the partial sums alternate between two buffers: those of the step before the last have
    // been read by every CTA once the last step's barrier is passed
    float* mine = red + (k & 1) * S::kSumFloats;
    const float sa = exp2i(st.ea - 2 * st.ex);
    const auto summed = [&](int at) {
      float4 s = *reinterpret_cast<const float4*>(part + at);
#pragma unroll
      for (int w = 1; w < S::kSplits; ++w) {
        const float4 q = *reinterpret_cast<const float4*>(part + w * S::kSumFloats + at);
        s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
      }
      return s;
    };
    const auto write_a = [&](int at, float4 s) {
      split2(s.x * sa, s.y * sa, ah + at, al + at);
      split2(s.z * sa, s.w * sa, ah + at + 2, al + at + 2);
    };
    if (cluster > 1) {
      for (int e = tid; e < P * P / 4; e += kThreads) {
        const int at = e / (P / 4) * kPitch + e % (P / 4) * 4;
        *reinterpret_cast<float4*>(mine + at) = summed(at);
      }
      cta2::cluster_sync_all();
      for (int e = tid; e < P * P / 4; e += kThreads) {
        const int at = e / (P / 4) * kPitch + e % (P / 4) * 4;
        float4 v[kMaxCluster];
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r)
          if (r < cluster)
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(v[r].x), "=f"(v[r].y), "=f"(v[r].z), "=f"(v[r].w)
                         : "r"(cta2::map_to(mine + at, (uint32_t)r)) : "memory");
        float4 s = v[0];
#pragma unroll
        for (int r = 1; r < kMaxCluster; ++r)
          if (r < cluster) {
            s.x += v[r].x; s.y += v[r].y; s.z += v[r].z; s.w += v[r].w;
          }
        write_a(at, s);
      }
    } else {
      for (int e = tid; e < P * P / 4; e += kThreads) {
        const int at = e / (P / 4) * kPitch + e % (P / 4) * 4;
        write_a(at, summed(at));
      }
    }
    __syncthreads();
    {
      // ---- B = b A + c A A: rows 16 m, kQ x 16 columns from 16 q on
      constexpr int kQ = P == 64 ? 2 : 1;
      const float s0 = st.b * exp2i(st.eb - st.ea), s1 = st.c * exp2i(st.eb - 2 * st.ea);
      if (warp < S::kM * S::kM / kQ) {
        const int m = warp % S::kM, q = warp / S::kM * kQ;
        float2 v[2 * kQ][2];
#pragma unroll
        for (int t = 0; t < 2 * kQ; ++t)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int at = (16 * m + row + 8 * h) * kPitch + 16 * q + 8 * t + col;
            v[t][h] = pair2(ah + at, al + at);
          }
        float d[2 * kQ][4] = {}, large[P == 64 ? 2 * kQ : 1][4] = {};    // (large: hi.hi)
#pragma unroll
        for (int kt = 0; kt < S::kM; ++kt) {
          uint32_t a[2][4], b[kQ][2][4];
          const int at = (16 * m + (lane & 15)) * kPitch + 16 * kt + (lane >> 4) * 8;
          ldmatrix_x4(a[0], smem_u32(ah + at));
          ldmatrix_x4(a[1], smem_u32(al + at));
#pragma unroll
          for (int t = 0; t < kQ; ++t) {
            const int bt = (16 * (q + t) + (lane & 15)) * kPitch + 16 * kt + (lane >> 4) * 8;
            ldmatrix_x4(b[t][0], smem_u32(ah + bt));
            ldmatrix_x4(b[t][1], smem_u32(al + bt));
          }
          if constexpr (P <= 32) {
#pragma unroll
            for (int h = 0; h < 2 * kQ; ++h) mma(d[h], a[1], b[h / 2][1][h % 2], b[h / 2][1][h % 2 + 2]);
          }
#pragma unroll
          for (int h = 0; h < 2 * kQ; ++h) mma(d[h], a[0], b[h / 2][1][h % 2], b[h / 2][1][h % 2 + 2]);
#pragma unroll
          for (int h = 0; h < 2 * kQ; ++h) mma(d[h], a[1], b[h / 2][0][h % 2], b[h / 2][0][h % 2 + 2]);
#pragma unroll
          for (int h = 0; h < 2 * kQ; ++h) {
            if constexpr (P == 64) {
              float g[4] = {};
              mma(g, a[0], b[h / 2][0][h % 2], b[h / 2][0][h % 2 + 2]);
#pragma unroll
              for (int e = 0; e < 4; ++e) large[h][e] += g[e];
            } else {
              mma(d[h], a[0], b[h / 2][0][h % 2], b[h / 2][0][h % 2 + 2]);
            }
          }
        }
        if constexpr (P == 64) {
#pragma unroll
          for (int h = 0; h < 2 * kQ; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[h][e] += large[h][e];
        }
#pragma unroll
        for (int t = 0; t < 2 * kQ; ++t)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int at = (16 * m + row + 8 * h) * kPitch + 16 * q + 8 * t + col;
            split2(fmaf(s0, v[t][h].x, s1 * d[t][2 * h]), fmaf(s0, v[t][h].y, s1 * d[t][2 * h + 1]),
                   bh + at, bl + at);
          }
      }
    }
    __syncthreads();
    {
      // ---- X' = a X + B X: as many columns a warp as its registers hold, or eight where that
      // leaves warps idle (at 64 rows B's tiles are most of what is read: sixteen at least)
      constexpr int kNb = P == 64 ? 2 : 4;
      const float s0 = st.a * exp2i(st.last ? -st.ex : st.ex_next - st.ex);
      const float s1 = exp2i((st.last ? 0 : st.ex_next) - st.ex - st.eb);
      const bool last = st.last != 0;
      if (in_registers) {
        apply(x, cs, bh, bl, xh, xl, pitch, s0, s1, last);
      } else if (P < 64 && cs <= 8 * kWarps) {
        if (8 * warp < cs) apply<P, 1>(xh, xl, bh, bl, pitch, 8 * warp, s0, s1, last);
      } else {
        // (a multiple of 16 columns is left over at most, inside the row's padding)
        for (int j = 8 * kNb * warp; j < cs; j += 8 * kNb * kWarps)
          apply<P, kNb>(xh, xl, bh, bl, pitch, j, s0, s1, last);
      }
    }
    __syncthreads();
  }

  // ---------------------------------------------------------------- the result
  if (by_fours(mt.W, mt.ldw, mt.bf16, n)) {
    store_result<kThreads, 4>(mt, u, c0, cols, [&](int i, int j, float (&v)[4]) {
      if (mt.tall) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = get(i + e, j);
      } else {
        const uint2 h = *reinterpret_cast<const uint2*>(xh + i * pitch + j);
        const uint2 l = *reinterpret_cast<const uint2*>(xl + i * pitch + j);
        v[0] = first_of(h.x, l.x);
        v[1] = second_of(h.x, l.x);
        v[2] = first_of(h.y, l.y);
        v[3] = second_of(h.y, l.y);
      }
    });
  } else {
    store_result<kThreads, 1>(mt, u, c0, cols, [&](int i, int j, float (&v)[1]) { v[0] = get(i, j); });
  }
  if (cluster > 1) cta2::cluster_sync_all();     // the peers have read this CTA's sums
}

int smem_of(int P, int cs, int cluster) {
  return P == 16 ? Shape<16>::smem(cs, cluster)
         : P == 32 ? Shape<32>::smem(cs, cluster) : Shape<64>::smem(cs, cluster);
}

template <int P>
cudaError_t launch(const OrthoMat* mats, const int* which, int32_t n, int32_t cluster, int32_t smem,
                   const Steps& st, const OrthoUpdate& u, cudaStream_t s) {
  const cudaError_t e = cudaFuncSetAttribute(
      ortho_mma_kernel<P>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax);
  if (e != cudaSuccess) return e;
  return launch_dependent(ortho_mma_kernel<P>, (unsigned)n * (unsigned)cluster, kThreads,
                          (size_t)smem, s, (unsigned)cluster, true, mats, which, cluster, st, u);
}

}  // namespace

int32_t ortho_mma_rows(int64_t p) { return p <= 64 ? mma_rows(p) : 0; }
int32_t ortho_mma_cluster(int64_t p, int64_t c) {
  if (p > 64) return 0;
  const int P = mma_rows(p);
  for (int cl = 1; cl <= kMaxCluster; cl *= 2) {
    if (c > (int64_t)cl << 16) continue;
    const int cs = mma_cols(c, cl);
    // a CTA takes 10240 elements while the cluster can still grow
    if (cl < kMaxCluster && P * cs > 10240) continue;
    if (smem_of(P, cs, cl) <= kSmemMax) return cl;
  }
  return 0;
}
int32_t ortho_mma_smem(int64_t p, int64_t c, int32_t cluster) {
  return smem_of(mma_rows(p), mma_cols(c, cluster), cluster);
}

cudaError_t launch_ortho_mma(const OrthoMat* mats, const int* which, int32_t n, int32_t rows,
                             int32_t cluster, int32_t smem, const OrthoStep* steps,
                             int32_t n_steps, const OrthoUpdate& u, cudaStream_t s) {
  if (n <= 0) return cudaSuccess;
  if (n_steps > kOrthoMaxSteps || smem > kSmemMax) return cudaErrorInvalidValue;
  Steps st{};
  st.n = n_steps;
  std::copy(steps, steps + n_steps, st.s);
  switch (rows) {
    case 16: return launch<16>(mats, which, n, cluster, smem, st, u, s);
    case 32: return launch<32>(mats, which, n, cluster, smem, st, u, s);
    case 64: return launch<64>(mats, which, n, cluster, smem, st, u, s);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace zo
