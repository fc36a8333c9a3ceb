// The gated linear block's forward pass for at most 128 tokens, where reading Wg and Wu is what there is
// to do.
//
// A CTA owns all tokens and `cols` columns of H (rows of Wg and of Wu; a multiple of 16, chosen so
// that the CTAs fill the SMs evenly): an M = 128 tcgen05.mma with the tokens as its rows and the 2 cols
// rows of both weights, which lie behind one another in shared memory, as its N columns, over all of
// K.  So an accumulator's columns 0 .. cols - 1 are G's and the next cols U's.  On SM pairs an MMA
// of M = 256 takes 128 cycles for 16 of K however few its columns, since its A operand has to be read,
// and covers half as many weights of an SM (7B shapes, turned tiles: 33.9 us at one token, 38.8 at 128;
// this 31.1 and 33.6).
// Only the tokens' rows of X are loaded (rounded up to eight): the MMA's rows past them read whatever
// follows in shared memory and end in accumulator lanes that nothing reads.
//
// Bound by HBM (one token on the 7B shapes: 180 MB in 31 us).  Roles (256 threads): warp 0 loads by TMA, warp 1 issues the MMAs (an elected lane
// each) and owns the Tensor Memory, then all eight warps empty the accumulator.  Every wait is
// bounded; a give-up sets the status word, the producer waits for its copies in flight, the MMA warp
// for its MMAs, NaN is stored where the sums are not known to be whole, and Tensor Memory is freed.
#include <algorithm>

#include <cuda_bf16.h>

#include "zo_launch.cuh"
#include "zo_ops.h"
#include "zo_ortho_io.cuh"
#include "zo_sm100.cuh"
#include "zo_tc_common.cuh"

namespace zo {
namespace {

using namespace sm100;
using ortho::elected;

constexpr int kThreads = 256, kMaxStages = 12;
constexpr int kASpan = 128 * 128;                     // bytes of A that an MMA reads, whatever is loaded
constexpr int kRoom = 208 * 1024;                     // the stages, and A's span behind the last one
constexpr size_t kSmem = kRoom + 1024 /*barriers*/ + 1024 /*align*/;
static_assert(kSmem <= 227 * 1024, "shared memory per CTA");
constexpr long long kWait = 4000000000LL;             // ~2 s at 2 GHz

struct Shared {
  uint64_t full[kMaxStages], empty[kMaxStages];
  uint64_t acc_full;
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(Shared) <= 1024, "barriers");

__device__ __forceinline__ void give_up(Shared& sh, uint32_t* status) {
  atomicOr(status, 1u);
  *reinterpret_cast<volatile int*>(&sh.abort_flag) = 1;
}
// A wait by a whole warp, the same for every lane.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, const volatile int* abort) {
  return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abort, kWait)) != 0;
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// 16 values of this lane's row, from `col` on (a multiple of 16): F is a multiple of 8.
__device__ __forceinline__ void store_row(const float (&v)[16], uint16_t* row, int col, int F) {
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (col + 8 * c < F)
      *reinterpret_cast<uint4*>(row + col + 8 * c) =
          make_uint4(pack2(v[8 * c], v[8 * c + 1]), pack2(v[8 * c + 2], v[8 * c + 3]),
                     pack2(v[8 * c + 4], v[8 * c + 5]), pack2(v[8 * c + 6], v[8 * c + 7]));
}

__global__ void __launch_bounds__(kThreads, 1)
gated_few_kernel(const __grid_constant__ GatedFew a, uint32_t* __restrict__ status) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  Shared& sh = *reinterpret_cast<Shared*>(smem + kRoom);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const volatile int* abort = &sh.abort_flag;
  const int col0 = blockIdx.x * a.cols, steps = (a.D + 63) / 64;
  const int a_bytes = a.box_rows * 128, b_bytes = a.cols * 128;   // of X; of Wg, and of Wu
  const int stage_bytes = a_bytes + 2 * b_bytes;

  if (threadIdx.x == 0) {
    for (int s = 0; s < a.stages; ++s) {
      mbar_init(&sh.full[s], 1);
      mbar_init(&sh.empty[s], 1);
    }
    mbar_init(&sh.acc_full, 1);
    sh.abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&sh.tmem_base, (uint32_t)a.tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;
  pdl_wait();

  if (warp == 0) {
    bool ok = true;
    int stage = 0, filled = 0;
    uint32_t free_parity = 1;                  // of empty[stage]: the first round needs no wait
    for (int k = 0; k < steps; ++k) {
      if (!warp_wait(&sh.empty[stage], free_parity, abort)) {
        ok = false;
        break;
      }
      if (elected()) {
        uint8_t* dst = smem + stage * stage_bytes;
        mbar_arrive_expect_tx(&sh.full[stage], (uint32_t)stage_bytes);
        tma_load_2d(dst, &a.x, 64 * k, 0, &sh.full[stage]);
        tma_load_2d(dst + a_bytes, &a.w[0], 64 * k, col0, &sh.full[stage]);
        tma_load_2d(dst + a_bytes + b_bytes, &a.w[1], 64 * k, col0, &sh.full[stage]);
      }
      __syncwarp();
      ++filled;
      if (++stage == a.stages) {
        stage = 0;
        free_parity ^= 1u;
      }
    }
    if (!ok && lane == 0) give_up(sh, status);
    if (!ok) {                                 // the copies in flight
      for (int s = 0; s < a.stages; ++s) {
        const int64_t last = tc::last_in_slot(filled, s, a.stages);
        if (last >= 0) mbar_wait_bounded(&sh.full[s], (uint32_t)((last / a.stages) & 1), nullptr, kWait);
      }
    }
  } else if (warp == 1) {
    const uint32_t idesc = idesc_bf16_f32(128, 16) - (2u << 17) + ((uint32_t)(2 * a.cols) >> 3 << 17);
    bool ok = true;
    int stage = 0;
    uint32_t parity = 0;
    for (int k = 0; k < steps; ++k) {
      if (!warp_wait(&sh.full[stage], parity, abort)) {
        ok = false;
        break;
      }
      tc_fence_after();
      const uint32_t at = smem_u32(smem + stage * stage_bytes);
      const uint64_t ad = sdesc_k_sw128(at), bd = sdesc_k_sw128(at + (uint32_t)a_bytes);
      if (elected()) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          mma_f16(tmem, ad + 2 * e, bd + 2 * e, idesc, e != 0 || k != 0 ? 1u : 0u);
        mma_commit(&sh.empty[stage]);
        if (k + 1 == steps) mma_commit(&sh.acc_full);
      }
      __syncwarp();
      if (++stage == a.stages) {
        stage = 0;
        parity ^= 1u;
      }
    }
    if (!ok) {
      if (lane == 0) {
        give_up(sh, status);
        __threadfence_block();                  // (the flag is seen by whoever sees the commit)
      }
      __syncwarp();
      if (elected()) mma_commit(&sh.acc_full);  // every MMA has completed before Tensor Memory is freed
      __syncwarp();
    }
  }
  __syncwarp();
  // (after a give-up acc_full says that the MMAs so far are done; nothing of them is stored.  One
  // answer for the whole warp, as its lanes read Tensor Memory together.)
  const bool done = warp_wait(&sh.acc_full, 0, nullptr);
  if (!done && lane == 0) give_up(sh, status);
  const bool lost = __any_sync(0xffffffffu, !done || *abort);
  tc_fence_after();
  const int row = 32 * (warp & 3) + lane;
  if (32 * (warp & 3) < a.T) {
    const uint32_t from = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    for (int c = warp >> 2; c < a.cols / 16 && col0 + 16 * c < a.F; c += 2) {
      uint32_t gr[16], ur[16];
      if (!lost) {
        tmem_ld_32x32b_x16(from + (uint32_t)(16 * c), gr);
        tmem_ld_32x32b_x16(from + (uint32_t)(a.cols + 16 * c), ur);
        tmem_ld_wait();
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) gr[e] = ur[e] = 0x7FC00000u;
      }
      float g[16], u[16], h[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        g[e] = __uint_as_float(gr[e]);
        u[e] = __uint_as_float(ur[e]);
        h[e] = g[e] * gated_gate(g[e], a.act) * u[e];
      }
      if (row < a.T) {
        const int col = col0 + 16 * c;
        store_row(h, a.out[0] + row * a.ld[0], col, a.F);
        if (a.save) {
          store_row(g, a.out[1] + row * a.ld[1], col, a.F);
          store_row(u, a.out[2] + row * a.ld[2], col, a.F);
        }
      }
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, (uint32_t)a.tmem_cols);
  }
}

}  // namespace

// Columns by the busiest SM's cycles: rounds of CTAs, each D / 64 stages that take the longer of their
// MMAs (~118 cycles for 16 of K and few columns: 16384 of K 62 us) and their operands' way from L2 (~54
// bytes a cycle), and ~5000 for its beginning and end, which nothing overlaps.
bool gated_few_plan(GatedFew* a, int32_t sms) {
  if (a->T > 128) return false;
  const int64_t rows = gated_box_rows(a->T), steps = (a->D + 63) / 64;
  int64_t least = INT64_MAX;
  for (int32_t cols = 16; cols <= 128; cols += 16) {            // (of equals, the most CTAs)
    const int64_t ctas = (a->F + cols - 1) / cols;
    const int64_t stage = std::max<int64_t>(4 * std::max(cols, 118), (rows + 2 * cols) * 128 / 54);
    const int64_t cycles = (ctas + sms - 1) / sms * (steps * stage + 5000);
    if (cycles < least) {
      least = cycles;
      a->cols = cols;
    }
  }
  a->box_rows = gated_box_rows(a->T);
  const int32_t stage = (a->box_rows + 2 * a->cols) * 128;
  a->stages = std::min(kMaxStages, (kRoom - kASpan) / stage);
  a->tmem_cols = 32;
  while (a->tmem_cols < 2 * a->cols) a->tmem_cols *= 2;
  return true;
}

cudaError_t launch_gated_few(const GatedFew& a, uint32_t* status, cudaStream_t s) {
  const cudaError_t e = cudaFuncSetAttribute(gated_few_kernel,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
  if (e != cudaSuccess) return e;
  return launch_dependent(gated_few_kernel, (unsigned)((a.F + a.cols - 1) / a.cols), kThreads, kSmem, s,
                          1, true, a, status);
}

}  // namespace zo
