// The products of a Newton-Schulz step on SM pairs: M = 256 tcgen05.mma.cta_group::2 across
// the two SMs of a cluster, fp16 operands, fp32 accumulators in Tensor Memory.
//
//   Gram:   A  = X X^T            both operands rows of X, K along them
//   Poly:   B  = b A + c A A      both operands rows of A (A is symmetric)
//   Apply:  X' = a X + B X        rows of B, and X itself as an MN-major operand: the
//                                 descriptor's transpose bit reads X's columns, so no
//                                 transposed copy of X is kept
//
// Pair tile = 256 x N of the result; CTA c of the cluster holds rows 128 c .. of the A
// operand and N / 2 of the B operand's rows (columns of X).  A and B are symmetric: tiles that
// meet or lie left of the diagonal blocks of 256 are computed, those left of them are stored a
// second time transposed.  The accumulators are buffered: the epilogue of one runs under the
// next one's products.
//
// kPairs = false: hi parts only, N = 256 (32 KB per 64 of K for 128 x 256 x 64 multiply-adds
// of an SM) or 128, one accumulation per tile.
// kPairs = true: hi + lo, the products hi.lo + lo.hi + hi.hi.  The tensor cores' fp32 sums
// round towards zero, which over K = 5120 moved an 8 x 5120 result by 3.3e-5 of its norm; so
// every 64 of K the accumulator is drained and added up in the epilogue's registers, rounded
// to nearest, and the small products come first.  N = 128 (64 sums per thread) or 64.
// The narrow tiles are for launches that do not fill the device: their epilogue, the larger part
// of a short launch, is half as long.  Gram's K is split over several SM pairs where few tiles
// are deep (zo_muon.cu): a part's epilogue warps leave their fp32 sums in memory, and the last
// part's add them up, in the parts' order.
// b A, a X and the stored X_k are a pair's sum in both.
//
// Bound by the operands' way from L2 to the SMs (~50 bytes a cycle each, all at work) and, where
// the launches are long, by the power cap's clock; short launches by their latencies (operands
// 1.2 us, drain and stores 1.6 us).  Five steps of 4096 x 4096: bf16 1.01 ms, 1.37 PFLOP/s
// (symmetric products counted once); fp32 2.75 ms, 1.50 PFLOP/s of fp16 products; 1001 x 333
// fp32 0.13 ms in 17 launches.
//
// Roles (320 threads per CTA, one CTA per SM):
//   warp 0:     an elected lane is the TMA producer of this CTA's halves; both halves of a stage
//               complete their bytes on the leader's full barrier, which its producer arms.
//   warp 1:     Tensor Memory; in the leader an elected lane issues the MMAs.
//   warps 2..9: epilogue: warp w reads TMEM lanes 32 (w % 4) .. + 31 and one half of the
//               columns, 32 at a time, and stores 32 x 32 boxes by TMA (64-byte swizzle).
// Every wait is bounded; a give-up sets the abort flag of both CTAs and the status word.
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
using namespace cta2;
using ortho::elected;
using tc::exp2i;

constexpr int kTileRows = 256;
constexpr int kBlockBytes = 64 * 128;                 // a TMA box: 64 rows x 64 fp16
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kBoxBytes = 32 * 32 * 2;
constexpr int kSetBytes = 2 * kBoxBytes;              // a warp's direct and mirrored box
// The ring of stages and the epilogue's boxes share 224 KB.  Narrow tiles of single products have
// two sets of boxes a warp, so that both chunks' X or A are on their way under the MMAs (ninety-six
// 256 x 256 bf16: 220 -> 208 us); for wide ones the ring's sixth stage is worth more (a 7B model's
// 4096 x 4096 and 11008 x 4096: 3395 us with it, 3447 with the second set).
__host__ __device__ constexpr int box_sets(bool pairs, bool narrow) { return !pairs && narrow ? 2 : 1; }
constexpr int kRoom = 224 * 1024;
__host__ __device__ constexpr int ring_bytes(bool pairs, bool narrow) {
  return kRoom - box_sets(pairs, narrow) * kEpiWarps * kSetBytes;
}
constexpr int kTmemCols = 512;
constexpr size_t kSmem = kRoom + 1024 /*barriers*/ + 1024 /*align*/;
static_assert(kSmem <= 227 * 1024, "shared memory per CTA");
constexpr long long kWait = 4000000000LL;             // ~2 s at 2 GHz

struct Shared {
  uint64_t full[8], empty[8];
  uint64_t acc_full[4], acc_empty[4];
  uint64_t drain;                // one commit after the leader's last MMA
  uint64_t in_full[2 * kEpiWarps];   // an epilogue warp's boxes of A or X have arrived, by set
  uint32_t tmem_base;
  int abort_flag;
};

__device__ __forceinline__ void give_up(Shared& sh, uint32_t* status) {
  atomicOr(status, 1u);
  *reinterpret_cast<volatile int*>(&sh.abort_flag) = 1;
  store_peer(&sh.abort_flag, 1);
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
}
// A wait by a whole warp, the same for every lane.  (A lane's own wait may run out where another's
// does not; the warp-wide instructions behind a wait need all lanes, and lane 0 to report it.)
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, const volatile int* abort) {
  return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abort, kWait)) != 0;
}

// Descriptor of an MN-major operand in 128-byte swizzled blocks of 64 columns x 64 K-rows:
// K-rows 128 bytes apart, groups of eight 1024 bytes apart (stride offset), blocks of 64
// columns 8192 bytes apart (leading offset).
__device__ __forceinline__ uint64_t sdesc_mn_sw128(uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(8192u >> 4) << 16;
  d |= static_cast<uint64_t>(1024u >> 4) << 32;
  d |= static_cast<uint64_t>(1u) << 46;
  d |= static_cast<uint64_t>(2u) << 61;
  return d;
}
constexpr uint32_t kMnMajorB = 1u << 16;               // instruction descriptor: B MN-major

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

struct Phase {
  OrthoStep st;
  OrthoUpdate u;
};

// W <- keep W - lr s v, or W <- v, of 32 values of one row of X.  `w` points at the first;
// the next is `step` elements on, `n` are inside.
template <typename T, bool kWide>
__device__ __forceinline__ void write_weights(T* w, int64_t step, int n, const float (&v)[32],
                                              const OrthoUpdate& u, float rate) {
  if constexpr (kWide) {            // 32 neighbours of a 16-byte aligned row
    constexpr int kE = 16 / sizeof(T);
#pragma unroll
    for (int q = 0; q < 32; q += kE) {
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (u.step) raw = *reinterpret_cast<const uint4*>(w + q);
      uint32_t r[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) {
          const float o = u.step ? fmaf(-rate, v[q + e], u.keep * __uint_as_float(r[e])) : v[q + e];
          r[e] = __float_as_uint(o);
        } else {
          float a = v[q + 2 * e], b = v[q + 2 * e + 1];
          if (u.step) {
            a = fmaf(-rate, a, u.keep * __uint_as_float(r[e] << 16));
            b = fmaf(-rate, b, u.keep * __uint_as_float(r[e] & 0xFFFF0000u));
          }
          const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
          r[e] = *reinterpret_cast<const uint32_t*>(&h);
        }
      }
      *reinterpret_cast<uint4*>(w + q) = make_uint4(r[0], r[1], r[2], r[3]);
    }
  } else {
    float old[32];
    if (u.step) {
#pragma unroll
      for (int q = 0; q < 32; ++q)
        if (q < n) old[q] = static_cast<float>(w[q * step]);
    }
#pragma unroll
    for (int q = 0; q < 32; ++q)
      if (q < n) w[q * step] = static_cast<T>(u.step ? fmaf(-rate, v[q], u.keep * old[q]) : v[q]);
  }
}

// Rows i0 .. + 31 of X, columns j0 .. + n - 1, in the caller's matrix.
__device__ __forceinline__ void prefetch_weights(const OrthoMat& mt, int64_t j0, int n, int64_t i0) {
  const int lane = threadIdx.x & 31, size = mt.bf16 ? 2 : 4;
  const uint8_t* w = static_cast<const uint8_t*>(mt.W);
  const int64_t i = i0 + lane;
  if (mt.tall) {
    for (int q = lane; q < n; q += 32)
      if (i0 < mt.p && j0 + q < mt.c)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(w + ((j0 + q) * mt.ldw + i0) * size));
  } else {
    for (int q = 0; q < n; q += 128 / size)
      if (i < mt.p && j0 + q < mt.c)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(w + (i * mt.ldw + j0 + q) * size));
  }
}

// kLast: Apply of the last step, which writes W.
template <bool kPairs, bool kNarrow, int phase, bool kLast>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
ortho_gemm_kernel(const OrthoMat* __restrict__ mats, const CUtensorMap* __restrict__ maps,
                  const OrthoTile* __restrict__ tiles, const int32_t* __restrict__ first,
                  float* __restrict__ sums, uint32_t* __restrict__ counters, const Phase ph,
                  uint32_t* __restrict__ status) {
  constexpr int kCols = ortho_tile_cols(kPairs, kNarrow);
  // boxes of B per CTA: kCols / 2 rows (at 64 columns a box's other half is not read)
  constexpr int kBBoxes = kCols >= 128 ? kCols / 128 : 1;
  constexpr int kABytes = 2 * kBlockBytes, kBBytes = kBBoxes * kBlockBytes;   // per CTA
  constexpr int kStageBytes = (kPairs ? 2 : 1) * (kABytes + kBBytes);
  constexpr int kSets = box_sets(kPairs, kNarrow), kRing = ring_bytes(kPairs, kNarrow);
  constexpr int kStages = kRing / kStageBytes < 8 ? kRing / kStageBytes : 8;
  constexpr int kBufs = kTmemCols / kCols < 4 ? kTmemCols / kCols : 4;
  constexpr int kWarpCols = kCols / 2, kChunks = kWarpCols / 32;
  // a pair's stage is one accumulation: the barrier that tells the epilogue that it is done
  // tells the producer that the stage is free
  static_assert(kStages <= 8 && kBufs <= 4 && sizeof(Shared) <= 1024 && (!kPairs || kStages == kBufs));
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  uint8_t* out_smem = smem + kRing;
  Shared& sh = *reinterpret_cast<Shared*>(smem + kRoom);
  const uint32_t rank = cluster_rank();
  const bool leader = rank == 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int pair = blockIdx.x >> 1;
  const int t_begin = first[pair], t_end = first[pair + 1];
  const volatile int* abort = &sh.abort_flag;
  uint64_t* const released = kPairs ? sh.acc_full : sh.empty;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sh.full[s], 1);
      mbar_init(&sh.empty[s], 1);
    }
    for (int s = 0; s < kBufs; ++s) {
      mbar_init(&sh.acc_full[s], 1);
      mbar_init(&sh.acc_empty[s], 2 * kEpiWarps);
    }
    mbar_init(&sh.drain, 1);
    for (int w = 0; w < 2 * kEpiWarps; ++w) mbar_init(&sh.in_full[w], 1);
    sh.abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc_pair(&sh.tmem_base, kTmemCols);
  tc_fence_before();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;
  // the context's tables are older than the launches before this one: the first tile's entry
  // and tensor maps are fetched under their tail
  if (t_begin < t_end && (warp == 0 || warp == 2) && lane == 0) {
    const CUtensorMap* m = maps + (int64_t)tiles[t_begin].maps * kOrthoMaps;
    const int cur = ph.st.k & 1;
    constexpr int kSide = phase == kOrthoGram ? kMapX : phase == kOrthoPoly ? kMapA : kMapB;
    if (warp == 0) {
      prefetch_map(m + kSide + (phase == kOrthoGram ? cur : 0));
      if (phase == kOrthoApply) prefetch_map(m + kMapX + cur);
      if (kPairs) prefetch_map(m + kSide + (phase == kOrthoGram ? 2 + cur : 1));
      if (kPairs && phase == kOrthoApply) prefetch_map(m + kMapX + 2 + cur);
    } else {
      if (phase != kOrthoGram) prefetch_map(m + (phase == kOrthoPoly ? kMapStoreA : kMapStoreX + cur));
      if (!kLast)
        prefetch_map(m + (phase == kOrthoGram ? kMapStoreA
                          : phase == kOrthoPoly ? kMapStoreB : kMapStoreX + (cur ^ 1)));
    }
  }
  __syncwarp();
  pdl_wait();
  pdl_trigger();

  if (warp == 0) {
    // ---------------------------------------------------------------- operands (this CTA)
    int stage = 0;
    uint32_t free_parity = 1;                  // of empty[stage]: the first round needs no wait
    int64_t filled = 0;
    bool ok = true;
    for (int t = t_begin; t < t_end && ok; ++t) {
      const OrthoTile tl = tiles[t];
      const CUtensorMap* m = maps + (int64_t)tl.maps * kOrthoMaps;
      const int cur = ph.st.k & 1;
      const CUtensorMap* ah = m + (phase == kOrthoGram ? kMapX + cur
                                   : phase == kOrthoPoly ? kMapA : kMapB);
      const CUtensorMap* al = ah + (phase == kOrthoGram ? 2 : 1);
      const CUtensorMap* bh = m + (phase == kOrthoPoly ? kMapA : kMapX + cur);
      const CUtensorMap* bl = bh + (phase == kOrthoPoly ? 1 : 2);
      const int i0 = tl.i0 + 128 * (int)rank, j0 = tl.j0 + kCols / 2 * (int)rank;
      for (int k0 = 64 * tl.k0; k0 < 64 * tl.k1; k0 += 64) {
        if (!warp_wait(&released[stage], free_parity, abort)) {
          ok = false;
          break;
        }
        if (elected()) {
          uint64_t* full = &sh.full[stage];
          if (leader) mbar_arrive_expect_tx(full, 2 * kStageBytes);
          // hi parts of A and B, then the lo parts
          uint8_t* dst = smem + stage * kStageBytes;
#pragma unroll
          for (int part = 0; part < (kPairs ? 2 : 1); ++part) {
            const CUtensorMap* a = part ? al : ah;
            const CUtensorMap* bm = part ? bl : bh;
#pragma unroll
            for (int q = 0; q < 2; ++q, dst += kBlockBytes)
              tma_load_2d_to_leader(dst, a, k0, i0 + 64 * q, full);
#pragma unroll
            for (int q = 0; q < kBBoxes; ++q, dst += kBlockBytes) {
              if (phase == kOrthoApply) tma_load_2d_to_leader(dst, bm, j0 + 64 * q, k0, full);
              else tma_load_2d_to_leader(dst, bm, k0, j0 + 64 * q, full);
            }
          }
        }
        __syncwarp();
        ++filled;
        if (++stage == kStages) {
          stage = 0;
          free_parity ^= 1u;
        }
      }
    }
    if (!ok && lane == 0) give_up(sh, status);
    // the leader's MMAs have released every stage this CTA filled
    for (int s = 0; s < kStages; ++s) {
      const int64_t last = tc::last_in_slot(filled, s, kStages);
      if (last >= 0)
        mbar_wait_bounded(&released[s], (uint32_t)((last / kStages) & 1), nullptr, kWait);
    }
  } else if (warp == 1 && leader) {
    // ---------------------------------------------------------------- MMA issuer (leader)
    // One lane feeds the tensor cores of two SMs, an MMA every 64 (pairs) or 128 cycles, and
    // every instruction between two MMAs is time they may lose: descriptors and barriers move
    // by additions (with 64-bit remainders in this loop a stage of 64 took 715 to 906 cycles).
    const bool mn = phase == kOrthoApply;
    const uint32_t idesc = idesc_f16_f32(kTileRows, kCols) | (mn ? kMnMajorB : 0u);
    const uint32_t ring = smem_u32(smem);
    constexpr uint64_t kStageStep = kStageBytes >> 4, kLoStep = (kABytes + kBBytes) >> 4;
    const uint64_t a_first = sdesc_k_sw128(ring);
    const uint64_t b_first = mn ? sdesc_mn_sw128(ring + kABytes) : sdesc_k_sw128(ring + kABytes);
    const uint64_t b_step = (mn ? 2048 : 32) >> 4;
    int stage = 0, acc = 0;
    uint32_t parity = 0, acc_parity = 1;
    bool ok = true;
    for (int t = t_begin; t < t_end && ok; ++t) {
      const int n = tiles[t].k1 - tiles[t].k0;
      if constexpr (!kPairs) {
        if (!warp_wait(&sh.acc_empty[acc], acc_parity, abort)) {
          ok = false;
          break;
        }
      }
      for (int k = 0; k < n; ++k) {
        // a pair's stage is an accumulation of its own
        if (kPairs && !warp_wait(&sh.acc_empty[stage], parity ^ 1u, abort)) ok = false;
        if (!ok || !warp_wait(&sh.full[stage], parity, abort)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint64_t ad = a_first + (uint64_t)stage * kStageStep;
        const uint64_t bd = b_first + (uint64_t)stage * kStageStep;
        const uint32_t d = tmem + (uint32_t)((kPairs ? stage : acc) * kCols);
        if (elected()) {
          if constexpr (kPairs) {
            // hi.lo, lo.hi, hi.hi
#pragma unroll
            for (int e = 0; e < 12; ++e)
              mma_pair_ss(d, ad + 2 * (e % 4) + (e / 4 == 1 ? kLoStep : 0),
                          bd + b_step * (e % 4) + (e / 4 == 0 ? kLoStep : 0), idesc, e != 0 ? 1u : 0u);
            commit_both(&sh.acc_full[stage]);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              mma_pair_ss(d, ad + 2 * e, bd + b_step * e, idesc, e != 0 || k != 0 ? 1u : 0u);
            commit_both(&sh.empty[stage]);
            if (k + 1 == n) commit_both(&sh.acc_full[acc]);
          }
        }
        __syncwarp();
        if (++stage == kStages) {
          stage = 0;
          parity ^= 1u;
        }
      }
      if constexpr (!kPairs) {
        if (++acc == kBufs) {
          acc = 0;
          acc_parity ^= 1u;
        }
      }
    }
    if (!ok && lane == 0) give_up(sh, status);
    // every MMA has completed before Tensor Memory is freed
    if (elected()) commit_both(&sh.drain);
    __syncwarp();
    mbar_wait_bounded(&sh.drain, 0u, nullptr, kWait);
  } else if (warp >= 2) {
    // ---------------------------------------------------------------- epilogue (each CTA)
    const int g = warp & 3;                        // TMEM lane group
    const int half = (warp - 2) >> 2;              // half of the columns
    uint8_t* const boxes = out_smem + (warp - 2) * kSets * kSetBytes;
    uint64_t* const in_full = &sh.in_full[2 * (warp - 2)];
    constexpr bool kTwo = phase == kOrthoApply || kPairs;
    uint32_t in_parity[kSets] = {};
    bool pending[kSets] = {};                      // lane 0: boxes requested and not yet taken
    int64_t n_acc = 0;
    bool ok = true;
    for (int t = t_begin; t < t_end && ok; ++t) {
      const OrthoTile tl = tiles[t];
      const OrthoMat& mt = mats[tl.mat];
      const CUtensorMap* m = maps + (int64_t)tl.maps * kOrthoMaps;
      const int cur = ph.st.k & 1;
      const int64_t i0 = tl.i0 + 128 * (int64_t)rank + 32 * g, i = i0 + lane;
      const int64_t p = mt.p, cols = phase == kOrthoApply ? mt.c : mt.p;
      const uint32_t col0 = ((uint32_t)(32 * g) << 16) + (uint32_t)(kWarpCols * half);
      const auto outside = [&](int q) {            // the same in every lane
        return i0 >= p || tl.j0 + kWarpCols * half + 32 * q >= cols;
      };
      // lane 0: what is added to the product (A in Poly, X in Apply), 32 x 32 of hi and of lo,
      // into the warp's boxes once their last stores have read them
      const auto request = [&](int q) {
        if (phase == kOrthoGram || outside(q)) return;
        const CUtensorMap* from = m + (phase == kOrthoPoly ? kMapStoreA : kMapStoreX + cur);
        const int j = tl.j0 + kWarpCols * half + 32 * q;
        uint8_t* to = boxes + q % kSets * kSetBytes;
        uint64_t* full = in_full + q % kSets;
        bulk_wait_read_all();
        pending[q % kSets] = true;
        mbar_arrive_expect_tx(full, (kTwo ? 2 : 1) * kBoxBytes);
        tma_load_2d(to, from, j, (int)i0, full);
        if (kTwo) tma_load_2d(to + kBoxBytes, from + (phase == kOrthoPoly ? 1 : 2), j, (int)i0, full);
      };
      if (lane == 0) {
#pragma unroll
        for (int q = 0; q < (kSets < kChunks ? kSets : kChunks); ++q) request(q);
      }
      __syncwarp();
      if constexpr (kLast) {
        // the weights that this warp will update, on their way to L2 while the MMAs run
        if (ph.u.step) prefetch_weights(mt, tl.j0 + kWarpCols * half, kWarpCols, i0);
      }
      uint32_t raw[kPairs ? kChunks : 1][32];
      int acc = 0;
      if constexpr (kPairs) {
        // the stages' sums, added up in fp32
        const int segs = tl.k1 - tl.k0;
#pragma unroll
        for (int q = 0; q < kChunks; ++q)
#pragma unroll
          for (int e = 0; e < 32; ++e) raw[q][e] = 0u;
        for (int sg = 0; sg < segs; ++sg, ++n_acc) {
          acc = (int)(n_acc % kBufs);
          if (!warp_wait(&sh.acc_full[acc], (uint32_t)((n_acc / kBufs) & 1), abort)) {
            ok = false;
            break;
          }
          tc_fence_after();
#pragma unroll
          for (int q = 0; q < kChunks; ++q) {
            uint32_t part[32];
            tmem_ld_32x32b_x32(tmem + col0 + (uint32_t)(acc * kCols + 32 * q), part);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e)
              raw[q][e] = __float_as_uint(__uint_as_float(raw[q][e]) + __uint_as_float(part[e]));
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_leader(&sh.acc_empty[acc]);
        }
      } else {
        acc = (int)(n_acc % kBufs);
        ok = warp_wait(&sh.acc_full[acc], (uint32_t)((n_acc / kBufs) & 1), abort);
        ++n_acc;
        tc_fence_after();
      }
      if (!ok) break;
      bool finish = true, shared = false;
      if (phase == kOrthoGram && tl.parts > 1 && !outside(0)) {
        // this warp's sums of every part lie together: 32 lanes apart for coalescing
        shared = true;
        constexpr int kOwn = 32 * 32 * kChunks;
        float* mine = sums + (int64_t)(tl.sum0 + tl.part) * ortho_part_floats(kPairs, kNarrow) +
                      ((int)rank * kEpiWarps + warp - 2) * kOwn + lane;
#pragma unroll
        for (int q = 0; q < kChunks; ++q) {
          if constexpr (!kPairs) {
            tmem_ld_32x32b_x32(tmem + col0 + (uint32_t)(acc * kCols + 32 * q), raw[0]);
            tmem_ld_wait();
          }
#pragma unroll
          for (int e = 0; e < 32; ++e)
            mine[(q * 32 + e) * 32] = __uint_as_float(raw[kPairs ? q : 0][e]);
        }
        __threadfence();
        __syncwarp();
        uint32_t* counter = counters + tl.slot * kOrthoSlotCounters + (int)rank * kEpiWarps + warp - 2;
        uint32_t seen = 0;
        if (lane == 0) {
          seen = atomicAdd(counter, 1u);
          if (seen == (uint32_t)tl.parts - 1) *counter = 0;    // for the next launch
        }
        finish = __shfl_sync(0xffffffffu, seen, 0) == (uint32_t)tl.parts - 1;
        __threadfence();
      }
#pragma unroll
      for (int q = 0; q < kChunks; ++q) {
        const int64_t j0 = tl.j0 + kWarpCols * half + 32 * q;
        if (outside(q) || !finish) continue;
        uint8_t* const direct = boxes + q % kSets * kSetBytes;
        uint8_t* const mirror = direct + kBoxBytes;
        if (phase == kOrthoGram && shared) {
          constexpr int kOwn = 32 * 32 * kChunks;
          const float* from = sums + (int64_t)tl.sum0 * ortho_part_floats(kPairs, kNarrow) +
                              ((int)rank * kEpiWarps + warp - 2) * kOwn + lane;
          float total[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) total[e] = __ldcg(from + (q * 32 + e) * 32);
          for (int s = 1; s < tl.parts; ++s) {
            from += ortho_part_floats(kPairs, kNarrow);
#pragma unroll
            for (int e = 0; e < 32; ++e) total[e] += __ldcg(from + (q * 32 + e) * 32);
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) raw[kPairs ? q : 0][e] = __float_as_uint(total[e]);
        } else if constexpr (!kPairs) {
          tmem_ld_32x32b_x32(tmem + col0 + (uint32_t)(acc * kCols + 32 * q), raw[0]);
          tmem_ld_wait();
        }
        const uint32_t (&sum)[32] = raw[kPairs ? q : 0];
        float v[32];
        if (phase == kOrthoGram) {
          const float s = exp2i(ph.st.ea - 2 * ph.st.ex);
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(sum[e]) * s;
        } else {
          if (!warp_wait(in_full + q % kSets, in_parity[q % kSets], abort)) {
            ok = false;
            break;
          }
          in_parity[q % kSets] ^= 1u;
          pending[q % kSets] = false;
          constexpr bool kPoly = phase == kOrthoPoly;
          const float s0 = kPoly ? ph.st.b * exp2i(ph.st.eb - ph.st.ea)
                                 : ph.st.a * exp2i(kLast ? -ph.st.ex : ph.st.ex_next - ph.st.ex);
          const float s1 = kPoly ? ph.st.c * exp2i(ph.st.eb - 2 * ph.st.ea)
                                 : exp2i((kLast ? 0 : ph.st.ex_next) - ph.st.ex - ph.st.eb);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int at = lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4);
            const uint4 h = *reinterpret_cast<const uint4*>(direct + at);
            const uint4 l = kTwo ? *reinterpret_cast<const uint4*>(mirror + at) : make_uint4(0, 0, 0, 0);
            const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const float2 x = unpack2(hw[w]), y = unpack2(lw[w]);
              const int e = 8 * c + 2 * w;
              v[e] = fmaf(s0, x.x + y.x, s1 * __uint_as_float(sum[e]));
              v[e + 1] = fmaf(s0, x.y + y.y, s1 * __uint_as_float(sum[e + 1]));
            }
          }
          __syncwarp();                            // every lane has read the boxes
        }
        if constexpr (kLast) {
          const float fm = (float)mt.m, fn = (float)mt.n;
          const float rate = ph.u.lr * (ph.u.adjust == 1 ? sqrtf(fmaxf(1.0f, fm / fn))
                                        : ph.u.adjust == 2 ? 0.2f * sqrtf(fmaxf(fm, fn)) : 1.0f);
          const int n = (int)min((int64_t)32, cols - j0);
          const int64_t at = mt.tall ? j0 * mt.ldw + i : i * mt.ldw + j0;
          const int64_t step = mt.tall ? mt.ldw : 1;
          const bool wide = !mt.tall && n == 32 && mt.wide_rows;
          if (i >= p) {
            // a row past the matrix
          } else if (mt.bf16) {
            __nv_bfloat16* w = static_cast<__nv_bfloat16*>(mt.W) + at;
            if (wide) write_weights<__nv_bfloat16, true>(w, step, n, v, ph.u, rate);
            else write_weights<__nv_bfloat16, false>(w, step, n, v, ph.u, rate);
          } else {
            float* w = static_cast<float*>(mt.W) + at;
            if (wide) write_weights<float, true>(w, step, n, v, ph.u, rate);
            else write_weights<float, false>(w, step, n, v, ph.u, rate);
          }
          if (lane == 0 && q + kSets < kChunks) request(q + kSets);
          __syncwarp();
          continue;
        }
        // hi, then (a pair, or X in any case) lo, as 32 x 32 boxes; below the diagonal of a
        // symmetric result the box of the transposed place too
        const bool both = phase != kOrthoApply && tl.j0 + kCols <= tl.i0;
        const int parts = phase == kOrthoApply || kPairs ? 2 : 1;
        const CUtensorMap* to = m + (phase == kOrthoGram ? kMapStoreA
                                     : phase == kOrthoPoly ? kMapStoreB : kMapStoreX + (cur ^ 1));
        const int to_lo = phase == kOrthoApply ? 2 : 1;
        for (int part = 0; part < parts; ++part) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            w[e] = pack2(v[2 * e], v[2 * e + 1]);
            const float2 h = unpack2(w[e]);        // what is left for the lo part
            v[2 * e] -= h.x;
            v[2 * e + 1] -= h.y;
          }
          // the box's last store has read it: Apply's parts take the boxes that held X's
          uint8_t* box = phase == kOrthoApply && part == 1 ? mirror : direct;
          if (phase != kOrthoApply) {
            if (lane == 0) bulk_wait_read_all();
            __syncwarp();
          }
#pragma unroll
          for (int c = 0; c < 4; ++c)
            *reinterpret_cast<uint4*>(box + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)) =
                make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
          if (both) {
            // two rows' values of one column to a word: neighbouring lanes trade halves
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const uint32_t o = __shfl_xor_sync(0xffffffffu, w[e], 1);
              const uint32_t mine = (lane & 1) ? (o >> 16) | (w[e] & 0xFFFF0000u)
                                               : (w[e] & 0xFFFFu) | (o << 16);
              const int row = 2 * e + (lane & 1);  // column 2 e + (lane & 1) of the tile
              *reinterpret_cast<uint32_t*>(mirror + row * 64 + (((lane >> 3) ^ ((row >> 1) & 3)) << 4) +
                                           (lane & 6) * 2) = mine;
            }
          }
          fence_async_smem();
          __syncwarp();
          if (lane == 0) {
            tma_store_2d(to + part * to_lo, (int)j0, (int)i0, box);
            if (both) tma_store_2d(to + part * to_lo, (int)i0, (int)j0, mirror);
            bulk_commit();
          }
        }
        if (lane == 0 && q + kSets < kChunks) request(q + kSets);
        __syncwarp();
      }
      if constexpr (!kPairs) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_leader(&sh.acc_empty[acc]);
      }
    }
    if (!ok && lane == 0) give_up(sh, status);
#pragma unroll
    for (int q = 0; q < kSets; ++q)
      if (lane == 0 && pending[q]) mbar_wait_bounded(in_full + q, in_parity[q], nullptr, kWait);
    if (lane == 0) bulk_wait_all();
  }

  tc_fence_before();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, kTmemCols);
  }
}

// f(kernel) with the instance of a launch
template <typename F>
auto with_kernel(bool pairs, bool narrow, int phase, bool last, F f) {
#define ZO_PHASE(P, N)                                                    \
  phase == kOrthoGram ? f(ortho_gemm_kernel<P, N, kOrthoGram, false>)     \
  : phase == kOrthoPoly ? f(ortho_gemm_kernel<P, N, kOrthoPoly, false>)   \
  : last ? f(ortho_gemm_kernel<P, N, kOrthoApply, true>)                  \
         : f(ortho_gemm_kernel<P, N, kOrthoApply, false>)
  if (pairs) return narrow ? ZO_PHASE(true, true) : ZO_PHASE(true, false);
  return narrow ? ZO_PHASE(false, true) : ZO_PHASE(false, false);
#undef ZO_PHASE
}

}  // namespace

int32_t ortho_max_pairs() {
  // (every instance has the same launch shape and shared memory)
  return with_kernel(true, false, kOrthoApply, true, [](auto kernel) -> int32_t {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = kSmem;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem) !=
            cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) != cudaSuccess)
      return 0;
    return clusters;
  });
}

cudaError_t launch_ortho_product(const OrthoMat* mats, const CUtensorMap* maps,
                                 const OrthoTile* tiles, const int32_t* first, float* sums,
                                 uint32_t* counters, bool pairs, bool narrow, int32_t n_pairs,
                                 OrthoPhase phase, const OrthoStep& st, const OrthoUpdate& u,
                                 uint32_t* status, cudaStream_t s) {
  if (n_pairs <= 0) return cudaErrorInvalidValue;
  return with_kernel(pairs, narrow, (int)phase, st.last != 0, [&](auto kernel) -> cudaError_t {
    const cudaError_t e =
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    if (e != cudaSuccess) return e;
    return launch_dependent(kernel, 2u * (unsigned)n_pairs, kThreads, kSmem, s, 1, true, mats, maps,
                            tiles, first, sums, counters, Phase{st, u}, status);
  });
}

}  // namespace zo
