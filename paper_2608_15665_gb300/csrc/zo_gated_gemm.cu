// The products of the gated linear block on SM pairs: M = 256 tcgen05.mma.cta_group::2 across the
// two SMs of a cluster, bf16 operands, fp32 accumulators in Tensor Memory.
//
//   forward:  (beyond 128 tokens; below, zo_gated_few.cu) tile = 256 tokens x `side` columns of G and
//             the same of U.  CTA c of the pair holds 128 of the tokens, and its half of the B operand is `side` rows of Wg (c = 0) or of
//             Wu (c = 1): accumulator columns 0 .. side - 1 are G's, the next `side` U's, in both
//             CTAs, and the epilogue has both of an element in one thread.
//   turned:   the forward pass with the tokens as the MMAs' columns: tile = 256 columns of G and the
//             same of U x `tokens` tokens, a multiple of 16.  CTA c holds 128 rows of Wg and of Wu
//             (two A operands, an accumulator each) and half of the tokens.  A tile of 256 tokens
//             takes less from L2 than two of the above, and 777 tokens are four tiles of 208 rather
//             than of 256; but the two accumulators leave room for no second pair beyond 128 tokens.
//             gated_plan takes one or the other by what the busiest pair has to do.
//   dX:       tile = 256 tokens x 256 columns; K runs over F twice, dG Wg and then dU Wu into one
//             accumulator.  dG's and dU's rows lie along K, Wg and Wu are MN-major operands (the
//             instruction descriptor's transpose bit), so no transposed copy is kept.
//             Up to 128 tokens dG and dU are sums of two bf16, in two rows a token that the tile has
//             to spare: neighbouring accumulator lanes, which the epilogue adds up.
//   dWg, dWu: tile = 256 rows of F x 256 columns of D, K = the tokens: both operands MN-major.
//
// dX's tiles are the deepest and few (where very few, K is split: gated_parts): they are dealt to the pairs first, round by round, and dW's
// behind them in the same launch, the pairs that have no tile in dX's last round beginning as many
// rounds of dW's earlier as a tile of dX takes.  Neighbouring pairs take neighbouring tiles of
// one block of F's rows: few panels of dG are in use at a time.  (In runs of neighbours per pair the
// panels in use, 160 MB at 4096 tokens, came from HBM once for every tile: dWg and dWu of the 7B
// shapes 525 us.)
//
// Bound by the power cap's clock and the operands' way from L2 to the SMs (4096 tokens on the 7B
// shapes: 366 us forward in a short run, 1.65 PFLOP/s and 447 us in a long one, where cuBLAS takes 443
// for the two products alone; tensor pipe 90% of active cycles forward, 95% backward).  Accumulators
// are fp32 (the tensor cores' sums round towards zero: 2^-23 of the sum's running size a step, far
// below bf16's 2^-9).
//
// Roles (320 threads per CTA, one CTA per SM):
//   warp 0:     an elected lane is the TMA producer of this CTA's halves; both halves of a stage
//               complete their bytes on the leader's full barrier, which its producer arms.
//   warp 1:     Tensor Memory; in the leader an elected lane issues the MMAs into one of two
//               accumulators.
//   warps 2..9: epilogue: warp w reads TMEM lanes 32 (w % 4) .. + 31, every other 16 columns, and
//               stores 32 x 16 boxes by TMA (32-byte swizzle), three of them in turn.
// Every wait is bounded; a give-up sets the abort flag of both CTAs and the status word, and the
// epilogue's warps store NaN for the tiles that they have not seen the end of.
#include <algorithm>

#include <cuda_bf16.h>

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

constexpr int kTileRows = 256, kTileCols = 256;
constexpr int kHalfBytes = 128 * 128;                 // 128 rows x 64 bf16, or two MN-major blocks
constexpr int kRing = 12 * kHalfBytes;
// a CTA's stages: the A operands (128 rows each), then B
template <typename Args>
struct Ring {
  static constexpr int kA = 1;
  static constexpr int kStageBytes = (kA + 1) * kHalfBytes, kStages = kRing / kStageBytes;
};
template <>
struct Ring<GatedTurned> {
  static constexpr int kA = 2;
  static constexpr int kStageBytes = (kA + 1) * kHalfBytes, kStages = kRing / kStageBytes;
};
constexpr int kMaxStages = 6;
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kBoxBytes = kGatedOutRows * kGatedOutCols * 2;
constexpr int kBoxes = 3;                             // of an epilogue warp
constexpr int kBufs = 2, kTmemCols = 512;
constexpr int kRoom = kRing + kEpiWarps * kBoxes * kBoxBytes;
constexpr size_t kSmem = kRoom + 1024 /*barriers*/ + 1024 /*align*/;
static_assert(kSmem <= 227 * 1024, "shared memory per CTA");
constexpr long long kWait = 4000000000LL;             // ~2 s at 2 GHz

struct Shared {
  uint64_t full[kMaxStages], empty[kMaxStages];
  uint64_t acc_full[kBufs], acc_empty[kBufs];
  uint64_t drain;                // one commit after the leader's last MMA
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(Shared) <= 1024, "barriers");

__device__ __forceinline__ void give_up(Shared& sh, uint32_t* status) {
  atomicOr(status, 1u);
  *reinterpret_cast<volatile int*>(&sh.abort_flag) = 1;
  store_peer(&sh.abort_flag, 1);
}
// A wait by a whole warp, the same for every lane.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, const volatile int* abort) {
  return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abort, kWait)) != 0;
}

// Descriptor of an MN-major operand in 128-byte swizzled blocks of 64 columns x 64 K-rows: K-rows
// 128 bytes apart, groups of eight 1024 bytes apart (stride offset), blocks of 64 columns 8192
// bytes apart (leading offset).
__device__ __forceinline__ uint64_t sdesc_mn_sw128(uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(8192u >> 4) << 16;
  d |= static_cast<uint64_t>(1024u >> 4) << 32;
  d |= static_cast<uint64_t>(1u) << 46;
  d |= static_cast<uint64_t>(2u) << 61;
  return d;
}
constexpr uint32_t kMnMajorA = 1u << 15, kMnMajorB = 1u << 16;

// A pair's tiles in their order, the same for every role.
struct Tile {
  int i0, j0;                    // first row and column of the result
  int k0, n;                     // its stages of 64 of K: the first, and their number
  int n0;                        // stages of the first operands (dX)
  int dw;                        // -1: forward or dX; 0, 1: dWg, dWu
  int at, part;                  // dX's tile, and which part of its K
};
__device__ __forceinline__ bool tile_at(const GatedForward& a, int pair, int pairs, int k, Tile* t) {
  // groups of 16 blocks of tokens; within one, the tokens first: the pairs at work share few
  // columns of the weights, and the group's X stays in L2
  const int rows = (a.T + kTileRows - 1) / kTileRows, cols = (a.F + a.side - 1) / a.side;
  const int64_t at = (int64_t)pair + (int64_t)k * pairs;
  if (at >= (int64_t)rows * cols) return false;
  const int group = (int)(at / (16 * (int64_t)cols)), in = (int)(at - (int64_t)group * 16 * cols);
  const int height = min(16, rows - 16 * group);
  t->i0 = (16 * group + in % height) * kTileRows;
  t->j0 = in / height * a.side;
  t->k0 = 0;
  t->n0 = t->n = (a.D + 63) / 64;
  t->dw = -1;
  return true;
}
__device__ __forceinline__ bool tile_at(const GatedBackward& a, int pair, int pairs, int k, Tile* t) {
  const int cols = (a.D + kTileCols - 1) / kTileCols;
  const int mine = a.n_dx > pair ? (a.n_dx - pair + pairs - 1) / pairs : 0;
  if (k < mine) {
    const int item = pair + k * pairs, rows = (a.T + kTileRows - 1) / kTileRows;
    const int at = item / a.parts;
    const int group = at / (16 * cols), in = at - group * 16 * cols;
    const int height = min(16, rows - 16 * group);
    t->i0 = (16 * group + in % height) * kTileRows;
    t->j0 = in / height * kTileCols;
    t->n0 = (a.F + 63) / 64;
    t->at = at;
    t->part = item - at * a.parts;
    t->k0 = 2 * t->n0 * t->part / a.parts;
    t->n = 2 * t->n0 * (t->part + 1) / a.parts - t->k0;
    t->dw = -1;
    return true;
  }
  // dW's rounds: the pairs without a last tile of dX begin `skip` rounds earlier
  const int late = a.n_dx % pairs, early = pairs - late;
  const int round = k - mine + (pair < late ? a.skip : 0);
  const int64_t at = round < a.skip ? (int64_t)round * early + pair - late
                                    : (int64_t)a.skip * early + (int64_t)(round - a.skip) * pairs + pair;
  if (at >= a.n_dw) return false;
  const int half = a.n_dw / 2;
  t->dw = at >= half;
  const int in = (int)at - t->dw * half;
  t->i0 = in / cols * kTileRows;
  t->j0 = in % cols * kTileCols;
  t->k0 = 0;
  t->n0 = (a.T + 63) / 64;
  t->n = a.twin ? 2 * t->n0 : t->n0;
  return true;
}

__device__ __forceinline__ bool tile_at(const GatedTurned& a, int pair, int pairs, int k, Tile* t) {
  // the tokens first: the weights are read by pairs at work at the same time
  const int blocks = (a.T + a.tokens - 1) / a.tokens, rows = (a.F + kTileRows - 1) / kTileRows;
  const int64_t at = (int64_t)pair + (int64_t)k * pairs;
  if (at >= (int64_t)rows * blocks) return false;
  // (many tokens: in groups of 16 blocks of them, as above)
  const int group = (int)(at / (16 * (int64_t)rows)), in = (int)(at - (int64_t)group * 16 * rows);
  const int height = min(16, blocks - 16 * group);
  t->j0 = (16 * group + in % height) * a.tokens;
  t->i0 = in / height * kTileRows;
  t->k0 = 0;
  t->n0 = t->n = (a.D + 63) / 64;
  t->dw = -1;
  return true;
}

// One stage of a tile's operands for CTA `rank`.  Tokens past the last are not loaded where they
// fill a CTA's half (in dX: or are beyond a call's only box): what shared memory holds in their
// place ends in accumulator lanes that nothing reads.
__device__ __forceinline__ void load_stage(const GatedForward& a, const Tile& t, int k, uint32_t rank,
                                           uint8_t* dst, uint64_t* full, bool leader) {
  const bool second = t.i0 + 128 < a.T;
  if (leader)
    mbar_arrive_expect_tx(full, (second ? 2u : 1u) * kHalfBytes + 2u * (uint32_t)a.side * 128u);
  if (rank == 0 || second) tma_load_2d_to_leader(dst, &a.x, 64 * k, t.i0 + 128 * (int)rank, full);
  tma_load_2d_to_leader(dst + kHalfBytes, &a.w[rank], 64 * k, t.j0, full);
}
__device__ __forceinline__ void load_stage(const GatedBackward& a, const Tile& t, int k, uint32_t rank,
                                           uint8_t* dst, uint64_t* full, bool leader) {
  const bool second = t.dw >= 0 || t.i0 + 128 < (a.twin ? 2 * a.T : a.T);
  if (leader)
    mbar_arrive_expect_tx(full, t.dw >= 0 ? 4u * kHalfBytes
                                          : 2u * kHalfBytes + (second ? 2u : 1u) * (uint32_t)a.box_rows * 128u);
  const int i0 = t.i0 + 128 * (int)rank, j0 = t.j0 + 128 * (int)rank;
  const CUtensorMap* b;
  if (t.dw < 0) {
    const int which = k >= t.n0 ? 1 : 0;
    k -= which * t.n0;
    if (rank == 0 || second) tma_load_2d_to_leader(dst, &a.d_rows[which], 64 * k, i0, full);
    b = &a.w_cols[which];
  } else {
    const int which = k >= t.n0 ? 1 : 0;          // (twin: the second parts, with the same X)
    k -= which * t.n0;
    const CUtensorMap* d = &a.d_cols[t.dw][which];
    tma_load_2d_to_leader(dst, d, i0, 64 * k, full);
    tma_load_2d_to_leader(dst + 8192, d, i0 + 64, 64 * k, full);
    b = &a.x_cols;
  }
  tma_load_2d_to_leader(dst + kHalfBytes, b, j0, 64 * k, full);
  tma_load_2d_to_leader(dst + kHalfBytes + 8192, b, j0 + 64, 64 * k, full);
}

__device__ __forceinline__ void load_stage(const GatedTurned& a, const Tile& t, int k, uint32_t rank,
                                           uint8_t* dst, uint64_t* full, bool leader) {
  if (leader) mbar_arrive_expect_tx(full, 4u * kHalfBytes + (uint32_t)a.tokens * 128u);
  tma_load_2d_to_leader(dst, &a.w[0], 64 * k, t.i0 + 128 * (int)rank, full);
  tma_load_2d_to_leader(dst + kHalfBytes, &a.w[1], 64 * k, t.i0 + 128 * (int)rank, full);
  tma_load_2d_to_leader(dst + 2 * kHalfBytes, &a.x, 64 * k, t.j0 + a.tokens / 2 * (int)rank, full);
}

// Accumulators, how many of them take turns, and where the next product's columns begin.
template <typename Args>
__device__ __forceinline__ int bufs_of(const Args&) { return kBufs; }
__device__ __forceinline__ int bufs_of(const GatedTurned& a) { return a.tokens <= 128 ? kBufs : 1; }
template <typename Args>
__device__ __forceinline__ uint32_t acc_at(int acc) {
  return (uint32_t)(acc * (Ring<Args>::kA == 2 ? 128 : kTileCols));
}

// Columns of a tile's accumulator, and how its operands are read.
__device__ __forceinline__ uint32_t idesc_of(const GatedForward& a, const Tile&) {
  return idesc_bf16_f32(kTileRows, 16) - (2u << 17) + ((uint32_t)(2 * a.side) >> 3 << 17);
}
__device__ __forceinline__ uint32_t idesc_of(const GatedTurned& a, const Tile&) {
  return idesc_bf16_f32(kTileRows, 16) - (2u << 17) + ((uint32_t)a.tokens >> 3 << 17);
}
__device__ __forceinline__ uint32_t idesc_of(const GatedBackward&, const Tile& t) {
  return idesc_bf16_f32(kTileRows, kTileCols) | kMnMajorB | (t.dw >= 0 ? kMnMajorA : 0u);
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// The boxes of an epilogue warp, taken in turn.
struct Boxes {
  uint8_t* base;
  int next = 0;
  // 16 values of this lane's row, as a box at (col, row0) of `to`
  __device__ __forceinline__ void store(const float (&v)[16], const CUtensorMap* to, int col, int row0) {
    const int lane = threadIdx.x & 31;
    uint8_t* box = base + next * kBoxBytes;
    next = next == kBoxes - 1 ? 0 : next + 1;
    // (the store of three boxes ago has read it)
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kBoxes - 1) : "memory");
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 2; ++c)
      *reinterpret_cast<uint4*>(box + lane * 32 + ((c ^ ((lane >> 2) & 1)) << 4)) =
          make_uint4(pack2(v[8 * c], v[8 * c + 1]), pack2(v[8 * c + 2], v[8 * c + 3]),
                     pack2(v[8 * c + 4], v[8 * c + 5]), pack2(v[8 * c + 6], v[8 * c + 7]));
    fence_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_2d(to, col, row0, box);
      bulk_commit();
    }
  }
  // 16 tokens' values (from row0 on) of this lane's column col0 + lane, as a box of 16 rows of 32: two
  // columns to a word, for which neighbouring lanes trade halves
  __device__ __forceinline__ void store_turned(const float (&v)[16], const CUtensorMap* to, int col0,
                                               int row0) {
    const int lane = threadIdx.x & 31;
    uint8_t* box = base + next * kBoxBytes;
    next = next == kBoxes - 1 ? 0 : next + 1;
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kBoxes - 1) : "memory");
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t w = pack2(v[2 * e], v[2 * e + 1]);
      const uint32_t o = __shfl_xor_sync(0xffffffffu, w, 1);
      const int row = 2 * e + (lane & 1);
      *reinterpret_cast<uint32_t*>(box + row * 64 + (((lane >> 3) ^ ((row >> 1) & 3)) << 4) + (lane & 6) * 2) =
          (lane & 1) ? (o >> 16) | (w & 0xFFFF0000u) : (w & 0xFFFFu) | (o << 16);
    }
    fence_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_2d(to, col0, row0, box);
      bulk_commit();
    }
  }
};

__device__ __forceinline__ void to_floats(const uint32_t (&r)[16], float (&v)[16]) {
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(r[e]);
}
__device__ __forceinline__ void to_nan(float (&v)[16]) {
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = __int_as_float(0x7FC00000);
}
// Sixteen columns of this warp's lanes of an accumulator, or of two; lost: there is none.
__device__ __forceinline__ void columns(uint32_t tmem, bool lost, float (&v)[16]) {
  if (lost) {
    to_nan(v);
    return;
  }
  uint32_t r[16];
  tmem_ld_32x32b_x16(tmem, r);
  tmem_ld_wait();
  to_floats(r, v);
}
__device__ __forceinline__ void columns(uint32_t g_at, uint32_t u_at, bool lost, float (&g)[16], float (&u)[16]) {
  if (lost) {
    to_nan(g);
    to_nan(u);
    return;
  }
  uint32_t gr[16], ur[16];
  tmem_ld_32x32b_x16(g_at, gr);
  tmem_ld_32x32b_x16(u_at, ur);
  tmem_ld_wait();
  to_floats(gr, g);
  to_floats(ur, u);
}

__device__ __forceinline__ void activate(int32_t act, const float (&g)[16], const float (&u)[16],
                                         float (&h)[16]) {
  if (act == kGatedSilu) {
#pragma unroll
    for (int e = 0; e < 16; ++e) h[e] = g[e] * gated_gate(g[e], kGatedSilu) * u[e];
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) h[e] = g[e] * gated_gate(g[e], kGatedGelu) * u[e];
  }
}

// The accumulator at `tmem` (this warp's lanes) to the results: 32 rows from row0 on, or NaN in their place.
__device__ __forceinline__ void finish(const GatedForward& a, const Tile& t, uint32_t tmem, int half,
                                       int row0, int, bool lost, Boxes& boxes) {
  for (int c = half; c < a.side / 16; c += 2) {
    const int col = t.j0 + 16 * c;
    if (row0 >= a.T || col >= a.F) break;
    float g[16], u[16], h[16];
    columns(tmem + (uint32_t)(16 * c), tmem + (uint32_t)(a.side + 16 * c), lost, g, u);
    activate(a.act, g, u, h);
    boxes.store(h, &a.out[0], col, row0);
    if (a.save) {
      boxes.store(g, &a.out[1], col, row0);
      boxes.store(u, &a.out[2], col, row0);
    }
  }
}
__device__ __forceinline__ void finish(const GatedTurned& a, const Tile& t, uint32_t tmem, int half,
                                       int row0, int, bool lost, Boxes& boxes) {
  for (int c = half; c < a.tokens / 16; c += 2) {
    const int token = t.j0 + 16 * c;
    if (row0 >= a.F || token >= a.T) break;
    float g[16], u[16], h[16];
    columns(tmem + (uint32_t)(16 * c), tmem + (uint32_t)(kTileCols + 16 * c), lost, g, u);
    activate(a.act, g, u, h);
    boxes.store_turned(h, &a.out[0], row0, token);
    if (a.save) {
      boxes.store_turned(g, &a.out[1], row0, token);
      boxes.store_turned(u, &a.out[2], row0, token);
    }
  }
}
// warp: of the pair's sixteen.  Of a tile whose K is split, each warp leaves its part's sums in
// memory (32 lanes apart for coalescing), and the last part's adds them up in the parts' order.
__device__ __forceinline__ void finish(const GatedBackward& a, const Tile& t, uint32_t tmem, int half,
                                       int row0, int warp, bool lost, Boxes& boxes) {
  constexpr int kChunks = kTileCols / 32;             // of a warp
  const CUtensorMap* to = t.dw < 0 ? &a.dx : &a.dw[t.dw];
  const bool twin = t.dw < 0 && a.twin;
  const int rows = t.dw >= 0 ? a.F : twin ? 2 * a.T : a.T, lane = threadIdx.x & 31;
  if (row0 >= rows) return;
  const bool split = t.dw < 0 && a.parts > 1;
  const float* from = nullptr;
  if (split) {
    constexpr int kOwn = 32 * 16 * kChunks;
    float* first = a.sums + (int64_t)t.at * a.parts * kGatedPartFloats + warp * kOwn + lane;
    float* mine = first + t.part * kGatedPartFloats;
#pragma unroll 1
    for (int i = 0; i < kChunks; ++i) {
      if (t.j0 + 16 * (half + 2 * i) >= a.D) break;
      float v[16];
      columns(tmem + (uint32_t)(16 * (half + 2 * i)), lost, v);
#pragma unroll
      for (int e = 0; e < 16; ++e) mine[(i * 16 + e) * 32] = v[e];
    }
    __threadfence();
    __syncwarp();
    uint32_t seen = 0;
    if (lane == 0) seen = atomicAdd(a.counters + t.at * kGatedCounters + warp, 1u);
    if (__shfl_sync(0xffffffffu, seen, 0) != (uint32_t)a.parts - 1) return;
    __threadfence();
    from = first;
  }
#pragma unroll 1
  for (int i = 0; i < kChunks; ++i) {
    const int c = half + 2 * i;
    if (t.j0 + 16 * c >= a.D) break;
    float v[16];
    if (split) {
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = __ldcg(from + (i * 16 + e) * 32);
      for (int p = 1; p < a.parts; ++p)
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] += __ldcg(from + p * kGatedPartFloats + (i * 16 + e) * 32);
    } else {
      columns(tmem + (uint32_t)(16 * c), lost, v);
    }
    if (!twin) {
      boxes.store(v, to, t.j0 + 16 * c, row0);
      continue;
    }
    // the token's two rows are neighbouring lanes
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] += __shfl_xor_sync(0xffffffffu, v[e], 1);
    const int token = (row0 + lane) / 2, col = t.j0 + 16 * c + 8 * (lane & 1);
    if (token < a.T && col < a.D) {
      const bool odd = lane & 1;                    // (each of the two stores eight columns)
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = odd ? pack2(v[2 * e + 8], v[2 * e + 9]) : pack2(v[2 * e], v[2 * e + 1]);
      *reinterpret_cast<uint4*>(a.dx_rows + token * a.lddx + col) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

template <typename Args>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
gated_kernel(const __grid_constant__ Args a, uint32_t* __restrict__ status) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  Shared& sh = *reinterpret_cast<Shared*>(smem + kRoom);
  const uint32_t rank = cluster_rank();
  const bool leader = rank == 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const volatile int* abort = &sh.abort_flag;
  constexpr int kStages = Ring<Args>::kStages, kStageBytes = Ring<Args>::kStageBytes;
  constexpr int kBAt = Ring<Args>::kA * kHalfBytes;
  const int bufs = bufs_of(a);

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
    sh.abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc_pair(&sh.tmem_base, kTmemCols);
  tc_fence_before();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;
  pdl_wait();

  if (warp == 0) {
    // ---------------------------------------------------------------- operands (this CTA)
    int stage = 0;
    uint32_t free_parity = 1;                  // of empty[stage]: the first round needs no wait
    int64_t filled = 0;
    bool ok = true;
    Tile t;
    for (int k = 0; ok && tile_at(a, pair, pairs, k, &t); ++k) {
      for (int q = 0; q < t.n; ++q) {
        if (!warp_wait(&sh.empty[stage], free_parity, abort)) {
          ok = false;
          break;
        }
        if (elected()) load_stage(a, t, t.k0 + q, rank, smem + stage * kStageBytes, &sh.full[stage], leader);
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
        mbar_wait_bounded(&sh.empty[s], (uint32_t)((last / kStages) & 1), nullptr, kWait);
    }
  } else if (warp == 1 && leader) {
    // ---------------------------------------------------------------- MMA issuer (leader)
    const uint32_t ring = smem_u32(smem);
    constexpr uint64_t kStageStep = kStageBytes >> 4;
    int stage = 0, acc = 0;
    uint32_t parity = 0, acc_parity = 1;
    bool ok = true;
    Tile t;
    for (int k = 0; ok && tile_at(a, pair, pairs, k, &t); ++k) {
      const uint32_t idesc = idesc_of(a, t);
      const bool a_mn = (idesc & kMnMajorA) != 0, b_mn = (idesc & kMnMajorB) != 0;
      const uint64_t a_first = a_mn ? sdesc_mn_sw128(ring) : sdesc_k_sw128(ring);
      const uint64_t b_first = b_mn ? sdesc_mn_sw128(ring + kBAt) : sdesc_k_sw128(ring + kBAt);
      const uint64_t a_step = (a_mn ? 2048 : 32) >> 4, b_step = (b_mn ? 2048 : 32) >> 4;
      const uint32_t d = tmem + acc_at<Args>(acc);
      if (!warp_wait(&sh.acc_empty[acc], acc_parity, abort)) {
        ok = false;
        break;
      }
      for (int q = 0; q < t.n; ++q) {
        if (!warp_wait(&sh.full[stage], parity, abort)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint64_t ad = a_first + (uint64_t)stage * kStageStep;
        const uint64_t bd = b_first + (uint64_t)stage * kStageStep;
        if (elected()) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            mma_pair_ss(d, ad + a_step * e, bd + b_step * e, idesc, e != 0 || q != 0 ? 1u : 0u);
            if constexpr (Ring<Args>::kA == 2)
              mma_pair_ss(d + kTileCols, ad + (kHalfBytes >> 4) + a_step * e, bd + b_step * e, idesc,
                          e != 0 || q != 0 ? 1u : 0u);
          }
          commit_both(&sh.empty[stage]);
          if (q + 1 == t.n) commit_both(&sh.acc_full[acc]);
        }
        __syncwarp();
        if (++stage == kStages) {
          stage = 0;
          parity ^= 1u;
        }
      }
      if (++acc == bufs) {
        acc = 0;
        acc_parity ^= 1u;
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
    const int half = (warp - 2) >> 2;
    Boxes boxes{smem + kRing + (warp - 2) * kBoxes * kBoxBytes};
    int acc = 0;
    uint32_t parity = 0;
    bool ok = true;
    Tile t;
    for (int k = 0; tile_at(a, pair, pairs, k, &t); ++k) {
      if (ok && !warp_wait(&sh.acc_full[acc], parity, abort)) {
        ok = false;                            // this tile and the later ones: NaN, and no more waits
        if (lane == 0) give_up(sh, status);
      }
      tc_fence_after();
      finish(a, t, tmem + ((uint32_t)(32 * g) << 16) + acc_at<Args>(acc), half,
             t.i0 + 128 * (int)rank + 32 * g, (int)rank * kEpiWarps + warp - 2, !ok, boxes);
      if (!ok) continue;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_leader(&sh.acc_empty[acc]);
      if (++acc == bufs) {
        acc = 0;
        parity ^= 1u;
      }
    }
    if (lane == 0) bulk_wait_all();
  }

  tc_fence_before();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, kTmemCols);
  }
}

template <typename Args>
cudaError_t launch(const Args& a, int32_t pairs, uint32_t* status, cudaStream_t s) {
  const cudaError_t e = cudaFuncSetAttribute(gated_kernel<Args>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
  if (e != cudaSuccess) return e;
  return launch_dependent(gated_kernel<Args>, 2u * (unsigned)pairs, kThreads, kSmem, s, 1, true, a, status);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

int32_t gated_max_pairs() {
  static int32_t pairs[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  if (pairs[dev] > 0) return pairs[dev];
  int32_t least = kGatedMaxPairs;
  const auto ask = [&](auto kernel) {
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
      clusters = 0;
    least = std::min(least, (int32_t)clusters);
  };
  ask(gated_kernel<GatedForward>);
  ask(gated_kernel<GatedTurned>);
  ask(gated_kernel<GatedBackward>);
  return pairs[dev] = least;
}

int32_t gated_box_rows(int64_t T) { return (int32_t)std::min<int64_t>(128, (T + 7) / 8 * 8); }

// The busiest pair's cycles: rounds of tiles, each D / 64 stages that take the longer of their
// MMAs (128 cycles for 16 of K and N = 256, and not below 90) and their operands' way from L2 (~54
// bytes a cycle), and epilogues of ~100 cycles a column, under the next tile's stages where there
// are two accumulators.  Measured, the one kind of tile against the other (D = 4096, F = 11008): 256
// tokens 41 us, turned 46; 300 57, 56; 512 58, 65; 4096 366, 397; and 777 x 5120 x 13824 149, 130.
// (Up to 128 tokens zo_gated_few.cu is faster than either: 31 us at one token, 38 and 35 here.)
GatedPlan gated_plan(int64_t T, int64_t D, int64_t F, int32_t pairs) {
  GatedPlan best{128, 0};
  int64_t least = INT64_MAX;
  const int64_t stages = ceil_div(D, 64);
  const auto consider = [&](GatedPlan p, int64_t tiles, int64_t mma, int64_t bytes, int64_t epilogue, bool alone) {
    const int64_t rounds = ceil_div(tiles, pairs);
    const int64_t products = stages * std::max<int64_t>(mma, bytes / 54) + 600;
    const int64_t cycles = alone ? rounds * (products + epilogue)
                                 : rounds * std::max(products, epilogue) + std::min(products, epilogue);
    if (cycles < least) {
      least = cycles;
      best = p;
    }
  };
  for (int32_t side = 128; side >= 16; side -= 16)
    consider({side, 0}, ceil_div(T, kTileRows) * ceil_div(F, side), std::max<int64_t>(4 * side, 360),
             kHalfBytes + side * 128, 100 * side, false);
  for (int32_t tokens = 256; tokens >= 32; tokens -= 16)
    consider({0, tokens}, ceil_div(T, tokens) * ceil_div(F, kTileRows), std::max<int64_t>(4 * tokens, 720),
             2 * kHalfBytes + tokens * 64, 100 * tokens, tokens > 128);
  return best;
}

int64_t gated_dx_tiles(int64_t T, int64_t D) { return ceil_div(T, kTileRows) * ceil_div(D, kTileCols); }

int32_t gated_parts(int64_t T, int64_t D, int64_t F) {
  constexpr int64_t kPairs = 76;
  const int64_t tiles = gated_dx_tiles(T, D), stages = 2 * ceil_div(F, 64);
  int32_t parts = 1;
  while (2 * parts <= kGatedMaxParts && 2 * parts * tiles <= kPairs && 16 * parts <= stages) parts *= 2;
  return parts;
}

void gated_deal(GatedBackward* a, bool want_x, bool want_w, int32_t pairs) {
  const int64_t cols = ceil_div(a->D, kTileCols);
  a->parts = gated_parts(a->T, a->D, a->F);
  a->n_dx = want_x ? (int32_t)(gated_dx_tiles(a->T, a->D) * a->parts) : 0;
  a->n_dw = want_w ? (int32_t)(2 * ceil_div(a->F, kTileRows) * cols) : 0;
  // stages of a tile, with what its beginning costs
  const int64_t deep = 2 * ceil_div(a->F, 64) / a->parts + 4, flat = (a->twin ? 2 : 1) * ceil_div(a->T, 64) + 4;
  const int64_t late = a->n_dx % pairs;
  a->skip = late == 0 ? 0 : (int32_t)std::min<int64_t>((deep + flat / 2) / flat, ceil_div(a->n_dw, pairs - late));
}

cudaError_t launch_gated_forward(const GatedForward& a, int32_t pairs, uint32_t* status, cudaStream_t s) {
  const int64_t tiles = ceil_div(a.T, kTileRows) * ceil_div(a.F, a.side);
  return launch(a, (int32_t)std::min<int64_t>(pairs, tiles), status, s);
}

cudaError_t launch_gated_turned(const GatedTurned& a, int32_t pairs, uint32_t* status, cudaStream_t s) {
  const int64_t tiles = ceil_div(a.T, a.tokens) * ceil_div(a.F, kTileRows);
  return launch(a, (int32_t)std::min<int64_t>(pairs, tiles), status, s);
}

cudaError_t launch_gated_backward(const GatedBackward& a, int32_t pairs, uint32_t* status, cudaStream_t s) {
  return launch(a, pairs, status, s);
}

}  // namespace zo
