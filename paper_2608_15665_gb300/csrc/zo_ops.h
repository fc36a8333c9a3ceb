// Host-side launchers of the first-order operators (internal to the library): layer
// normalisation, Newton-Schulz orthogonalisation with the Muon update, and the products of the
// gated linear block.
#pragma once

#include <cstdint>

#include <cuda.h>
#include <cuda_runtime.h>

namespace zo {

// ---- layer normalisation (zo_layernorm.cu) ------------------------------------------
struct LayerNormArgs {
  // forward: x (+ r) -> h = rnd(x + r) (only with r), y, mean, rstd (either may be null)
  // backward: dy, x (= h), mean, rstd (+ dr) -> dx, dweight, dbias
  const void *x, *r, *dy;
  const void *weight, *bias;      // null: 1 and 0
  void *y, *h, *dx;
  float *mean, *rstd;
  void *dweight, *dbias;          // null: not wanted
  float* partial;                 // backward: layernorm_partial_rows() x 2 x cols sums
  int64_t rows, cols;
  int64_t ldx, ldr, lddy, ldy, ldh, lddx;
  int32_t dtype, wdtype;          // of x, r, y, h, dy, dx, dr; of weight, bias, dweight, dbias
  float eps;
  uint32_t* status;               // set where a wait has run out
};

cudaError_t launch_layernorm_forward(const LayerNormArgs& a, int32_t sms, cudaStream_t s);
// CTAs of the backward pass: rows of the partial sums of dweight and of dbias
int64_t layernorm_partial_rows(int64_t rows, int64_t cols, int32_t sms);
cudaError_t launch_layernorm_backward(const LayerNormArgs& a, int32_t sms, cudaStream_t s);

// ---- Newton-Schulz orthogonalisation and the Muon update (zo_ortho.cu) ----------------
// One matrix: U (m x n) is worked on as X (p x c, p = min(m, n)), transposed where m > n.
// Iterates are held as fp16 values of x 2^e, with e of the step (OrthoStep).
struct OrthoMat {
  const void* G;
  void* W;
  float* M;
  int64_t ldg, ldw, m, n, p, c;
  int32_t grad_bf16, bf16, tall;
  int32_t pairs;                    // products of hi + lo pairs (ortho_pairs)
  int32_t small;                    // its cluster's CTAs in a one-launch kernel, which uses
                                    // none of the fields below; 0: the others'
  int32_t maps;                     // index of its kOrthoMaps tensor maps
  int32_t unit0, n_units;           // its slots of the norm's partial sums
  int32_t wide_rows;                // W's rows start on 16 bytes
  int64_t ldx, ldp;                 // row strides of X, and of A and B (multiples of 64)
  uint16_t *xh[2], *xl[2];          // X_k in xh[k & 1], xl[k & 1].  Without pairs no other
                                    // tile reads an element's lo part: one buffer serves both
  uint16_t *ah, *al, *bh, *bl;      // A and B = b A + c A A (lo parts only with pairs)
};
// kOrthoUnitRows x kOrthoUnitCols elements of U: (matrix, first row, first column, slot)
constexpr int kOrthoUnitRows = 32, kOrthoUnitCols = 256;
// A tile of a product, kOrthoTileRows x ortho_tile_cols(): stages [k0, k1) of 64 of K.  Where few
// deep tiles would leave SM pairs idle, a tile's K is split: its parts share a slot of counters,
// their sums lie side by side, and the last one to finish adds them up.
struct OrthoTile {
  int32_t mat, i0, j0, maps;        // matrix, first row and column, index of its tensor maps
  int32_t k0, k1;
  int32_t slot, part, parts;        // parts > 1: one of a split tile's
  int32_t sum0;                     // the first of its parts' sums, in ortho_part_floats()
};
constexpr int kOrthoTileRows = 256, kOrthoMaxParts = 8;
__host__ __device__ constexpr int ortho_tile_cols(bool pairs, bool narrow) {
  return (pairs ? 128 : 256) / (narrow ? 2 : 1);
}
// floats of one part's sums, and a slot's counters (one for each of 8 epilogue warps of two CTAs)
__host__ __device__ constexpr int64_t ortho_part_floats(bool pairs, bool narrow) {
  return (int64_t)kOrthoTileRows * ortho_tile_cols(pairs, narrow);
}
constexpr int kOrthoSlotCounters = 16;

// Tensor maps of one matrix: 64 x 64 loads of X_k (hi of even and odd k, lo of even and odd
// k), of A and of B (hi, lo), and the 32 x 32 stores in the same order.
enum OrthoMap : int32_t {
  kMapX = 0, kMapA = 4, kMapB = 6, kMapStoreX = 8, kMapStoreA = 12, kMapStoreB = 14,
  kOrthoMaps = 16
};

enum OrthoPhase : int32_t { kOrthoGram = 0, kOrthoPoly = 1, kOrthoApply = 2 };

struct OrthoStep {
  float a, b, c;
  int32_t ex, ea, eb;               // exponents of X_k, A and B
  int32_t ex_next;                  // of X_(k+1)
  int32_t k;                        // index of the step: X_k is in xh[k & 1]
  int32_t last;                     // the result goes to W instead of X_(k+1)
};
constexpr int kOrthoMaxSteps = 32;
// The steps of a call with the exponents of their iterates (zo_muon.cu); coeffs: 3 per step, or
// null for the quintic.  False, with zo_last_error set: steps out of range, or coefficients
// under which the iterates can leave the range they are held in.
bool plan_ortho_steps(int32_t steps, const float* coeffs, OrthoStep* out);

// A mode of the coefficient kernel beside CoeffMode: C_i holds D_i, and becomes
// -lr D_i + restore_coef eps Z_i^(restore_query).
constexpr int32_t kCoeffFromDirection = 2;

struct OrthoUpdate {
  float momentum;
  int32_t step;                     // 0: U = G, W <- NS(U); 1: the Muon update
  int32_t nesterov, adjust;
  float keep, lr;                   // W <- keep W - lr s NS(U)
  float eps;
};

// fp32 results take products of fp32 grade.  So do bf16 results of at most 128 rows: their few
// singular directions do not average rounding out (8 x 8: 4.1e-3 of the result's norm with
// single factors, rounding the result 1.7e-3), and their time is latency, not products.  Larger
// bf16 matrices take single factors (1.1 to 1.3 times the rounding's error for gradients, 1.2 to 1.5
// times for Gaussian matrices, whose spectra are flat) unless their caller asks for pairs (4096 x
// 4096: 2.81 ms instead of 0.96; 96 of 256 x 256 327 us instead of 196, eight 103 instead of 95).
inline bool ortho_pairs(bool bf16, int64_t p) { return !bf16 || p <= 128; }

// partial: one per unit; counter (zero before the first call) and inverse (a power of two, and
// what U is multiplied by after it): one per matrix
cudaError_t launch_ortho_momentum(const OrthoMat* mats, const int4* units, int32_t n_units,
                                  const OrthoUpdate& u, double* partial, uint32_t* counter,
                                  float2* inverse, cudaStream_t s);
cudaError_t launch_ortho_scale(const OrthoMat* mats, const int4* units, int32_t n_units,
                               const OrthoUpdate& u, int32_t ex, const float2* inverse,
                               cudaStream_t s);
// Clusters of the product kernels that fit on the device at once
int32_t ortho_max_pairs();
constexpr int kOrthoMaxPairs = 128;
// pair q of n_pairs takes the tiles first[q] .. first[q + 1] - 1
// sums, counters: of the split tiles' slots (counters are zero between launches)
cudaError_t launch_ortho_product(const OrthoMat* mats, const CUtensorMap* maps,
                                 const OrthoTile* tiles, const int32_t* first, float* sums,
                                 uint32_t* counters, bool pairs, bool narrow, int32_t n_pairs,
                                 OrthoPhase phase, const OrthoStep& st, const OrthoUpdate& u,
                                 uint32_t* status, cudaStream_t s);

// Matrices of at most 64 rows (zo_ortho_mma.cu, `rows` = 16, 32 or 64) and of 65 to 128
// (zo_ortho_small.cu), each kind in one launch: the CTAs of a matrix's cluster
// (0: not one of these, or too wide), and a CTA's shared memory.  A launch takes the matrices
// mats[which[0 .. n)], all of one cluster size (and rows), and the largest of their shared
// memories.
int32_t ortho_mma_rows(int64_t p);
int32_t ortho_mma_cluster(int64_t p, int64_t c);
int32_t ortho_mma_smem(int64_t p, int64_t c, int32_t cluster);
cudaError_t launch_ortho_mma(const OrthoMat* mats, const int* which, int32_t n, int32_t rows,
                             int32_t cluster, int32_t smem, const OrthoStep* steps,
                             int32_t n_steps, const OrthoUpdate& u, cudaStream_t s);
int32_t ortho_small_cluster(int64_t p, int64_t c);
int32_t ortho_small_smem(int64_t p, int64_t c, int32_t cluster);
cudaError_t launch_ortho_small(const OrthoMat* mats, const int* which, int32_t n, int32_t cluster,
                               int32_t smem, const OrthoStep* steps, int32_t n_steps,
                               const OrthoUpdate& u, uint32_t* status, cudaStream_t s);

// ---- gated linear block (zo_gated.cu; its products in zo_gated_gemm.cu) ----------------
// All bf16.  Forward: G = X Wg^T, U = X Wu^T, H = act(G) U.  Backward, from dG and dU:
// dX = dG Wg + dU Wu, dWg = dG^T X, dWu = dU^T X.
constexpr int kGatedMaxPairs = 128;
enum GatedAct : int32_t { kGatedSilu = 0, kGatedGelu = 1 };

// act(g) = g s with s = sig(g) (SiLU) or sig(2 sqrt(2 / pi) (g + 0.044715 g^3)) (GELU by tanh: half of
// 1 + tanh(y) is sig(2 y), without the cancellation at negative y).  The exponential's argument:
#ifdef __CUDACC__
__device__ __forceinline__ float gated_gate(float g, int32_t act) {
  const float y = act == kGatedSilu ? g : 1.5957691216057308f * g * fmaf(0.044715f * g, g, 1.0f);
  float e, s;                       // (without the library forms' care for subnormal numbers)
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-1.4426950408889634f * y));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + e));
  return s;
}
#endif

struct GatedForward {
  CUtensorMap x, w[2], out[3];      // X; Wg and Wu; H, G and U
  int32_t T, D, F, act, save;
  int32_t side;                     // columns of Wg (and of Wu) to a tile
};
// the same with the tokens as the products' columns
struct GatedTurned {
  CUtensorMap x, w[2], out[3];
  int32_t T, D, F, act, save;
  int32_t tokens;                   // of a tile: a multiple of 16
};
// the same for at most 128 tokens (zo_gated_few.cu)
struct GatedFew {
  CUtensorMap x, w[2];
  uint16_t* out[3];                 // H, G and U
  int64_t ld[3];
  int32_t T, D, F, act, save;
  int32_t cols, box_rows;           // of a CTA: columns of H; tokens in a box of X
  int32_t stages, tmem_cols;
};
struct GatedBackward {
  CUtensorMap d_rows[2], w_cols[2], dx;           // dX: dG, dU along F; Wg, Wu by rows of F
  CUtensorMap d_cols[2][2], x_cols, dw[2];        // dW: dG, dU and X by rows of T
  int32_t T, D, F;
  int32_t twin;                     // dG and dU are sums of two bf16, in rows 2 t and 2 t + 1; their
                                    // columns' maps: [0] of the first parts, [1] of the second
  uint16_t* dx_rows;                // twin: dX, by plain stores
  int64_t lddx;
  int32_t box_rows;                 // tokens in a box of dG's and dU's rows
  int32_t n_dx, n_dw;               // tiles of dX, times parts, and of both dW (0: not wanted)
  int32_t parts;                    // of the K of a tile of dX
  float* sums;                      // parts > 1: kGatedPartFloats of every part of every tile,
  uint32_t* counters;               // and kGatedCounters of every tile, zero before the launch
  int32_t skip;                     // rounds of dW's tiles that take as long as a tile of dX
};
// columns and rows of a box of a result (of turned tiles: the other way round); tokens in a box of an
// operand: at most a CTA's 128
constexpr int kGatedOutCols = 16, kGatedOutRows = 32;
int32_t gated_box_rows(int64_t T);
// The tiles of a call: `side` columns of each half, or (side = 0) `tokens` tokens to a turned tile
struct GatedPlan {
  int32_t side, tokens;
};
GatedPlan gated_plan(int64_t T, int64_t D, int64_t F, int32_t pairs);
// SM pairs that run at once, or 0
int32_t gated_max_pairs();
// Parts of the K of dX's tiles: where the tiles leave half of a GB300's SM pairs or more without one,
// as many as they have room for, each of eight stages at least.  By the sizes alone: the sums' order
// does not depend on the device.
constexpr int kGatedMaxParts = 8, kGatedCounters = 16;
constexpr int64_t kGatedPartFloats = 256 * 256;
int64_t gated_dx_tiles(int64_t T, int64_t D);
// Up to a CTA's 128 tokens a tile's other 128 rows are idle: dG and dU take two rows a token.
inline bool gated_twin(int64_t T) { return T <= 128; }
int32_t gated_parts(int64_t T, int64_t D, int64_t F);
// fills n_dx, n_dw, parts and skip
void gated_deal(GatedBackward* a, bool want_x, bool want_w, int32_t pairs);
cudaError_t launch_gated_forward(const GatedForward& a, int32_t pairs, uint32_t* status, cudaStream_t s);
// fills cols, box_rows, stages and tmem_cols; false: more than 128 tokens
bool gated_few_plan(GatedFew* a, int32_t sms);
cudaError_t launch_gated_few(const GatedFew& a, uint32_t* status, cudaStream_t s);
cudaError_t launch_gated_turned(const GatedTurned& a, int32_t pairs, uint32_t* status, cudaStream_t s);
cudaError_t launch_gated_backward(const GatedBackward& a, int32_t pairs, uint32_t* status, cudaStream_t s);

}  // namespace zo
