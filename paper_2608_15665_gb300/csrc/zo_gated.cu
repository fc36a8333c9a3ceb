// The gated linear block of a feed-forward layer (C ABI: include/zo.h): checks, tensor maps, the
// backward pass's elementwise kernel, and the launches of the products (zo_gated_gemm.cu).
//
//   forward:  G = X Wg^T, U = X Wu^T, H = act(G) U                  one launch
//   backward: dG = dH U act'(G), dU = dH act(G)                     one launch, into the workspace
//             dX = dG Wg + dU Wu, dWg = dG^T X, dWu = dU^T X        one launch
//
// dG and dU are rounded to bf16 for the products, as X and the weights are: each product then errs
// by its terms' 2^-9 in random directions, about what rounding its result costs again (of 4096 tokens
// 2.3e-3 of the result's norm, 1.7e-3 by the last rounding alone).  Up to 128 tokens they are kept as
// sums of two bf16, which costs nothing there.
#include <algorithm>
#include <cmath>

#include <cuda_bf16.h>

#include "../../include/zo.h"
#include "zo_host.h"
#include "zo_launch.cuh"
#include "zo_ops.h"

namespace {

using namespace zo::host;

// Set by a product whose wait has run out; one per device.
__device__ uint32_t g_gated_status;

uint32_t* status_word() {
  static uint32_t* word[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
  if (word[dev] == nullptr) {
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_gated_status) != cudaSuccess) return nullptr;
    word[dev] = static_cast<uint32_t*>(p);
  }
  return word[dev];
}

constexpr int kThreads = 256;

struct Gradients {
  const uint16_t *dh, *g, *u;
  uint16_t *dg, *du;                  // rows of F without gaps; twin: two a token
  int64_t lddh, ldg, ldu;
  uint32_t vectors, per_row;          // of 8 elements
  int32_t act, twin;
  uint32_t* counters;                 // of the products' split tiles: zero before them
  uint32_t n_counters;
};

__device__ __forceinline__ float value(const uint4& v, int i) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
}
__device__ __forceinline__ uint4 packed(const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// dG and dU: bound by HBM (three reads, two writes).
__global__ void __launch_bounds__(kThreads) gated_gradients_kernel(const Gradients a) {
  const uint32_t at = blockIdx.x * kThreads + threadIdx.x;
  zo::pdl_wait();
  zo::pdl_trigger();
  for (uint32_t i = at; i < a.n_counters; i += gridDim.x * kThreads) a.counters[i] = 0;
  if (at >= a.vectors) return;
  const int64_t row = at / a.per_row, col = 8 * (int64_t)(at % a.per_row);
  const uint4 dh = __ldcs(reinterpret_cast<const uint4*>(a.dh + row * a.lddh + col));
  const uint4 g = __ldcs(reinterpret_cast<const uint4*>(a.g + row * a.ldg + col));
  const uint4 u = __ldcs(reinterpret_cast<const uint4*>(a.u + row * a.ldu + col));
  float dg[8], du[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = value(g, i), d = value(dh, i);
    const float s = zo::gated_gate(x, a.act);
    // the argument's derivative: 1, or 2 sqrt(2 / pi) (1 + 3 0.044715 x^2), of which no more than
    // |x| = 64 is needed: s is 0 or 1 there, and x's powers stay in range
    const float z = a.act == zo::kGatedSilu ? x : fminf(fmaxf(x, -64.0f), 64.0f);
    const float y1 = a.act == zo::kGatedSilu ? 1.0f : fmaf(0.2140644488f * z, z, 1.5957691216f);
    const float slope = s * fmaf(z * y1, 1.0f - s, 1.0f) + (x - x);   // (NaN and infinity stay NaN)
    dg[i] = d * value(u, i) * slope;
    du[i] = d * x * s;
  }
  const int64_t F = 8 * (int64_t)a.per_row, out = (a.twin ? 2 : 1) * row * F + col;
  const auto store = [&](uint16_t* to, float (&v)[8]) {
    const uint4 hi = packed(v);
    *reinterpret_cast<uint4*>(to + out) = hi;
    if (!a.twin) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float rest = v[i] - value(hi, i);
      // (infinities stay in the first row, those that the rounding makes as well)
      v[i] = fabsf(rest) < __int_as_float(0x7F800000) ? rest : 0.0f;
    }
    *reinterpret_cast<uint4*>(to + out + F) = packed(v);
  };
  store(a.dg, dg);
  store(a.du, du);
}

constexpr int64_t kMaxExtent = int64_t(1) << 24;

zo_status check_sizes(int64_t T, int64_t D, int64_t F, int32_t act) {
  if (act != ZO_GATED_SILU && act != ZO_GATED_GELU_TANH)
    return refuse(ZO_ERR_INVALID_ARG, "zo_gated: unknown activation");
  if (T < 0 || T >= kMaxExtent || D < 8 || D >= kMaxExtent || F < 8 || F >= kMaxExtent ||
      D % 8 != 0 || F % 8 != 0 || (T > 0 && F > (int64_t(1) << 34) / T) ||
      (T > 0 && D > (int64_t(1) << 34) / T) || F > (int64_t(1) << 37) / D)
    return refuse(ZO_ERR_SHAPE, "zo_gated: need 0 <= T < 2^24, D and F multiples of 8 below 2^24, "
                                "T D, T F <= 2^34 and D F <= 2^37");
  return ZO_OK;
}

// A bf16 matrix with rows of `cols`: 16-byte aligned, its stride a multiple of 8.
struct Buffer {
  const void* p;
  int64_t ld, cols;
};
zo_status check_buffers(const Buffer* b, int n) {
  for (int i = 0; i < n; ++i) {
    if (!b[i].p) return refuse(ZO_ERR_INVALID_ARG, "zo_gated: a null matrix");
    if (b[i].ld < b[i].cols || b[i].ld >= (int64_t(1) << 38))
      return refuse(ZO_ERR_SHAPE, "zo_gated: a row stride is smaller than its row, or too large");
    if (!aligned16(b[i].p) || b[i].ld % 8 != 0)
      return refuse(ZO_ERR_ALIGN, "zo_gated: matrices must be 16-byte aligned with strides of multiples of 8");
  }
  return ZO_OK;
}

bool map_of(CUtensorMap* m, const void* p, int64_t cols, int64_t rows, int64_t ld, uint32_t box_cols,
            uint32_t box_rows, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
  return encode_bf16_2d(m, const_cast<void*>(p), (uint64_t)cols, (uint64_t)rows, (uint64_t)ld * 2,
                        box_cols, box_rows, swizzle);
}
bool out_map(CUtensorMap* m, void* p, int64_t cols, int64_t rows, int64_t ld) {
  return map_of(m, p, cols, rows, ld, zo::kGatedOutCols, zo::kGatedOutRows, CU_TENSOR_MAP_SWIZZLE_32B);
}

int64_t round_up(int64_t v) { return (v + 255) / 256 * 256; }
int64_t gradient_bytes(int64_t T, int64_t F) { return round_up((zo::gated_twin(T) ? 2 : 1) * T * F * 2); }

// The workspace: dG, dU, then what the split tiles of dX take.
struct Layout {
  int64_t sums_at, counters_at, counters, bytes;
};
Layout layout(int64_t T, int64_t D, int64_t F) {
  const int64_t parts = zo::gated_parts(T, D, F), tiles = parts > 1 ? zo::gated_dx_tiles(T, D) : 0;
  Layout L;
  L.sums_at = 2 * gradient_bytes(T, F);
  L.counters_at = L.sums_at + tiles * parts * zo::kGatedPartFloats * (int64_t)sizeof(float);
  L.counters = tiles * zo::kGatedCounters;
  L.bytes = L.counters_at + round_up(L.counters * (int64_t)sizeof(uint32_t));
  return L;
}

}  // namespace

extern "C" {

zo_status zo_gated_forward(const void* X, int64_t ldx, int64_t T, int64_t D, const void* Wg,
                           int64_t ldwg, const void* Wu, int64_t ldwu, int64_t F, int32_t act,
                           void* H, int64_t ldh, void* G, int64_t ldg, void* U, int64_t ldu,
                           void* stream) {
  zo_status st = check_sizes(T, D, F, act);
  if (st != ZO_OK) return st;
  if ((G == nullptr) != (U == nullptr))
    return refuse(ZO_ERR_INVALID_ARG, "zo_gated_forward: G and U are kept together, or neither");
  if (T == 0) return ZO_OK;
  const Buffer all[6] = {{X, ldx, D}, {Wg, ldwg, D}, {Wu, ldwu, D}, {H, ldh, F}, {G, ldg, F}, {U, ldu, F}};
  st = check_buffers(all, G ? 6 : 4);
  if (st != ZO_OK) return st;
  const int32_t pairs = zo::gated_max_pairs();
  uint32_t* status = status_word();
  if (pairs <= 0 || !status) return refuse(ZO_ERR_CUDA, "zo_gated_forward: no usable CUDA device");
  void* const out[3] = {H, G, U};
  const int64_t ld[3] = {ldh, ldg, ldu};
  const int outs = G ? 3 : 1;
  const auto s = reinterpret_cast<cudaStream_t>(stream);
  const char* const no_map = "zo_gated_forward: cuTensorMapEncodeTiled rejected a descriptor";
  const auto sizes = [&](auto& a) {
    a.T = (int32_t)T;
    a.D = (int32_t)D;
    a.F = (int32_t)F;
    a.act = act == ZO_GATED_SILU ? zo::kGatedSilu : zo::kGatedGelu;
    a.save = G != nullptr;
  };
  const auto maps = [&](auto& a, uint32_t x_rows, uint32_t w_rows) {
    return map_of(&a.x, X, D, T, ldx, 64, x_rows) && map_of(&a.w[0], Wg, D, F, ldwg, 64, w_rows) &&
           map_of(&a.w[1], Wu, D, F, ldwu, 64, w_rows);
  };
  zo::GatedFew few{};
  sizes(few);
  if (zo::gated_few_plan(&few, 2 * pairs)) {
    for (int k = 0; k < outs; ++k) {
      few.out[k] = static_cast<uint16_t*>(out[k]);
      few.ld[k] = ld[k];
    }
    if (!maps(few, few.box_rows, few.cols)) return refuse(ZO_ERR_CUDA, no_map);
    ZO_CUDA(zo::launch_gated_few(few, status, s), "gated forward kernel");
    return ZO_OK;
  }
  const zo::GatedPlan plan = zo::gated_plan(T, D, F, pairs);
  if (plan.side == 0) {
    zo::GatedTurned a{};
    sizes(a);
    a.tokens = plan.tokens;
    bool ok = maps(a, plan.tokens / 2, 128);
    for (int k = 0; k < outs; ++k)
      ok = ok && map_of(&a.out[k], out[k], F, T, ld[k], zo::kGatedOutRows, zo::kGatedOutCols,
                        CU_TENSOR_MAP_SWIZZLE_64B);
    if (!ok) return refuse(ZO_ERR_CUDA, no_map);
    ZO_CUDA(zo::launch_gated_turned(a, pairs, status, s), "gated forward kernel");
  } else {
    zo::GatedForward a{};
    sizes(a);
    a.side = plan.side;
    bool ok = maps(a, 128, a.side);
    for (int k = 0; k < outs; ++k) ok = ok && out_map(&a.out[k], out[k], F, T, ld[k]);
    if (!ok) return refuse(ZO_ERR_CUDA, no_map);
    ZO_CUDA(zo::launch_gated_forward(a, pairs, status, s), "gated forward kernel");
  }
  return ZO_OK;
}

int64_t zo_gated_workspace(int64_t T, int64_t D, int64_t F) {
  return check_sizes(T, D, F, ZO_GATED_SILU) == ZO_OK && T > 0 ? layout(T, D, F).bytes : 0;
}

zo_status zo_gated_backward(const void* dH, int64_t lddh, const void* X, int64_t ldx, int64_t T,
                            int64_t D, const void* Wg, int64_t ldwg, const void* Wu, int64_t ldwu,
                            int64_t F, int32_t act, const void* G, int64_t ldg, const void* U,
                            int64_t ldu, void* dX, int64_t lddx, void* dWg, int64_t lddwg, void* dWu,
                            int64_t lddwu, void* workspace, int64_t workspace_bytes, void* stream) {
  zo_status st = check_sizes(T, D, F, act);
  if (st != ZO_OK) return st;
  if ((dWg == nullptr) != (dWu == nullptr))
    return refuse(ZO_ERR_INVALID_ARG, "zo_gated_backward: dWg and dWu are wanted together, or neither");
  const auto s = reinterpret_cast<cudaStream_t>(stream);
  const Buffer dw[2] = {{dWg, lddwg, D}, {dWu, lddwu, D}};
  if (dWg) {
    st = check_buffers(dw, 2);
    if (st != ZO_OK) return st;
  }
  if (T == 0) {                                    // sums over no tokens
    for (int k = 0; dWg && k < 2; ++k)
      ZO_CUDA(cudaMemset2DAsync(const_cast<void*>(dw[k].p), (size_t)dw[k].ld * 2, 0, (size_t)D * 2,
                                (size_t)F, s),
              "clear a gradient");
    return ZO_OK;
  }
  if (!dX && !dWg) return ZO_OK;
  const Buffer in[5] = {{dH, lddh, F}, {G, ldg, F}, {U, ldu, F}, {Wg, ldwg, D}, {Wu, ldwu, D}};
  st = check_buffers(in, dX ? 5 : 3);
  const Buffer x[2] = {{X, ldx, D}, {dX, lddx, D}};
  if (st == ZO_OK && dWg) st = check_buffers(x, 1);
  if (st == ZO_OK && dX) st = check_buffers(x + 1, 1);
  if (st != ZO_OK) return st;
  const Layout L = layout(T, D, F);
  if (!workspace || workspace_bytes < L.bytes)
    return refuse(ZO_ERR_INVALID_ARG, "zo_gated_backward: the workspace is missing or smaller than "
                                      "zo_gated_workspace(T, D, F)");
  if (!aligned16(workspace))
    return refuse(ZO_ERR_ALIGN, "zo_gated_backward: the workspace must be 16-byte aligned");
  const int32_t pairs = zo::gated_max_pairs();
  uint32_t* status = status_word();
  if (pairs <= 0 || !status) return refuse(ZO_ERR_CUDA, "zo_gated_backward: no usable CUDA device");
  Gradients e{};
  e.dh = static_cast<const uint16_t*>(dH);
  e.g = static_cast<const uint16_t*>(G);
  e.u = static_cast<const uint16_t*>(U);
  e.dg = static_cast<uint16_t*>(workspace);
  e.du = e.dg + gradient_bytes(T, F) / 2;
  e.lddh = lddh;
  e.ldg = ldg;
  e.ldu = ldu;
  e.per_row = (uint32_t)(F / 8);
  e.vectors = (uint32_t)(T * (F / 8));
  e.act = act == ZO_GATED_SILU ? zo::kGatedSilu : zo::kGatedGelu;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  e.counters = reinterpret_cast<uint32_t*>(ws + L.counters_at);
  e.n_counters = (uint32_t)L.counters;
  zo::GatedBackward a{};
  a.sums = reinterpret_cast<float*>(ws + L.sums_at);
  a.counters = e.counters;
  a.T = (int32_t)T;
  a.D = (int32_t)D;
  a.F = (int32_t)F;
  const int64_t twin = zo::gated_twin(T) ? 2 : 1;
  a.twin = e.twin = twin == 2;
  a.dx_rows = static_cast<uint16_t*>(dX);
  a.lddx = lddx;
  a.box_rows = zo::gated_box_rows(twin * T);
  const uint16_t* d[2] = {e.dg, e.du};
  const void* w[2] = {Wg, Wu};
  const int64_t ldw[2] = {ldwg, ldwu};
  bool ok = true;
  for (int k = 0; k < 2; ++k) {
    if (dX)
      ok = ok && map_of(&a.d_rows[k], d[k], F, twin * T, F, 64, a.box_rows) &&
           map_of(&a.w_cols[k], w[k], D, F, ldw[k], 64, 64);
    if (dWg)
      ok = ok && map_of(&a.d_cols[k][0], d[k], F, T, twin * F, 64, 64) &&
           (twin == 1 || map_of(&a.d_cols[k][1], d[k] + F, F, T, twin * F, 64, 64)) &&
           out_map(&a.dw[k], const_cast<void*>(dw[k].p), D, F, dw[k].ld);
  }
  if (dX) ok = ok && out_map(&a.dx, dX, D, T, lddx);
  if (dWg) ok = ok && map_of(&a.x_cols, X, D, T, ldx, 64, 64);
  if (!ok) return refuse(ZO_ERR_CUDA, "zo_gated_backward: cuTensorMapEncodeTiled rejected a descriptor");
  zo::gated_deal(&a, dX != nullptr, dWg != nullptr, pairs);
  ZO_CUDA(zo::launch_dependent(gated_gradients_kernel, (e.vectors + kThreads - 1) / kThreads, kThreads,
                               0, s, 1, true, e),
          "gated gradients kernel");
  ZO_CUDA(zo::launch_gated_backward(a, pairs, status, s), "gated backward kernel");
  return ZO_OK;
}

zo_status zo_gated_sync_status(void* stream) {
  const auto s = reinterpret_cast<cudaStream_t>(stream);
  uint32_t* word = status_word();
  if (!word) return refuse(ZO_ERR_CUDA, "zo_gated_sync_status: no usable CUDA device");
  uint32_t status = 0;
  ZO_CUDA(cudaMemcpyAsync(&status, word, sizeof(status), cudaMemcpyDeviceToHost, s), "read status");
  ZO_CUDA(cudaStreamSynchronize(s), "stream synchronize");
  if (status != 0) {
    ZO_CUDA(cudaMemsetAsync(word, 0, sizeof(status), s), "clear status");
    ZO_CUDA(cudaStreamSynchronize(s), "stream synchronize");
    return refuse(ZO_ERR_TIMEOUT, "gated linear block: a device-side wait ran out");
  }
  return ZO_OK;
}

}  // extern "C"
