// Layer normalisation over the rows of a matrix, forward and backward.
//
//   h = rnd(x + r) (r: an optional residual), mean = (1/N) sum_j h_j,
//   rstd = ((1/N) sum_j (h_j - mean)^2 + eps)^(-1/2),  xh = (h - mean) rstd,
//   y = xh w + b
// and with g = dy w
//   dx = rstd (g - (1/N) sum_j g_j - xh (1/N) sum_j g_j xh_j) (+ the residual's gradient),
//   dw = sum over rows of dy xh,  db = sum over rows of dy.
//
// Bound by HBM: x in, y out (forward), x and dy in, dx out (backward), so a row is read
// once into registers; the variance is the mean of the squared distances from the mean (a
// second sweep over registers), not a difference of moments that cancels where |mean| is
// large against the spread.  Sums, statistics and gradients are held in fp32 and every
// output is rounded once.
//
// A row belongs to a group of threads: a warp where its lanes hold it, else a whole CTA.
// Thread t of a group takes the chunks t, t + group, ... of VEC consecutive columns: 16
// bytes of the activations' type where every pointer, stride and the width allow it, else
// single elements.  Rows wider than a CTA's registers are swept from memory (kE = 0).
//
// Many rows: a few resident CTAs take the rows blockIdx, blockIdx + gridDim, ..., and what
// keeps HBM busy is a ring of rows per group in shared memory, filled by bulk copies several
// rows ahead.  A row that does not start or end on 16 bytes is copied with the rest of its
// first and last 16 (never past an aligned 16 bytes that hold a part of the row).  At 16384 x
// 5120 bf16 with a residual the backward pass took 271 us without the ring, 115 us with it.
// Few rows, one per group: straight from memory, which has the shorter latency.
//
// The backward pass keeps dw and db of a thread's own columns in registers over all its
// rows, so that each CTA writes one row of partial sums, which a second kernel adds up in a
// fixed order: no atomics, the same bits on every run.
#include <algorithm>

#include <cuda_bf16.h>

#include "zo_launch.cuh"
#include "zo_ops.h"
#include "zo_sm100.cuh"

namespace zo {
namespace {

constexpr int kF32 = 0;                 // ZO_F32; the other type is ZO_BF16

template <typename T> struct Elem;
template <> struct Elem<float> {
  static __device__ float to(float v) { return v; }
  static __device__ float from(float v) { return v; }
};
template <> struct Elem<__nv_bfloat16> {
  static __device__ float to(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __nv_bfloat16 from(float v) { return __float2bfloat16_rn(v); }
};

// V consecutive elements as floats.  kReadOnly: of buffers that no kernel writes meanwhile, so
// that the loads can be issued ahead of stores.
template <typename T, int V, bool kReadOnly = false>
__device__ __forceinline__ void load(const T* p, float (&v)[V]) {
  const auto get = [](const auto* q) {
    if constexpr (kReadOnly) return __ldg(q);
    else return *q;
  };
  if constexpr (V == 1) {
    v[0] = Elem<T>::to(get(p));
  } else if constexpr (sizeof(T) == 4) {
    static_assert(V % 4 == 0);
#pragma unroll
    for (int k = 0; k < V / 4; ++k) {
      const float4 q = get(reinterpret_cast<const float4*>(p) + k);
      v[4 * k] = q.x; v[4 * k + 1] = q.y; v[4 * k + 2] = q.z; v[4 * k + 3] = q.w;
    }
  } else if constexpr (V == 8) {
    const uint4 q = get(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(w[k] << 16);
      v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
  } else {
    static_assert(V == 4);
    const uint2 q = get(reinterpret_cast<const uint2*>(p));
    v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xFFFF0000u);
    v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xFFFF0000u);
  }
}
template <typename T, int V>
__device__ __forceinline__ void store(T* p, const float (&v)[V]) {
  if constexpr (V == 1) {
    *p = Elem<T>::from(v[0]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < V / 4; ++k)
      reinterpret_cast<float4*>(p)[k] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
  } else {
    uint32_t w[V / 2];
#pragma unroll
    for (int k = 0; k < V / 2; ++k) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
      w[k] = *reinterpret_cast<const uint32_t*>(&b);
    }
    if constexpr (V == 8) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sum over the group (a warp, or the whole CTA of kGroup threads), in every thread.  `buf`
// holds one value per warp; two calls in a row take different buffers.
template <int kGroup>
__device__ __forceinline__ float group_sum(float v, float* buf) {
  v = warp_sum(v);
  if constexpr (kGroup == 32) {
    return v;
  } else {
    constexpr int kWarps = kGroup / 32;
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_sum(lane < kWarps ? buf[lane] : 0.0f);
  }
}

// threads of a CTA whose rows take `group` threads each
__host__ __device__ constexpr int block_of(int group) { return group == 32 ? 128 : group; }

// resident CTAs of the many-row kernels on an SM: as many as leave a thread its columns' registers
__host__ __device__ constexpr int resident_of(int block) { return block <= 128 ? 3 : block <= 320 ? 2 : 1; }

// columns per thread and row, in registers: of a warp's rows, of a CTA's
constexpr int kWarpElems = 32, kCtaElems = 16;

// ------------------------------------------------------------------------------- ring
constexpr int kMaxStages = 8;
constexpr long long kWait = 4000000000LL;     // ~2 s at 2 GHz

// an untiled bulk copy of `bytes` (16-byte aligned, a multiple of 16) into shared memory
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
          sm100::smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(sm100::smem_u32(bar))
      : "memory");
}

// The rows of one group, `stages` of them in flight; up to three matrices, row `row` of each
// in one stage.  `slot` bytes hold a row and the rest of its first and last 16.
template <typename T>
struct Ring {
  const T* base[3];
  int64_t ld[3];
  int n, stages;
  uint32_t slot, bytes;
  uint8_t* smem;
  uint64_t* full;
  int stage = 0;
  uint32_t phase = 0;

  __device__ const T* row_of(int m, int64_t row) const { return base[m] + row * ld[m]; }
  static __device__ uint32_t lead(const T* p) { return (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u); }
  // by one thread of the group
  __device__ void fetch(int64_t row, int s) const {
    uint8_t* dst = smem + (size_t)s * n * slot;
    uint32_t total = 0, part[3];
#pragma unroll
    for (int m = 0; m < 3; ++m) {
      part[m] = m < n ? (lead(row_of(m, row)) + bytes + 15u) & ~15u : 0u;
      total += part[m];
    }
    sm100::mbar_arrive_expect_tx(&full[s], total);
#pragma unroll
    for (int m = 0; m < 3; ++m)
      if (m < n) {
        const T* p = row_of(m, row);
        bulk_load(dst + m * slot, reinterpret_cast<const uint8_t*>(p) - lead(p), part[m], &full[s]);
      }
  }
  // the matrices' pointers to row `row`: in shared memory (or, should the copies not have
  // come, in memory itself)
  __device__ void take(int64_t row, const T* (&p)[3]) const {
    const bool here = sm100::mbar_wait_bounded(&full[stage], phase, nullptr, kWait);
    const uint8_t* src = smem + (size_t)stage * n * slot;
#pragma unroll
    for (int m = 0; m < 3; ++m) {
      const T* q = m < n ? row_of(m, row) : nullptr;
      p[m] = m < n && here ? reinterpret_cast<const T*>(src + m * slot + lead(q)) : q;
    }
  }
  __device__ void advance() {
    if (++stage == stages) {
      stage = 0;
      phase ^= 1u;
    }
  }
};

// ---------------------------------------------------------------------------- forward
template <typename T, typename TW, int kGroup, int kE, int V>
__global__ void __launch_bounds__(block_of(kGroup))
forward_kernel(const LayerNormArgs a) {
  constexpr int kBlock = block_of(kGroup), kRows = kBlock / kGroup;
  __shared__ float buf[2][32];
  const int t = threadIdx.x % kGroup;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kGroup;
  pdl_wait();
  pdl_trigger();
  if (row >= a.rows) return;                    // whole groups: kRows > 1 only for warps
  const int64_t cols = a.cols;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* r = a.r ? static_cast<const T*>(a.r) + row * a.ldr : nullptr;
  T* h = a.r ? static_cast<T*>(a.h) + row * a.ldh : nullptr;
  T* y = static_cast<T*>(a.y) + row * a.ldy;
  const TW* w = static_cast<const TW*>(a.weight);
  const TW* b = static_cast<const TW*>(a.bias);
  const float inv_n = 1.0f / (float)cols;

  auto fetch = [&](int64_t j, float (&v)[V]) {
    load<T, V, true>(x + j, v);
    if (r) {
      float q[V];
      load<T, V, true>(r + j, q);
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = Elem<T>::to(Elem<T>::from(v[k] + q[k]));
    }
  };
  auto finish = [&](int64_t j, const float (&v)[V], float mean, float rstd) {
    float wv[V], bv[V], o[V];
#pragma unroll
    for (int k = 0; k < V; ++k) { wv[k] = 1.0f; bv[k] = 0.0f; }
    if (w) load<TW, V, true>(w + j, wv);
    if (b) load<TW, V, true>(b + j, bv);
#pragma unroll
    for (int k = 0; k < V; ++k) o[k] = fmaf((v[k] - mean) * rstd, wv[k], bv[k]);
    store<T, V>(y + j, o);
  };

  float mean, rstd;
  if constexpr (kE > 0) {
    float v[kE][V];
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int64_t j = ((int64_t)e * kGroup + t) * V;
      if (j < cols) {
        fetch(j, v[e]);
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) v[e][k] = 0.0f;
      }
    }
#pragma unroll
    for (int e = 0; e < kE; ++e)
#pragma unroll
      for (int k = 0; k < V; ++k) s += v[e][k];
    if (h) {
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const int64_t j = ((int64_t)e * kGroup + t) * V;
        if (j < cols) store<T, V>(h + j, v[e]);
      }
    }
    mean = group_sum<kGroup>(s, buf[0]) * inv_n;
    float q = 0.0f;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int64_t j = ((int64_t)e * kGroup + t) * V;
      if (j < cols) {
#pragma unroll
        for (int k = 0; k < V; ++k) q = fmaf(v[e][k] - mean, v[e][k] - mean, q);
      }
    }
    rstd = 1.0f / sqrtf(group_sum<kGroup>(q, buf[1]) * inv_n + a.eps);
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int64_t j = ((int64_t)e * kGroup + t) * V;
      if (j < cols) finish(j, v[e], mean, rstd);
    }
  } else {
    float v[V], s = 0.0f, q = 0.0f;
    for (int64_t j = (int64_t)t * V; j < cols; j += (int64_t)kGroup * V) {
      fetch(j, v);
      if (h) store<T, V>(h + j, v);
#pragma unroll
      for (int k = 0; k < V; ++k) s += v[k];
    }
    mean = group_sum<kGroup>(s, buf[0]) * inv_n;
    for (int64_t j = (int64_t)t * V; j < cols; j += (int64_t)kGroup * V) {
      fetch(j, v);
#pragma unroll
      for (int k = 0; k < V; ++k) q = fmaf(v[k] - mean, v[k] - mean, q);
    }
    rstd = 1.0f / sqrtf(group_sum<kGroup>(q, buf[1]) * inv_n + a.eps);
    for (int64_t j = (int64_t)t * V; j < cols; j += (int64_t)kGroup * V) {
      fetch(j, v);
      finish(j, v, mean, rstd);
    }
  }
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

// Many rows: the group's rows by a ring; weight and bias stay in registers.
template <typename T, typename TW, int kGroup, int kE, int V>
__global__ void __launch_bounds__(block_of(kGroup), resident_of(block_of(kGroup)))
forward_ring_kernel(const LayerNormArgs a, int stages, uint32_t slot) {
  constexpr int kBlock = block_of(kGroup), kGroups = kBlock / kGroup;
  __shared__ float buf[2][2][32];
  __shared__ uint64_t full[kGroups][kMaxStages];
  extern __shared__ __align__(128) uint8_t dyn[];
  const int t = threadIdx.x % kGroup, grp = threadIdx.x / kGroup;
  const int64_t cols = a.cols;
  const float inv_n = 1.0f / (float)cols;
  Ring<T> ring{{static_cast<const T*>(a.x), static_cast<const T*>(a.r), nullptr},
               {a.ldx, a.ldr, 0}, a.r ? 2 : 1, stages, slot, (uint32_t)(cols * sizeof(T)),
               dyn + (size_t)grp * stages * (a.r ? 2 : 1) * slot, full[grp]};
  if (t == 0) {
    for (int s = 0; s < stages; ++s) sm100::mbar_init(&full[grp][s], 1);
    sm100::fence_mbar_init();
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const int64_t stride = (int64_t)gridDim.x * kGroups;
  const int64_t row0 = (int64_t)blockIdx.x * kGroups + grp;
  if (t == 0)
    for (int s = 0; s < stages; ++s)
      if (row0 + s * stride < a.rows) ring.fetch(row0 + s * stride, s);
  const TW* w = static_cast<const TW*>(a.weight);
  const TW* b = static_cast<const TW*>(a.bias);
  float wv[kE][V], bv[kE][V];
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    const int64_t j = ((int64_t)e * kGroup + t) * V;
#pragma unroll
    for (int k = 0; k < V; ++k) { wv[e][k] = 1.0f; bv[e][k] = 0.0f; }
    if (w && j < cols) load<TW, V, true>(w + j, wv[e]);
    if (b && j < cols) load<TW, V, true>(b + j, bv[e]);
  }
  int flip = 0;
  for (int64_t row = row0; row < a.rows; row += stride, flip ^= 1) {
    const T* src[3];
    ring.take(row, src);
    T* y = static_cast<T*>(a.y) + row * a.ldy;
    float v[kE][V];
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int64_t j = ((int64_t)e * kGroup + t) * V;
#pragma unroll
      for (int k = 0; k < V; ++k) v[e][k] = 0.0f;
      if (j < cols) {
        load<T, V>(src[0] + j, v[e]);
        if (a.r) {
          float q[V];
          load<T, V>(src[1] + j, q);
#pragma unroll
          for (int k = 0; k < V; ++k) v[e][k] = Elem<T>::to(Elem<T>::from(v[e][k] + q[k]));
          store<T, V>(static_cast<T*>(a.h) + row * a.ldh + j, v[e]);
        }
      }
#pragma unroll
      for (int k = 0; k < V; ++k) s += v[e][k];
    }
    const float mean = group_sum<kGroup>(s, buf[flip][0]) * inv_n;
    // every thread of the group has read the stage
    if (t == 0 && row + stages * stride < a.rows) ring.fetch(row + stages * stride, ring.stage);
    ring.advance();
    float q = 0.0f;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int64_t j = ((int64_t)e * kGroup + t) * V;
      if (j < cols) {
#pragma unroll
        for (int k = 0; k < V; ++k) q = fmaf(v[e][k] - mean, v[e][k] - mean, q);
      }
    }
    const float rstd = 1.0f / sqrtf(group_sum<kGroup>(q, buf[flip][1]) * inv_n + a.eps);
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int64_t j = ((int64_t)e * kGroup + t) * V;
      if (j < cols) {
#pragma unroll
        for (int k = 0; k < V; ++k) v[e][k] = fmaf((v[e][k] - mean) * rstd, wv[e][k], bv[e][k]);
        store<T, V>(y + j, v[e]);
      }
    }
    if (t == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

// --------------------------------------------------------------------------- backward
// Rows held in registers: each thread keeps its columns' weight, dw and db over all rows
// of its group.  kRing: the rows come through a ring, else straight from memory.
template <typename T, typename TW, int kGroup, int kE, int V, bool kRing>
__global__ void __launch_bounds__(block_of(kGroup), resident_of(block_of(kGroup)))
backward_kernel(const LayerNormArgs a, int stages, uint32_t slot) {
  constexpr int kBlock = block_of(kGroup), kGroups = kBlock / kGroup;
  static_assert(kE > 0, "rows in registers");
  __shared__ float buf[2][2][32];
  __shared__ uint64_t full[kGroups][kMaxStages];
  extern __shared__ __align__(128) uint8_t dyn[];   // the ring; then dw and db of each warp
  const int t = threadIdx.x % kGroup, grp = threadIdx.x / kGroup;
  const int64_t cols = a.cols;
  const float inv_n = 1.0f / (float)cols;
  Ring<T> ring{{static_cast<const T*>(a.x), static_cast<const T*>(a.dy), static_cast<const T*>(a.r)},
               {a.ldx, a.lddy, a.ldr}, a.r ? 3 : 2, stages, slot, (uint32_t)(cols * sizeof(T)),
               dyn + (size_t)grp * stages * (a.r ? 3 : 2) * slot, full[grp]};
  if constexpr (kRing) {
    if (t == 0) {
      for (int s = 0; s < stages; ++s) sm100::mbar_init(&full[grp][s], 1);
      sm100::fence_mbar_init();
    }
    __syncthreads();
  }
  pdl_wait();
  pdl_trigger();
  const TW* w = static_cast<const TW*>(a.weight);
  float wv[kE][V], dw[kE][V], db[kE][V];
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    const int64_t j = ((int64_t)e * kGroup + t) * V;
#pragma unroll
    for (int k = 0; k < V; ++k) { wv[e][k] = 1.0f; dw[e][k] = db[e][k] = 0.0f; }
    if (w && j < cols) load<TW, V, true>(w + j, wv[e]);
  }
  const int64_t stride = (int64_t)gridDim.x * kGroups;
  const int64_t row0 = (int64_t)blockIdx.x * kGroups + grp;
  if constexpr (kRing) {
    if (t == 0)
      for (int s = 0; s < stages; ++s)
        if (row0 + s * stride < a.rows) ring.fetch(row0 + s * stride, s);
  }
  int flip = 0;
  float mean_next = row0 < a.rows ? a.mean[row0] : 0.0f, rstd_next = row0 < a.rows ? a.rstd[row0] : 0.0f;
  for (int64_t row = row0; row < a.rows; row += stride, flip ^= 1) {
    const T* src[3] = {ring.row_of(0, row), ring.row_of(1, row), a.r ? ring.row_of(2, row) : nullptr};
    T* dx = static_cast<T*>(a.dx) + row * a.lddx;
    const float mean = mean_next, rstd = rstd_next;
    if (row + stride < a.rows) {
      mean_next = a.mean[row + stride];
      rstd_next = a.rstd[row + stride];
    }
    if constexpr (kRing) ring.take(row, src);
    float xh[kE][V], g[kE][V];
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int64_t j = ((int64_t)e * kGroup + t) * V;
      if (j < cols) {
        load<T, V>(src[0] + j, xh[e]);
        load<T, V>(src[1] + j, g[e]);
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) { xh[e][k] = mean; g[e][k] = 0.0f; }
      }
    }
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int e = 0; e < kE; ++e)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        xh[e][k] = (xh[e][k] - mean) * rstd;
        db[e][k] += g[e][k];
        dw[e][k] = fmaf(g[e][k], xh[e][k], dw[e][k]);
        g[e][k] *= wv[e][k];
        s1 += g[e][k];
        s2 = fmaf(g[e][k], xh[e][k], s2);
      }
    s1 = warp_sum(s1);
    s2 = warp_sum(s2);
    if constexpr (kGroup > 32) {
      constexpr int kWarps = kGroup / 32;
      if ((threadIdx.x & 31) == 0) {
        buf[flip][0][threadIdx.x >> 5] = s1;
        buf[flip][1][threadIdx.x >> 5] = s2;
      }
      __syncthreads();
      const int lane = threadIdx.x & 31;
      s1 = warp_sum(lane < kWarps ? buf[flip][0][lane] : 0.0f);
      s2 = warp_sum(lane < kWarps ? buf[flip][1][lane] : 0.0f);
    }
    s1 *= inv_n;
    s2 *= inv_n;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int64_t j = ((int64_t)e * kGroup + t) * V;
      if (j >= cols) continue;
      float o[V];
#pragma unroll
      for (int k = 0; k < V; ++k) o[k] = rstd * (g[e][k] - s1 - xh[e][k] * s2);
      if (a.r) {
        float q[V];
        load<T, V>(src[2] + j, q);
#pragma unroll
        for (int k = 0; k < V; ++k) o[k] += q[k];
      }
      store<T, V>(dx + j, o);
    }
    if constexpr (kRing) {
      // every thread of the group has read the stage: the row `stages` ahead may have it
      if constexpr (kGroup > 32) {
        if (a.r) __syncthreads();               // (dr was read behind the sums' barrier)
      } else {
        __syncwarp();
      }
      if (t == 0 && row + stages * stride < a.rows) ring.fetch(row + stages * stride, ring.stage);
      ring.advance();
    }
  }
  if (a.partial == nullptr) return;
  if constexpr (kGroups > 1) {
    // the warps' sums meet in shared memory, added in warp order
    float* joined = reinterpret_cast<float*>(dyn);
    const int width = kE * kGroup * V;
    __syncthreads();                            // the rings are no longer read
#pragma unroll
    for (int e = 0; e < kE; ++e)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        joined[(grp * 2 + 0) * width + (e * kGroup + t) * V + k] = dw[e][k];
        joined[(grp * 2 + 1) * width + (e * kGroup + t) * V + k] = db[e][k];
      }
    __syncthreads();
    for (int j = threadIdx.x; j < 2 * width; j += kBlock) {
      const int which = j / width, c = j % width;
      if (c >= cols) continue;
      float s = 0.0f;
      for (int q = 0; q < kGroups; ++q) s += joined[(q * 2 + which) * width + c];
      a.partial[((int64_t)blockIdx.x * 2 + which) * cols + c] = s;
    }
  } else {
    float* p = a.partial + (int64_t)blockIdx.x * 2 * cols;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int64_t j = ((int64_t)e * kGroup + t) * V;
      if (j >= cols) continue;
      if constexpr (V == 1) {
        p[j] = dw[e][0];
        p[cols + j] = db[e][0];
      } else {
        store<float, V>(p + j, dw[e]);          // (V divides cols: 16-byte aligned)
        store<float, V>(p + cols + j, db[e]);
      }
    }
  }
}

// Rows wider than the registers: one CTA per row at a time, each row swept twice from
// memory; the column sums are the next kernel's.
template <typename T, typename TW>
__global__ void __launch_bounds__(1024) backward_wide_kernel(const LayerNormArgs a) {
  __shared__ float buf[2][2][32];
  const int64_t cols = a.cols;
  const float inv_n = 1.0f / (float)cols;
  const TW* w = static_cast<const TW*>(a.weight);
  int flip = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, flip ^= 1) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
    const T* dr = a.r ? static_cast<const T*>(a.r) + row * a.ldr : nullptr;
    T* dx = static_cast<T*>(a.dx) + row * a.lddx;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int64_t j = threadIdx.x; j < cols; j += 1024) {
      const float g = Elem<T>::to(dy[j]) * (w ? Elem<TW>::to(w[j]) : 1.0f);
      s1 += g;
      s2 = fmaf(g, (Elem<T>::to(x[j]) - mean) * rstd, s2);
    }
    s1 = group_sum<1024>(s1, buf[flip][0]) * inv_n;
    s2 = group_sum<1024>(s2, buf[flip][1]) * inv_n;
    for (int64_t j = threadIdx.x; j < cols; j += 1024) {
      const float g = Elem<T>::to(dy[j]) * (w ? Elem<TW>::to(w[j]) : 1.0f);
      float o = rstd * (g - s1 - (Elem<T>::to(x[j]) - mean) * rstd * s2);
      if (dr) o += Elem<T>::to(dr[j]);
      dx[j] = Elem<T>::from(o);
    }
  }
}
// dw and db of the rows blockIdx.y, blockIdx.y + gridDim.y, ...: one column per thread
template <typename T>
__global__ void __launch_bounds__(256) wide_sums_kernel(const LayerNormArgs a) {
  const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (j >= a.cols) return;
  float dw = 0.0f, db = 0.0f;
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float dy = Elem<T>::to(static_cast<const T*>(a.dy)[row * a.lddy + j]);
    const float x = Elem<T>::to(static_cast<const T*>(a.x)[row * a.ldx + j]);
    db += dy;
    dw = fmaf(dy, (x - a.mean[row]) * a.rstd[row], dw);
  }
  a.partial[(int64_t)blockIdx.y * 2 * a.cols + j] = dw;
  a.partial[((int64_t)blockIdx.y * 2 + 1) * a.cols + j] = db;
}

// Adds the partial rows: 32 columns of dw or db per CTA, its 32 warps the rows w, w + 32,
// ..., then the 32 sums in warp order.
template <typename TW>
__global__ void __launch_bounds__(1024) column_sums_kernel(const float* __restrict__ partial,
                                                           int64_t n_partial, int64_t cols,
                                                           TW* dweight, TW* dbias) {
  __shared__ float part[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t j = (int64_t)blockIdx.x * 32 + lane;
  const int which = blockIdx.y;
  pdl_wait();
  pdl_trigger();
  float s = 0.0f;
  if (j < cols)
    for (int64_t p = warp; p < n_partial; p += 32) s += partial[(p * 2 + which) * cols + j];
  part[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || j >= cols) return;
  s = 0.0f;
#pragma unroll
  for (int w = 0; w < 32; ++w) s += part[w][lane];
  TW* out = which == 0 ? dweight : dbias;
  if (out) out[j] = Elem<TW>::from(s);
}

bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
// whether a matrix of esize-byte elements can be read in 16-byte chunks row by row
bool wide_rows(const void* p, int64_t ld, int esize) {
  return p == nullptr || (aligned(p, 16) && ld * esize % 16 == 0);
}

// f(Group, E) for the first shape whose threads hold a row's chunks of V columns
template <int V, typename F>
cudaError_t for_shape(int64_t cols, F f) {
  using std::integral_constant;
  const int64_t chunks = (cols + V - 1) / V;
  constexpr int EW = kWarpElems / V, E = kCtaElems / V;
  if (chunks <= 32 * EW) return f(integral_constant<int, 32>{}, integral_constant<int, EW>{});
  if (chunks <= 128 * E) return f(integral_constant<int, 128>{}, integral_constant<int, E>{});
  if (chunks <= 192 * E) return f(integral_constant<int, 192>{}, integral_constant<int, E>{});
  if (chunks <= 256 * E) return f(integral_constant<int, 256>{}, integral_constant<int, E>{});
  if (chunks <= 320 * E) return f(integral_constant<int, 320>{}, integral_constant<int, E>{});
  if (chunks <= 512 * E) return f(integral_constant<int, 512>{}, integral_constant<int, E>{});
  if (chunks <= 768 * E) return f(integral_constant<int, 768>{}, integral_constant<int, E>{});
  return f(integral_constant<int, 1024>{}, integral_constant<int, 0>{});
}

// stages of a ring of n matrices' rows, as many as an SM's resident CTAs have room for
template <int kGroup>
int ring_stages(int n, uint32_t slot) {
  constexpr int block = block_of(kGroup);
  const size_t room = 208 * 1024 / resident_of(block);
  return (int)std::min<size_t>(kMaxStages, room / ((size_t)(block / kGroup) * n * slot));
}
template <typename T>
uint32_t ring_slot(int64_t cols) {
  return (uint32_t)((cols * sizeof(T) + 15) / 16 * 16 + 16);
}

template <typename T, typename TW, int V>
cudaError_t forward_v(const LayerNormArgs& a, int32_t sms, cudaStream_t s) {
  return for_shape<V>(a.cols, [&](auto group, auto e) -> cudaError_t {
    constexpr int G = decltype(group)::value, E = decltype(e)::value;
    constexpr int block = block_of(G), per = block / G;
    if constexpr (E > 0) {
      const int64_t grid = (int64_t)resident_of(block) * sms;
      const uint32_t slot = ring_slot<T>(a.cols);
      const int n = a.r ? 2 : 1, stages = ring_stages<G>(n, slot);
      // more rows than the resident groups have at once
      if (a.rows > grid * per && stages >= 2) {
        const auto kernel = forward_ring_kernel<T, TW, G, E, V>;
        const size_t smem = (size_t)per * stages * n * slot;
        const cudaError_t err = cudaFuncSetAttribute(
            kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (err != cudaSuccess) return err;
        return launch_dependent(kernel, (unsigned)grid, block, smem, s, 1, true, a, stages, slot);
      }
    }
    return launch_dependent(forward_kernel<T, TW, G, E, V>, (unsigned)((a.rows + per - 1) / per),
                            block, 0, s, 1, true, a);
  });
}
template <typename T, typename TW>
cudaError_t forward_t(const LayerNormArgs& a, int32_t sms, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const bool wide = a.cols % V == 0 && wide_rows(a.x, a.ldx, sizeof(T)) &&
                    wide_rows(a.r, a.ldr, sizeof(T)) && wide_rows(a.y, a.ldy, sizeof(T)) &&
                    wide_rows(a.h, a.ldh, sizeof(T)) && aligned(a.weight, 16) &&
                    aligned(a.bias, 16);
  return wide ? forward_v<T, TW, V>(a, sms, s) : forward_v<T, TW, 1>(a, sms, s);
}

template <typename T, typename TW, int V>
cudaError_t backward_v(const LayerNormArgs& a, int64_t n_partial, cudaStream_t s) {
  return for_shape<V>(a.cols, [&](auto group, auto e) -> cudaError_t {
    constexpr int G = decltype(group)::value, E = decltype(e)::value;
    if constexpr (E == 0) {
      backward_wide_kernel<T, TW><<<(unsigned)std::min<int64_t>(a.rows, 1 << 20), 1024, 0, s>>>(a);
      cudaError_t err = cudaGetLastError();
      if (err != cudaSuccess || a.partial == nullptr) return err;
      wide_sums_kernel<T><<<dim3((unsigned)((a.cols + 255) / 256), (unsigned)n_partial), 256, 0, s>>>(a);
      return cudaGetLastError();
    } else {
      constexpr int block = block_of(G), groups = block / G;
      size_t smem = groups > 1 ? sizeof(float) * 2 * groups * E * G * V : 0;
      const uint32_t slot = ring_slot<T>(a.cols);
      const int n = a.r ? 3 : 2, stages = ring_stages<G>(n, slot);
      const bool ring = a.rows > n_partial * groups && stages >= 2;
      const auto kernel = ring ? backward_kernel<T, TW, G, E, V, true>
                               : backward_kernel<T, TW, G, E, V, false>;
      if (ring) smem = std::max(smem, (size_t)groups * stages * n * slot);
      const cudaError_t err = cudaFuncSetAttribute(
          kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)std::max<size_t>(smem, 1024));
      if (err != cudaSuccess) return err;
      return launch_dependent(kernel, (unsigned)n_partial, block, smem, s, 1, true, a, stages, slot);
    }
  });
}
template <typename T, typename TW>
cudaError_t backward_t(const LayerNormArgs& a, int64_t n_partial, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const bool wide = a.cols % V == 0 && wide_rows(a.x, a.ldx, sizeof(T)) &&
                    wide_rows(a.dy, a.lddy, sizeof(T)) && wide_rows(a.r, a.ldr, sizeof(T)) &&
                    wide_rows(a.dx, a.lddx, sizeof(T)) && aligned(a.weight, 16);
  cudaError_t e = cudaSuccess;
  if (a.rows > 0)
    e = wide ? backward_v<T, TW, V>(a, n_partial, s) : backward_v<T, TW, 1>(a, n_partial, s);
  if (e != cudaSuccess || (a.dweight == nullptr && a.dbias == nullptr)) return e;
  return launch_dependent(column_sums_kernel<TW>, dim3((unsigned)((a.cols + 31) / 32), 2), 1024, 0,
                          s, 1, true, a.partial, a.rows > 0 ? n_partial : 0, a.cols,
                          static_cast<TW*>(a.dweight), static_cast<TW*>(a.dbias));
}

}  // namespace

int64_t layernorm_partial_rows(int64_t rows, int64_t cols, int32_t sms) {
  // the resident CTAs, which hold four rows at a time where a row is a warp's
  const bool warps = cols <= 32 * kWarpElems;
  const int64_t at_once = warps ? 4 : 1, ctas = (int64_t)(warps ? resident_of(128) : 2) * sms;
  return std::max<int64_t>(1, std::min<int64_t>((rows + at_once - 1) / at_once, ctas));
}

cudaError_t launch_layernorm_forward(const LayerNormArgs& a, int32_t sms, cudaStream_t s) {
  if (a.rows <= 0) return cudaSuccess;
  if (a.dtype == kF32)
    return a.wdtype == kF32 ? forward_t<float, float>(a, sms, s)
                            : forward_t<float, __nv_bfloat16>(a, sms, s);
  return a.wdtype == kF32 ? forward_t<__nv_bfloat16, float>(a, sms, s)
                          : forward_t<__nv_bfloat16, __nv_bfloat16>(a, sms, s);
}

cudaError_t launch_layernorm_backward(const LayerNormArgs& a, int32_t sms, cudaStream_t s) {
  const int64_t n = layernorm_partial_rows(a.rows, a.cols, sms);
  if (a.dtype == kF32)
    return a.wdtype == kF32 ? backward_t<float, float>(a, n, s)
                            : backward_t<float, __nv_bfloat16>(a, n, s);
  return a.wdtype == kF32 ? backward_t<__nv_bfloat16, float>(a, n, s)
                          : backward_t<__nv_bfloat16, __nv_bfloat16>(a, n, s);
}

}  // namespace zo
