// Layer normalisation over the rows of a matrix, forward (zo_layernorm.cu) and backward
// (zo_layernorm_backward.cu): what the two passes share.
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
// A row belongs to a group of threads: 8, 16 or 32 lanes of a warp, or a whole CTA (Shape).
// Thread t of a group takes the chunks t, t + group, ... of VEC consecutive columns: 16
// bytes of the activations' type where every pointer, stride and the width allow it, else
// single elements.  Rows wider than a CTA's registers are swept from memory (kElems = 0).
//
// Many wide rows: a few resident CTAs take the rows blockIdx, blockIdx + gridDim, ..., and what
// keeps HBM busy is a ring of rows per group in shared memory, filled by bulk copies several
// rows ahead.  A row that does not start or end on 16 bytes is copied with the rest of its
// first and last 16 (never past an aligned 16 bytes that hold a part of the row).  At 16384 x
// 5120 bf16 with a residual the backward pass took 271 us without the ring, 115 us with it;
// at 20000 x 64, where a copy is 128 bytes, the forward pass 8 us without and 13 us with it.
// Few rows, and narrow ones: straight from memory.  Few wide rows go to CTAs with eight columns
// a thread, for latency.
//
// Measured, in graphs of calls over inputs larger than L2: forward 4096 x 4096 bf16 with a residual
// 22.7 us (5.9 TB/s), 50001 x 768 fp32 52.7 us (5.8), 8192 x 8192 bf16 61 us (4.4); backward 16384 x
// 5120 bf16 with a residual 104 us (6.5 TB/s with the column sums), 2048 x 2048 12.0 us (10.8 us
// its first kernel alone; the sums' launch lies under it); one row of 5120 2.1 us.  Rows that
// are swept: 2048 x 16384 bf16 57 us forward (2.3 TB/s), 160 us backward (1.3), against 24 and 54 us
// at 12288 columns.
//
// The backward pass keeps dw and db of a thread's own columns in registers over all its
// rows, so that each CTA writes one row of partial sums, which a second kernel adds up in a
// fixed order: no atomics, the same bits on every run.
#pragma once

#include <algorithm>
#include <type_traits>

#include <cuda_bf16.h>

#include "zo_launch.cuh"
#include "zo_ops.h"
#include "zo_sm100.cuh"

namespace zo {
namespace ln {

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

// Two columns at a time: packed fp32 arithmetic (each half an IEEE operation, round to nearest).
// At 24 instructions a column, and not by memory, a row's arithmetic bounded the passes.
union Pair {
  float2 f;
  uint64_t u;
};
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  Pair x{a}, y{b}, r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(x.u), "l"(y.u));
  return r.f;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  Pair x{a}, y{b}, r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(x.u), "l"(y.u));
  return r.f;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  Pair x{a}, y{b}, z{c}, r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.u) : "l"(x.u), "l"(y.u), "l"(z.u));
  return r.f;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float nan_value() { return __int_as_float(0x7FC00000); }
template <int kPairs>
__device__ __forceinline__ void to_nan(float2 (&v)[kPairs]) {
#pragma unroll
  for (int i = 0; i < kPairs; ++i) v[i] = both(nan_value());
}

// A thread's columns of a row as pairs: chunks of V columns, chunk e at column (e kGroup + t) V.
// f(e) says whether chunk e lies inside the row; the values of the others are `rest`.
template <typename T, int kElems, int kGroup, int V, bool kReadOnly, typename F>
__device__ __forceinline__ void load_columns(const T* p, F inside, float rest, float2 (&v)[kElems / 2]) {
#pragma unroll
  for (int e = 0; e < kElems / V; ++e) {
    float c[V];
#pragma unroll
    for (int k = 0; k < V; ++k) c[k] = rest;
    if (inside(e)) load<T, V, kReadOnly>(p + e * kGroup * V, c);
    if constexpr (V == 1) {
      if (e % 2 == 0) v[e / 2].x = c[0];
      else v[e / 2].y = c[0];
    } else {
#pragma unroll
      for (int k = 0; k < V; k += 2) v[(e * V + k) / 2] = make_float2(c[k], c[k + 1]);
    }
  }
}
template <typename T, int kElems, int kGroup, int V, typename F>
__device__ __forceinline__ void store_columns(T* p, F inside, const float2 (&v)[kElems / 2]) {
#pragma unroll
  for (int e = 0; e < kElems / V; ++e) {
    float c[V];
    if constexpr (V == 1) {
      c[0] = e % 2 == 0 ? v[e / 2].x : v[e / 2].y;
    } else {
#pragma unroll
      for (int k = 0; k < V; k += 2) {
        c[k] = v[(e * V + k) / 2].x;
        c[k + 1] = v[(e * V + k) / 2].y;
      }
    }
    if (inside(e)) store<T, V>(p + e * kGroup * V, c);
  }
}
template <typename T>
__device__ __forceinline__ float2 rounded(float2 v) {
  return make_float2(Elem<T>::to(Elem<T>::from(v.x)), Elem<T>::to(Elem<T>::from(v.y)));
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sum over the group (kGroup lanes of a warp, or the whole CTA of kGroup threads), in every
// thread.  `buf` holds one value per warp; two calls in a row take different buffers.
template <int kGroup>
__device__ __forceinline__ float group_sum(float v, float* buf) {
#pragma unroll
  for (int o = (kGroup < 32 ? kGroup : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if constexpr (kGroup > 32) {
    constexpr int kWarps = kGroup / 32;
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    v = warp_sum(lane < kWarps ? buf[lane] : 0.0f);
  }
  return v;
}

// threads of a CTA whose rows take `group` threads each
__host__ __device__ constexpr int block_of(int group) { return group <= 32 ? 128 : group; }
// Resident CTAs of the many-row kernels on an SM: as many as leave a thread the registers of
// its columns.  The backward pass holds five values of each (x, dy, dw, db and the weight), the
// forward pass three.
__host__ __device__ constexpr int resident_of(int group, int elems, bool backward) {
  if (group <= 32) return elems <= 8 ? 8 : elems <= 16 ? 5 : 3;
  if (backward) return group <= 128 ? 3 : group <= 320 ? 2 : 1;
  return group <= 128 ? 6 : group <= 192 ? 4 : group <= 320 ? 3 : group <= 512 ? 2 : 1;
}
__host__ __device__ constexpr bool ring_of(int group, int elems) { return group > 32 || elems == 32; }

// How a pass goes over its rows: threads of a row and columns of a thread (0: swept).
struct Shape {
  int group, elems;
};
// `few`: no more rows than the resident groups hold at once
inline Shape shape_of(int64_t cols, bool few) {
  if (cols <= 64) return {8, 8};
  if (cols <= 128) return {16, 8};
  if (cols <= 256) return {32, 8};
  if (cols <= 512) return {32, 16};
  if (few && cols <= 1024) return {128, 8};
  if (few && cols <= 2048) return {256, 8};
  if (few && cols <= 4096) return {512, 8};
  if (cols <= 1024) return {32, 32};
  if (cols <= 128 * 16) return {128, 16};
  if (cols <= 192 * 16) return {192, 16};
  if (cols <= 256 * 16) return {256, 16};
  if (cols <= 320 * 16) return {320, 16};
  if (cols <= 512 * 16) return {512, 16};
  if (cols <= 768 * 16) return {768, 16};
  return {1024, 0};
}
inline int64_t groups_at_once(Shape sh, int32_t sms, bool backward) {
  return (int64_t)resident_of(sh.group, sh.elems, backward) * (block_of(sh.group) / sh.group) * sms;
}
// the shape for `rows` rows
inline Shape shape_for(int64_t rows, int64_t cols, int32_t sms, bool backward) {
  const Shape many = shape_of(cols, false);
  return rows > groups_at_once(many, sms, backward) ? many : shape_of(cols, true);
}

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

// the first row of a group whose copies did not come in time
struct Lost {
  volatile int yes;
  volatile int64_t row;
};

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
  // Waits for the present stage, whose row's places in it are then at(m, row).  False: the copies have
  // not come within the limit, or a row before was lost (`gone`, read of lost.yes behind a barrier of
  // the group); the row's results are NaN, and the thread calls lose().  (The barrier alone does
  // not tell a stage that was not fetched again: two rounds on, its parity is the last copies'.)
  __device__ bool ready(const Lost& lost, bool gone) const {
    return !gone && (sm100::mbar_try_wait(&full[stage], phase) ||
                     sm100::mbar_wait_bounded(&full[stage], phase, &lost.yes, kWait));
  }
  static __device__ void lose(Lost& lost, int64_t row) {
    if (lost.yes) return;
    lost.row = row;
    lost.yes = 1;
  }
  // By the fetching thread after the last row: where one was lost (after which nothing is fetched: a
  // stage whose bytes may be still to come is not armed again), the call's status is set, and the
  // copies that were in flight come to rest.
  __device__ void finish(const Lost& lost, int64_t row0, int64_t stride, int64_t rows, uint32_t* status) const {
    if (!lost.yes) return;
    atomicOr(status, 1u);
    int64_t k = (lost.row - row0) / stride;
    for (int s = 0; s < stages && row0 + k * stride < rows; ++s, ++k)
      sm100::mbar_wait_bounded(&full[k % stages], (uint32_t)(k / stages & 1), nullptr, kWait);
  }
  __device__ const T* at(int m, int64_t row) const {
    return reinterpret_cast<const T*>(smem + (size_t)(stage * n + m) * slot + lead(row_of(m, row)));
  }
  __device__ void advance() {
    if (++stage == stages) {
      stage = 0;
      phase ^= 1u;
    }
  }
};

inline bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
// whether a matrix of esize-byte elements can be read in 16-byte chunks row by row
inline bool wide_rows(const void* p, int64_t ld, int esize) {
  return p == nullptr || (aligned(p, 16) && ld * esize % 16 == 0);
}

// f(group, elems) with a shape as constants
template <typename F>
cudaError_t with_shape(Shape sh, F f) {
  using std::integral_constant;
#define ZO_SHAPE(G, E) \
  if (sh.group == G && sh.elems == E) return f(integral_constant<int, G>{}, integral_constant<int, E>{});
  ZO_SHAPE(8, 8) ZO_SHAPE(16, 8) ZO_SHAPE(32, 8) ZO_SHAPE(32, 16) ZO_SHAPE(32, 32)
  ZO_SHAPE(128, 8) ZO_SHAPE(256, 8) ZO_SHAPE(512, 8)
  ZO_SHAPE(128, 16) ZO_SHAPE(192, 16) ZO_SHAPE(256, 16) ZO_SHAPE(320, 16) ZO_SHAPE(512, 16)
  ZO_SHAPE(768, 16) ZO_SHAPE(1024, 0)
#undef ZO_SHAPE
  return cudaErrorInvalidValue;
}

// a CTA's room for its rings: what an SM's resident CTAs share
template <int kGroup, int kElems, bool kBackward>
constexpr size_t kRingRoom = 208 * 1024 / resident_of(kGroup, kElems, kBackward);
// stages of a ring of n matrices' rows, as many as there is room for
template <int kGroup, int kElems, bool kBackward>
int ring_stages(int n, uint32_t slot) {
  return (int)std::min<size_t>(kMaxStages, kRingRoom<kGroup, kElems, kBackward> /
                                               ((size_t)(block_of(kGroup) / kGroup) * n * slot));
}
// Lets a kernel take up to `most` bytes of dynamic shared memory.  `most` is the instance's own and
// not one call's: the limit belongs to the kernel, and calls of several threads share it.
template <typename K>
cudaError_t allow_smem(K kernel, size_t most) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
}
template <typename T>
uint32_t ring_slot(int64_t cols) {
  return (uint32_t)((cols * sizeof(T) + 15) / 16 * 16 + 16);
}

}  // namespace ln
}  // namespace zo
