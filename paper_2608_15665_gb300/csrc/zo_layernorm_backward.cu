// Layer normalisation, backward pass (zo_layernorm.cuh).
#include "zo_layernorm.cuh"

namespace zo {
namespace {

using namespace ln;

// --------------------------------------------------------------------------- backward
// Rows held in registers: each thread keeps its columns' weight, dw and db over all rows
// of its group.  kRing: the rows come through a ring, else straight from memory.
template <typename T, typename TW, int kGroup, int kElems, int V, bool kRing>
__global__ void __launch_bounds__(block_of(kGroup), resident_of(kGroup, kElems, true))
backward_kernel(const LayerNormArgs a, int stages, uint32_t slot) {
  constexpr int kBlock = block_of(kGroup), kGroups = kBlock / kGroup;
  static_assert(kElems > 0, "rows in registers");
  __shared__ float buf[2][2][32];
  __shared__ uint64_t full[kGroups][kMaxStages];
  __shared__ Lost lost[kGroups];
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
      lost[grp].yes = 0;
      sm100::fence_mbar_init();
    }
    __syncthreads();
  }
  pdl_wait();
  pdl_trigger();
  const int col = t * V;                       // this thread's chunks: every kGroup V columns
  const auto inside = [&](int e) { return e * kGroup * V + col < (int)cols; };
  constexpr int kPairs = kElems / 2;
  float2 wv[kPairs], dw[kPairs], db[kPairs];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    wv[i] = both(1.0f);
    dw[i] = db[i] = both(0.0f);
  }
  if (a.weight)
    load_columns<TW, kElems, kGroup, V, true>(static_cast<const TW*>(a.weight) + col, inside, 0.0f, wv);
  const int64_t stride = (int64_t)gridDim.x * kGroups;
  const int64_t row0 = (int64_t)blockIdx.x * kGroups + grp;
  if constexpr (kRing) {
    if (t == 0)
      for (int s = 0; s < stages; ++s)
        if (row0 + s * stride < a.rows) ring.fetch(row0 + s * stride, s);
  }
  int flip = 0;
  bool gone = false;
  float mean_next = row0 < a.rows ? a.mean[row0] : 0.0f, rstd_next = row0 < a.rows ? a.rstd[row0] : 0.0f;
  // the groups of a warp go on together
  const int64_t first = kGroup < 32 ? row0 - (threadIdx.x % 32) / kGroup : row0;
  for (int64_t step = 0; first + step < a.rows; step += stride, flip ^= 1) {
    const bool live = kGroup >= 32 || row0 + step < a.rows;
    const int64_t row = live ? row0 + step : a.rows - 1;
    T* dx = static_cast<T*>(a.dx) + row * a.lddx + col;
    float mean = live ? mean_next : 0.0f;
    const float rstd = live ? rstd_next : 0.0f;
    if (row0 + step + stride < a.rows) {
      mean_next = a.mean[row0 + step + stride];
      rstd_next = a.rstd[row0 + step + stride];
    }
    const auto here = [&](int e) { return live && inside(e); };
    float2 xh[kPairs], g[kPairs];
    if constexpr (kRing) {
      if (!ring.ready(lost[grp], gone)) {
        // NaN in the row's sums, and with them in all of its dx, and in this thread's dw and db
        mean = nan_value();
        to_nan(db);
        ring.lose(lost[grp], row);
      }
      load_columns<T, kElems, kGroup, V, false>(ring.at(0, row) + col, here, mean, xh);
      load_columns<T, kElems, kGroup, V, false>(ring.at(1, row) + col, here, 0.0f, g);
    } else {
      load_columns<T, kElems, kGroup, V, true>(ring.row_of(0, row) + col, here, mean, xh);
      load_columns<T, kElems, kGroup, V, true>(ring.row_of(1, row) + col, here, 0.0f, g);
    }
    float2 p1 = both(0.0f), p2 = both(0.0f);
    const float2 minus = both(-mean), scale = both(rstd);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      xh[i] = mul2(add2(xh[i], minus), scale);
      db[i] = add2(db[i], g[i]);
      dw[i] = fma2(g[i], xh[i], dw[i]);
      g[i] = mul2(g[i], wv[i]);
      p1 = add2(p1, g[i]);
      p2 = fma2(g[i], xh[i], p2);
    }
    float s1 = p1.x + p1.y, s2 = p2.x + p2.y;
#pragma unroll
    for (int o = (kGroup < 32 ? kGroup : 32) / 2; o > 0; o >>= 1) {
      s1 += __shfl_xor_sync(0xffffffffu, s1, o);
      s2 += __shfl_xor_sync(0xffffffffu, s2, o);
    }
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
    const float2 m1 = both(-s1 * inv_n), m2 = both(-s2 * inv_n);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) g[i] = mul2(scale, fma2(xh[i], m2, add2(g[i], m1)));
    if (a.r) {
      if constexpr (kRing) load_columns<T, kElems, kGroup, V, false>(ring.at(2, row) + col, here, 0.0f, xh);
      else load_columns<T, kElems, kGroup, V, true>(ring.row_of(2, row) + col, here, 0.0f, xh);
#pragma unroll
      for (int i = 0; i < kPairs; ++i) g[i] = add2(g[i], xh[i]);
    }
    store_columns<T, kElems, kGroup, V>(dx, here, g);
    if constexpr (kRing) {
      // every thread of the group has read the stage: the row `stages` ahead may have it
      if constexpr (kGroup > 32) {
        if (a.r) __syncthreads();               // (dr was read behind the sums' barrier)
      } else {
        __syncwarp();
      }
      gone = lost[grp].yes;
      if (t == 0 && row + stages * stride < a.rows && !gone)
        ring.fetch(row + stages * stride, ring.stage);
      ring.advance();
    }
  }
  if constexpr (kRing) {
    if (t == 0) ring.finish(lost[grp], row0, stride, a.rows, a.status);
  }
  if (a.partial == nullptr) return;
  if constexpr (kGroups > 1) {
    // the warps' sums meet in shared memory, added in warp order
    float* joined = reinterpret_cast<float*>(dyn);
    constexpr int kWidth = kElems * kGroup;
    const auto all = [](int) { return true; };
    __syncthreads();                            // the rings are no longer read
    store_columns<float, kElems, kGroup, V>(joined + (grp * 2 + 0) * kWidth + col, all, dw);
    store_columns<float, kElems, kGroup, V>(joined + (grp * 2 + 1) * kWidth + col, all, db);
    __syncthreads();
    for (int j = threadIdx.x; j < 2 * kWidth; j += kBlock) {
      const int which = j / kWidth, c = j % kWidth;
      if (c >= cols) continue;
      float s = 0.0f;
      for (int q = 0; q < kGroups; ++q) s += joined[(q * 2 + which) * kWidth + c];
      a.partial[((int64_t)blockIdx.x * 2 + which) * cols + c] = s;
    }
  } else {
    // (V divides cols: 16-byte aligned)
    float* p = a.partial + (int64_t)blockIdx.x * 2 * cols + col;
    store_columns<float, kElems, kGroup, V>(p, inside, dw);
    store_columns<float, kElems, kGroup, V>(p + cols, inside, db);
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
#pragma unroll 8
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

template <typename T, typename TW, int V>
cudaError_t backward_v(const LayerNormArgs& a, int32_t sms, int64_t n_partial, cudaStream_t s) {
  const Shape sh = shape_for(a.rows, a.cols, sms, true);
  return with_shape(sh, [&](auto group, auto elems) -> cudaError_t {
    constexpr int G = decltype(group)::value, E = decltype(elems)::value;
    if constexpr (E == 0) {
      backward_wide_kernel<T, TW><<<(unsigned)std::min<int64_t>(a.rows, 1 << 20), 1024, 0, s>>>(a);
      cudaError_t err = cudaGetLastError();
      if (err != cudaSuccess || a.partial == nullptr) return err;
      wide_sums_kernel<T><<<dim3((unsigned)((a.cols + 255) / 256), (unsigned)n_partial), 256, 0, s>>>(a);
      return cudaGetLastError();
    } else {
      constexpr int block = block_of(G), groups = block / G;
      constexpr size_t joined = groups > 1 ? sizeof(float) * 2 * groups * E * G : 0;
      static_assert(joined <= 48 * 1024, "the sums fit without a limit of their own");
      if constexpr (ring_of(G, E)) {
        const uint32_t slot = ring_slot<T>(a.cols);
        const int n = a.r ? 3 : 2, stages = ring_stages<G, E, true>(n, slot);
        if (a.rows > groups_at_once(sh, sms, true) && stages >= 2) {
          const auto kernel = backward_kernel<T, TW, G, E, V, true>;
          const size_t smem = std::max(joined, (size_t)groups * stages * n * slot);
          const cudaError_t err = allow_smem(kernel, std::max(joined, kRingRoom<G, E, true>));
          if (err != cudaSuccess) return err;
          return launch_dependent(kernel, (unsigned)n_partial, block, smem, s, 1, true, a, stages, slot);
        }
      }
      return launch_dependent(backward_kernel<T, TW, G, E, V, false>, (unsigned)n_partial, block,
                              joined, s, 1, true, a, 0, 0u);
    }
  });
}
template <typename T, typename TW>
cudaError_t backward_t(const LayerNormArgs& a, int32_t sms, int64_t n_partial, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const bool wide = a.cols % V == 0 && wide_rows(a.x, a.ldx, sizeof(T)) &&
                    wide_rows(a.dy, a.lddy, sizeof(T)) && wide_rows(a.r, a.ldr, sizeof(T)) &&
                    wide_rows(a.dx, a.lddx, sizeof(T)) && aligned(a.weight, 16);
  cudaError_t e = cudaSuccess;
  if (a.rows > 0)
    e = wide ? backward_v<T, TW, V>(a, sms, n_partial, s) : backward_v<T, TW, 1>(a, sms, n_partial, s);
  if (e != cudaSuccess || (a.dweight == nullptr && a.dbias == nullptr)) return e;
  return launch_dependent(column_sums_kernel<TW>, dim3((unsigned)((a.cols + 31) / 32), 2), 1024, 0,
                          s, 1, true, a.partial, a.rows > 0 ? n_partial : 0, a.cols,
                          static_cast<TW*>(a.dweight), static_cast<TW*>(a.dbias));
}

}  // namespace

int64_t layernorm_partial_rows(int64_t rows, int64_t cols, int32_t sms) {
  const Shape sh = shape_for(rows, cols, sms, true);
  if (sh.elems == 0) return std::min<int64_t>(rows, 2 * sms);   // slabs of the sums' own kernel
  const int64_t at_once = block_of(sh.group) / sh.group;
  return std::min<int64_t>((rows + at_once - 1) / at_once, (int64_t)resident_of(sh.group, sh.elems, true) * sms);
}

cudaError_t launch_layernorm_backward(const LayerNormArgs& a, int32_t sms, cudaStream_t s) {
  const int64_t n = layernorm_partial_rows(a.rows, a.cols, sms);
  if (a.dtype == kF32)
    return a.wdtype == kF32 ? backward_t<float, float>(a, sms, n, s)
                            : backward_t<float, __nv_bfloat16>(a, sms, n, s);
  return a.wdtype == kF32 ? backward_t<__nv_bfloat16, float>(a, sms, n, s)
                          : backward_t<__nv_bfloat16, __nv_bfloat16>(a, sms, n, s);
}

}  // namespace zo
