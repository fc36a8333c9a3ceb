// Layer normalisation, forward pass (zo_layernorm.cuh).
#include "zo_layernorm.cuh"

namespace zo {
namespace {

using namespace ln;

// ---------------------------------------------------------------------------- forward
// One row per group.
template <typename T, typename TW, int kGroup, int kElems, int V>
__global__ void __launch_bounds__(block_of(kGroup))
forward_kernel(const LayerNormArgs a) {
  constexpr int kBlock = block_of(kGroup), kRows = kBlock / kGroup;
  __shared__ float buf[2][32];
  const int t = threadIdx.x % kGroup;
  const int64_t wanted = (int64_t)blockIdx.x * kRows + threadIdx.x / kGroup;
  pdl_wait();
  pdl_trigger();
  const bool live = wanted < a.rows;            // (the lanes of a warp stay together)
  const int64_t row = live ? wanted : a.rows - 1;
  const int64_t cols = a.cols;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* r = a.r ? static_cast<const T*>(a.r) + row * a.ldr : nullptr;
  T* h = a.r ? static_cast<T*>(a.h) + row * a.ldh : nullptr;
  T* y = static_cast<T*>(a.y) + row * a.ldy;
  const TW* w = static_cast<const TW*>(a.weight);
  const TW* b = static_cast<const TW*>(a.bias);
  const float inv_n = 1.0f / (float)cols;

  float mean, rstd;
  if constexpr (kElems > 0) {
    // every load is under way before anything is computed
    const int col = t * V;
    const auto inside = [&](int e) { return e * kGroup * V + col < (int)cols; };
    const auto written = [&](int e) { return live && inside(e); };
    float2 v[kElems / 2], wv[kElems / 2], bv[kElems / 2];
#pragma unroll
    for (int i = 0; i < kElems / 2; ++i) {
      wv[i] = both(1.0f);
      bv[i] = both(0.0f);
    }
    load_columns<T, kElems, kGroup, V, true>(x + col, inside, 0.0f, v);
    if (w) load_columns<TW, kElems, kGroup, V, true>(w + col, inside, 0.0f, wv);
    if (b) load_columns<TW, kElems, kGroup, V, true>(b + col, inside, 0.0f, bv);
    if (r) {
      float2 o[kElems / 2];
      load_columns<T, kElems, kGroup, V, true>(r + col, inside, 0.0f, o);
#pragma unroll
      for (int i = 0; i < kElems / 2; ++i) v[i] = rounded<T>(add2(v[i], o[i]));
      store_columns<T, kElems, kGroup, V>(h + col, written, v);
    }
    float2 s = both(0.0f), q = both(0.0f);
#pragma unroll
    for (int i = 0; i < kElems / 2; ++i) s = add2(s, v[i]);
    mean = group_sum<kGroup>(s.x + s.y, buf[0]) * inv_n;
    const float2 minus = both(-mean);
#pragma unroll
    for (int i = 0; i < kElems / 2; ++i) {
      v[i] = add2(v[i], minus);
      if constexpr (V == 1) {
        if (!inside(2 * i)) v[i].x = 0.0f;
        if (!inside(2 * i + 1)) v[i].y = 0.0f;
      } else if (!inside(2 * i / V)) {
        v[i] = both(0.0f);
      }
      q = fma2(v[i], v[i], q);
    }
    rstd = 1.0f / sqrtf(group_sum<kGroup>(q.x + q.y, buf[1]) * inv_n + a.eps);
    const float2 scale = both(rstd);
#pragma unroll
    for (int i = 0; i < kElems / 2; ++i) v[i] = fma2(mul2(v[i], scale), wv[i], bv[i]);
    store_columns<T, kElems, kGroup, V>(y + col, written, v);
  } else {
    float v[V], s = 0.0f, q = 0.0f;
    const auto fetch = [&](int64_t j) {
      load<T, V, true>(x + j, v);
      if (r) {
        float o[V];
        load<T, V, true>(r + j, o);
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = Elem<T>::to(Elem<T>::from(v[k] + o[k]));
      }
    };
    for (int64_t j = (int64_t)t * V; j < cols; j += (int64_t)kGroup * V) {
      fetch(j);
      if (h) store<T, V>(h + j, v);
#pragma unroll
      for (int k = 0; k < V; ++k) s += v[k];
    }
    mean = group_sum<kGroup>(s, buf[0]) * inv_n;
    for (int64_t j = (int64_t)t * V; j < cols; j += (int64_t)kGroup * V) {
      fetch(j);
#pragma unroll
      for (int k = 0; k < V; ++k) q = fmaf(v[k] - mean, v[k] - mean, q);
    }
    rstd = 1.0f / sqrtf(group_sum<kGroup>(q, buf[1]) * inv_n + a.eps);
    for (int64_t j = (int64_t)t * V; j < cols; j += (int64_t)kGroup * V) {
      fetch(j);
      float wv[V], bv[V];
#pragma unroll
      for (int k = 0; k < V; ++k) { wv[k] = 1.0f; bv[k] = 0.0f; }
      if (w) load<TW, V, true>(w + j, wv);
      if (b) load<TW, V, true>(b + j, bv);
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = fmaf((v[k] - mean) * rstd, wv[k], bv[k]);
      store<T, V>(y + j, v);
    }
  }
  if (t == 0 && live) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

// Many rows: the group's rows by a ring; weight and bias stay in registers.
template <typename T, typename TW, int kGroup, int kElems, int V>
__global__ void __launch_bounds__(block_of(kGroup), resident_of(kGroup, kElems, false))
forward_ring_kernel(const LayerNormArgs a, int stages, uint32_t slot) {
  constexpr int kBlock = block_of(kGroup), kGroups = kBlock / kGroup;
  __shared__ float buf[2][2][32];
  __shared__ uint64_t full[kGroups][kMaxStages];
  __shared__ Lost lost[kGroups];
  extern __shared__ __align__(128) uint8_t dyn[];
  const int t = threadIdx.x % kGroup, grp = threadIdx.x / kGroup;
  const int64_t cols = a.cols;
  const float inv_n = 1.0f / (float)cols;
  Ring<T> ring{{static_cast<const T*>(a.x), static_cast<const T*>(a.r), nullptr},
               {a.ldx, a.ldr, 0}, a.r ? 2 : 1, stages, slot, (uint32_t)(cols * sizeof(T)),
               dyn + (size_t)grp * stages * (a.r ? 2 : 1) * slot, full[grp]};
  if (t == 0) {
    for (int s = 0; s < stages; ++s) sm100::mbar_init(&full[grp][s], 1);
    lost[grp].yes = 0;
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
  const int col = t * V;                       // this thread's chunks: every kGroup V columns
  const auto inside = [&](int e) { return e * kGroup * V + col < (int)cols; };
  float2 wv[kElems / 2], bv[kElems / 2];
#pragma unroll
  for (int i = 0; i < kElems / 2; ++i) {
    wv[i] = both(1.0f);
    bv[i] = both(0.0f);
  }
  if (a.weight)
    load_columns<TW, kElems, kGroup, V, true>(static_cast<const TW*>(a.weight) + col, inside, 0.0f, wv);
  if (a.bias)
    load_columns<TW, kElems, kGroup, V, true>(static_cast<const TW*>(a.bias) + col, inside, 0.0f, bv);
  int flip = 0;
  bool gone = false;
  for (int64_t row = row0; row < a.rows; row += stride, flip ^= 1) {
    float2 s = both(0.0f), q = both(0.0f);
    const bool came = ring.ready(lost[grp], gone);
    if (!came) {
      s = both(nan_value());                   // the row's sum, and with it all of the row, is NaN
      ring.lose(lost[grp], row);
    }
    float2 v[kElems / 2];
    load_columns<T, kElems, kGroup, V, false>(ring.at(0, row) + col, inside, 0.0f, v);
    if (a.r) {
      float2 o[kElems / 2];
      load_columns<T, kElems, kGroup, V, false>(ring.at(1, row) + col, inside, 0.0f, o);
#pragma unroll
      for (int i = 0; i < kElems / 2; ++i) v[i] = rounded<T>(add2(v[i], o[i]));
      if (!came) to_nan(v);
      store_columns<T, kElems, kGroup, V>(static_cast<T*>(a.h) + row * a.ldh + col, inside, v);
    }
#pragma unroll
    for (int i = 0; i < kElems / 2; ++i) s = add2(s, v[i]);
    const float mean = group_sum<kGroup>(s.x + s.y, buf[flip][0]) * inv_n;
    // every thread of the group has read the stage
    gone = lost[grp].yes;
    if (t == 0 && row + stages * stride < a.rows && !gone)
      ring.fetch(row + stages * stride, ring.stage);
    ring.advance();
    const float2 minus = both(-mean);
#pragma unroll
    for (int i = 0; i < kElems / 2; ++i) {
      v[i] = add2(v[i], minus);
      if constexpr (V == 1) {
        if (!inside(2 * i)) v[i].x = 0.0f;
        if (!inside(2 * i + 1)) v[i].y = 0.0f;
      } else if (!inside(2 * i / V)) {
        v[i] = both(0.0f);
      }
      q = fma2(v[i], v[i], q);
    }
    const float rstd = 1.0f / sqrtf(group_sum<kGroup>(q.x + q.y, buf[flip][1]) * inv_n + a.eps);
    const float2 scale = both(rstd);
#pragma unroll
    for (int i = 0; i < kElems / 2; ++i) v[i] = fma2(mul2(v[i], scale), wv[i], bv[i]);
    store_columns<T, kElems, kGroup, V>(static_cast<T*>(a.y) + row * a.ldy + col, inside, v);
    if (t == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
  if (t == 0) ring.finish(lost[grp], row0, stride, a.rows, a.status);
}

template <typename T, typename TW, int V>
cudaError_t forward_v(const LayerNormArgs& a, int32_t sms, cudaStream_t s) {
  const Shape sh = shape_for(a.rows, a.cols, sms, false);
  return with_shape(sh, [&](auto group, auto elems) -> cudaError_t {
    constexpr int G = decltype(group)::value, E = decltype(elems)::value;
    constexpr int block = block_of(G), per = block / G;
    if constexpr (E > 0 && ring_of(G, E)) {
      const uint32_t slot = ring_slot<T>(a.cols);
      const int n = a.r ? 2 : 1, stages = ring_stages<G, E, false>(n, slot);
      if (a.rows > groups_at_once(sh, sms, false) && stages >= 2) {
        const auto kernel = forward_ring_kernel<T, TW, G, E, V>;
        const size_t smem = (size_t)per * stages * n * slot;
        const cudaError_t err = allow_smem(kernel, kRingRoom<G, E, false>);
        if (err != cudaSuccess) return err;
        return launch_dependent(kernel, (unsigned)(resident_of(G, E, false) * sms), block, smem, s, 1,
                                true, a, stages, slot);
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

}  // namespace

cudaError_t launch_layernorm_forward(const LayerNormArgs& a, int32_t sms, cudaStream_t s) {
  if (a.rows <= 0) return cudaSuccess;
  if (a.dtype == kF32)
    return a.wdtype == kF32 ? forward_t<float, float>(a, sms, s)
                            : forward_t<float, __nv_bfloat16>(a, sms, s);
  return a.wdtype == kF32 ? forward_t<__nv_bfloat16, float>(a, sms, s)
                          : forward_t<__nv_bfloat16, __nv_bfloat16>(a, sms, s);
}

}  // namespace zo
