// A preference loss over pairs of answers, forward and backward (C ABI: include/zo.h).
//
//   lse_r = log sum_j exp l_rj,   logp_r = l_r[y_r] - lse_r            (counted rows)
//   s_q = sum (or mean) of logp_r over the counted rows of sequence q
//   D = (s_c - ref_c) - (s_r - ref_r),  loss_p = f(D),  loss = mean_p loss_p
//   dl_rj = dloss dlogp_r ([j = y_r] - exp(l_rj - lse_r)),  dlogp_r = d loss / d logp_r
//
// Bound by HBM: the forward pass reads every counted row once (a running maximum c and the sum of
// e^(l - c) in each thread, joined over the CTA), the backward pass reads and writes them once;
// rows that do not count are not read (16 pairs of 600, 32000 bf16: 144 us, 92% of the copy rate;
// backward 8 of 1000: 341 us, 102%).  A CTA takes one row, or a part of one where the rows
// alone do not fill the device.  (l - c first, then its product with log2 e: logits of the type's
// lowest value, in one place or in all, overflow nowhere that matters.)
//
// The pairs' kernel is launched behind it: a CTA per pair sums its two sequences, in 64 bits,
// and the one that finishes last adds the losses up, in their order.
#include <algorithm>
#include <cmath>

#include <cuda_bf16.h>

#include "../../include/zo.h"
#include "zo_device.cuh"
#include "zo_host.h"
#include "zo_launch.cuh"

namespace {

using namespace zo::host;

// Small CTAs: one's first loads and last sums lie under the others' (16 pairs, 32000 wide: forward
// 144 us with 128 threads, 151 with 256, 177 with 512).
constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kPairThreads = 512;                // of a pair's two sequences
constexpr int kUnroll = 4;                       // vectors of 16 bytes a thread has on their way
constexpr int kMaxParts = 32, kPartCols = 4096;  // parts of a row, none narrower than this
// Whole rows of up to so many bytes belong to a warp each (256M logits in bf16, forward: rows of 1000 487 us
// by CTAs, 153 by warps; of 8000 104 and 93; backward of 1000 259 and 168, of 8000 152 and 158).
constexpr int kShortForward = 16384, kShortBackward = 8192;
// columns of a CTA's part in the backward pass (812 rows of 50257 fp32: 52 us; in whole rows 58, as 5.3
// rows an SM are 6 for some)
constexpr int kGradCols = 8192;
// log2 e in two parts: rounded once it is off by 1.3e-8, which at the logits' usual distance from their
// sum moves every row's lse by 1e-7 the same way, and a sequence's sum by that for each row
constexpr float kLog2e = 1.4426950216293335f, kLog2eLo = 1.9259629e-8f;

struct Rows {
  const void* x;
  int64_t ld;
  int32_t vocab, parts, part_cols;               // columns of a part: a multiple of 8
  int64_t rows;
  const int64_t* labels;
  const int64_t* offsets;                        // 2 pairs + 1
  int64_t pairs;
};

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A base and the sum of e^(x - base).  Bases are finite from below, so that -inf alone gives a sum
// of zero and not a NaN.
struct Sum {
  float c, s;
};
constexpr float kLowest = -3.402823466e38f;
__device__ __forceinline__ float exp_of(float x) { return exp2_approx(fmaf(x, kLog2e, x * kLog2eLo)); }
// (The hardware's exponential is 5e-8 low on average at negative arguments: once in a term, not again
// at every change of base, or all rows' sums lean by 1.4e-7 the same way.)
__device__ __forceinline__ Sum join(Sum a, Sum b) {
  const float c = fmaxf(a.c, b.c);
  return Sum{c, a.s * expf(a.c - c) + b.s * expf(b.c - c)};
}
__device__ __forceinline__ float lse_of(Sum a) { return (float)((double)a.c + (double)logf(a.s)); }
// x - lse, without lse's rounding
__device__ __forceinline__ float logp_of(Sum a, float x) {
  return (float)((double)x - (double)a.c - (double)logf(a.s));
}

template <typename T>
struct Vec {
  static constexpr int kN = 16 / (int)sizeof(T);
  uint4 raw;
  __device__ __forceinline__ void load(const T* p) { raw = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void clear() {                          // nothing: -inf
    const uint32_t w = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
    raw = make_uint4(w, w, w, w);
  }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
};

// live: how many of the vectors any thread of the team has (the same in all of them).  fp32's four
// values are too few for a branch around them (rows of 1000: 216 us with it, 177 without).
template <typename T>
__device__ __forceinline__ void add(Sum& a, const Vec<T> (&v)[kUnroll], int live) {
  float top = v[0].get(0);
#pragma unroll
  for (int u = 0; u < kUnroll; ++u)
    if (sizeof(T) == 4 || u < live)
#pragma unroll
      for (int i = 0; i < Vec<T>::kN; ++i) top = fmaxf(top, v[u].get(i));
  const float c = fmaxf(a.c, top);
  a.s *= expf(a.c - c);
  a.c = c;
  // (two values an instruction, but for the exponentials)
  const float2 less = make_float2(-c, -c), scale = make_float2(kLog2e, kLog2e);
  const float2 rest = make_float2(kLog2eLo, kLog2eLo);
  float2 s = make_float2(a.s, 0.0f);
#pragma unroll
  for (int u = 0; u < kUnroll; ++u)
    if (sizeof(T) == 4 || u < live)
#pragma unroll
      for (int i = 0; i < Vec<T>::kN; i += 2) {
        const float2 d = zo::add2(make_float2(v[u].get(i), v[u].get(i + 1)), less);
        const float2 e = zo::fma2(d, scale, zo::mul2(d, rest));
        s = zo::add2(s, make_float2(exp2_approx(e.x), exp2_approx(e.y)));
      }
  a.s = s.x + s.y;
}
__device__ __forceinline__ void add(Sum& a, float x) {
  const float c = fmaxf(a.c, x);
  a = Sum{c, a.s * expf(a.c - c) + expf(x - c)};
}

// Elements in front of the first 16-byte boundary, at most n.
template <typename T>
__device__ __forceinline__ int head_of(const T* p, int n) {
  const int bytes = (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15);
  return min(n, bytes / (int)sizeof(T));
}

// The rows' sums.  parts > 1: every part's to partial; else lse and logp.  Rows that do not count
// get zeros.  A team per row (part): a CTA, or a warp where a row is short.  Rows that do not count lie together, and with a fixed number of
// rows to a CTA the busiest had a third more to read than the others (16 pairs: 190 us).
template <typename T, int kTeam>
__global__ void __launch_bounds__(kThreads)
rows_kernel(const Rows a, Sum* __restrict__ partial, float* __restrict__ logp,
            float* __restrict__ lse, float* __restrict__ dlogp, uint32_t* __restrict__ ticket) {
  __shared__ Sum warp_sums[kWarps];
  const int member = threadIdx.x % kTeam;
  const int part = (int)(blockIdx.x % (unsigned)a.parts);
  const int64_t row = blockIdx.x / (unsigned)a.parts * (int64_t)(kThreads / kTeam) + threadIdx.x / kTeam;
  zo::pdl_wait();
  zo::pdl_trigger();
  if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;
  if (row >= a.rows) return;
  const int64_t label = a.labels[row];
  const bool counted = label >= 0 && row >= a.offsets[0] && row < a.offsets[2 * a.pairs];
  if (member == 0 && part == 0) {
    if (!counted) logp[row] = 0.0f;
    if (!counted && lse) lse[row] = 0.0f;
    if (dlogp) dlogp[row] = 0.0f;                // (of counted rows: until the pairs' kernel)
  }
  if (!counted) return;
  const int j0 = part * a.part_cols, n = min(a.part_cols, a.vocab - j0);
  const T* x = static_cast<const T*>(a.x) + row * a.ld + j0;
  const bool whole = a.parts == 1 && member == 0;
  const float hit = whole && label < a.vocab ? static_cast<float>(x[label]) : __int_as_float(0x7FC00000);
  Sum sum{kLowest, 0.0f};
  const int head = head_of(x, n);
  const int vecs = (n - head) / Vec<T>::kN;
  const T* xv = x + head;
  for (int i = member; i < vecs; i += kUnroll * kTeam) {
    Vec<T> v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      v[u].clear();
      if (i + u * kTeam < vecs) v[u].load(xv + (int64_t)(i + u * kTeam) * Vec<T>::kN);
    }
    add(sum, v, (vecs - (i - member) + kTeam - 1) / kTeam);
  }
  // what lies around the vectors
  const int around = head + (n - head) % Vec<T>::kN;
  if (member < around) {
    const int k = member < head ? member : n - around + member;
    add(sum, static_cast<float>(x[k]));
  }
  // the warp's common base first, then its sum
  float c = sum.c;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) c = fmaxf(c, __shfl_xor_sync(0xffffffffu, c, d));
  sum.s *= expf(sum.c - c);
  sum.c = c;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum.s += __shfl_xor_sync(0xffffffffu, sum.s, d);
  if constexpr (kTeam > 32) {
    if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5] = sum;
    __syncthreads();
  }
  if (member == 0) {
    if constexpr (kTeam > 32)
      for (int w = 1; w < kWarps; ++w) sum = join(sum, warp_sums[w]);
    if (a.parts > 1) {
      partial[row * a.parts + part] = sum;
    } else {
      if (lse) lse[row] = lse_of(sum);
      logp[row] = logp_of(sum, hit);               // (a label past the vocabulary: NaN)
    }
  }
}

struct Loss {
  int32_t kind, average;
  float beta, smoothing, margin;
};

// The loss of a pair and its derivative by D.  D and z stay in 64 bits as the sums are, and so do the
// parts that are linear in z; e = exp(-|z|) is fp32's, with the rest of z that fp32 drops (2^-24 of z, and
// as much of e) put back.  (exp and log1p in 64 bits would make a call 1.7 us longer: one thread of a
// pair works here, and the GPU's 64-bit units are few.)
__device__ __forceinline__ void pair_loss(const Loss& f, double D, double* loss, double* slope) {
  const double beta = f.beta;
  if (f.kind == ZO_PREFERENCE_SQUARE) {
    const double d = D - 0.5 / beta;
    *loss = d * d;
    *slope = 2.0 * d;
    return;
  }
  const double z = beta * D - (double)f.margin;
  if (f.kind == ZO_PREFERENCE_HINGE) {
    *loss = z < 1.0 ? 1.0 - z : z >= 1.0 ? 0.0 : z;                  // (NaN stays)
    *slope = z < 1.0 ? -beta : z >= 1.0 ? 0.0 : z;
    return;
  }
  // -log sig(z) = log(1 + e) + max(-z, 0), sig(-|z|) = e / (1 + e)
  const float size = fabsf((float)z), near = expf(-size);
  const float e = near > 0.0f ? fmaf(near, (float)((double)size - fabs(z)), near) : near;   // (0: so far that z may be infinite)
  const double far = e / (1.0f + e);
  const double a = f.smoothing;
  // (a product of zero with an infinite side is left out)
  *loss = (double)log1pf(e) + (z < 0.0 ? -z * (1.0 - a) : a > 0.0 ? z * a : z == z ? 0.0 : z);
  *slope = beta * (a - (z < 0.0 ? 1.0 - far : far));                 // a sig(z) - (1 - a) (1 - sig(z))
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// A CTA per pair: half of its warps sum the chosen sequence, half the rejected one, four rows a
// thread at a time.
template <typename T>
__global__ void __launch_bounds__(kPairThreads)
pairs_kernel(const Rows a, const Loss f, const Sum* __restrict__ partial,
             const float* __restrict__ logp, const float* __restrict__ ref, float* __restrict__ lse,
             float* __restrict__ dlogp, float* __restrict__ logps, float* __restrict__ losses,
             float* __restrict__ loss, uint32_t* __restrict__ ticket) {
  constexpr int kPairWarps = kPairThreads / 32, kSide = kPairThreads / 2, kAtOnce = 4;
  __shared__ double sums[kPairWarps], counts[kPairWarps];
  __shared__ float slopes[2];
  __shared__ bool last;
  const int64_t pair = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int side = warp / (kPairWarps / 2);                         // 0: chosen
  const int64_t seq = pair + side * a.pairs;
  const int first = (int)threadIdx.x - side * kSide;
  zo::pdl_wait();
  zo::pdl_trigger();
  // (offsets out of order or range: no row outside the matrix is touched)
  const int64_t begin = min(a.rows, max((int64_t)0, a.offsets[seq])), end = min(a.rows, a.offsets[seq + 1]);
  double sum = 0.0, count = 0.0;
  for (int64_t r0 = begin + first; r0 < end; r0 += kAtOnce * kSide) {
    int64_t label[kAtOnce];
    float lp[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int64_t r = r0 + i * kSide;
      label[i] = r < end ? a.labels[r] : -1;
      lp[i] = r < end && a.parts == 1 ? logp[r] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (label[i] < 0) continue;
      if (a.parts > 1) {
        const int64_t r = r0 + i * kSide;
        Sum s = partial[r * a.parts];
        for (int p = 1; p < a.parts; ++p) s = join(s, partial[r * a.parts + p]);
        if (lse) lse[r] = lse_of(s);
        lp[i] = label[i] < a.vocab
                    ? logp_of(s, static_cast<float>(static_cast<const T*>(a.x)[r * a.ld + label[i]]))
                    : __int_as_float(0x7FC00000);
      }
      sum += (double)lp[i];
      count += 1.0;
    }
  }
  sum = warp_sum(sum);
  count = warp_sum(count);
  if (lane == 0) {
    sums[warp] = sum;
    counts[warp] = count;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double gain[2], n[2];
    for (int k = 0; k < 2; ++k) {
      double s = 0.0;
      n[k] = 0.0;
      for (int w = 0; w < kPairWarps / 2; ++w) {
        s += sums[k * (kPairWarps / 2) + w];
        n[k] += counts[k * (kPairWarps / 2) + w];
      }
      if (f.average && n[k] > 0.0) s /= n[k];
      logps[pair + k * a.pairs] = (float)s;
      gain[k] = s - (ref ? (double)ref[pair + k * a.pairs] : 0.0);
    }
    double value, slope;
    pair_loss(f, gain[0] - gain[1], &value, &slope);
    losses[pair] = (float)value;
    for (int k = 0; k < 2; ++k) {
      const double by = (k ? -1.0 : 1.0) * slope / (double)a.pairs;
      slopes[k] = (float)(f.average && n[k] > 0.0 ? by / n[k] : by);
    }
    __threadfence();
    last = atomicAdd(ticket, 1u) == (uint32_t)a.pairs - 1u;
  }
  __syncthreads();
  if (dlogp) {
    const float d = slopes[side];
    for (int64_t r0 = begin + first; r0 < end; r0 += kAtOnce * kSide) {
      bool counted[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        counted[i] = r0 + i * kSide < end && a.labels[r0 + i * kSide] >= 0;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (counted[i]) dlogp[r0 + i * kSide] = d;
    }
  }
  if (!last) return;
  // the losses of all pairs, in an order of their own
  __threadfence();
  double total = 0.0;
  for (int64_t p = threadIdx.x; p < a.pairs; p += kPairThreads) total += (double)__ldcg(losses + p);
  total = warp_sum(total);
  if (lane == 0) sums[warp] = total;
  __syncthreads();
  if (threadIdx.x == 0) {
    total = 0.0;
    for (int w = 0; w < kPairWarps; ++w) total += sums[w];
    *loss = (float)(total / (double)a.pairs);
  }
}

// The gradient of a part of a row, or of a short row by a warp.
template <typename T, int kTeam>
__global__ void __launch_bounds__(kThreads)
gradient_kernel(const Rows a, const float* __restrict__ lse, const float* __restrict__ dlogp,
                const float* __restrict__ dloss, T* out, int64_t ldo) {
  const int part = (int)(blockIdx.x % (unsigned)a.parts);
  const int member = threadIdx.x % kTeam;
  const int64_t row = blockIdx.x / (unsigned)a.parts * (int64_t)(kThreads / kTeam) + threadIdx.x / kTeam;
  const int64_t j0 = (int64_t)part * a.part_cols;
  const int n = (int)min((int64_t)a.part_cols, a.vocab - j0);
  zo::pdl_wait();
  zo::pdl_trigger();
  if (row >= a.rows || n <= 0) return;                              // (many parts, each rounded up to eight columns)
  const int64_t label = a.labels[row];
  const float share = label < 0 ? 0.0f : dlogp[row];
  const float scale = share == 0.0f ? 0.0f : share * (dloss ? *dloss : 1.0f);   // (dloss may be no number)
  const float base = lse[row];
  // (x and out may be the same memory: a thread writes what it has read itself)
  const T* x = static_cast<const T*>(a.x) + row * a.ld + j0;
  T* y = out + row * ldo + j0;
  const int64_t hit = label - j0;
  const auto grad = [&](float v, int64_t j) {
    return scale * ((j == hit ? 1.0f : 0.0f) - exp_of(v - base));
  };
  const bool zero = scale == 0.0f;
  const int head = head_of(x, n);
  if (head == head_of(y, n)) {
    const int vecs = (n - head) / Vec<T>::kN;
    for (int i = member; i < vecs; i += kUnroll * kTeam) {
      uint4 v[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (!zero && i + u * kTeam < vecs)
          v[u] = __ldcs(reinterpret_cast<const uint4*>(x + head) + i + u * kTeam);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int at = i + u * kTeam;
        if (at >= vecs) break;
        uint4 r = make_uint4(0u, 0u, 0u, 0u);
        if (!zero) {
          Vec<T> w{v[u]};
          const int64_t j = head + (int64_t)at * Vec<T>::kN;
          float g[Vec<T>::kN];
#pragma unroll
          for (int k = 0; k < Vec<T>::kN; ++k) g[k] = grad(w.get(k), j + k);
          uint32_t o[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if constexpr (sizeof(T) == 4) {
              o[k] = __float_as_uint(g[k]);
            } else {
              const __nv_bfloat162 h = __floats2bfloat162_rn(g[2 * k], g[2 * k + 1]);
              o[k] = *reinterpret_cast<const uint32_t*>(&h);
            }
          }
          r = make_uint4(o[0], o[1], o[2], o[3]);
        }
        __stcs(reinterpret_cast<uint4*>(y + head) + at, r);
      }
    }
    const int around = head + (n - head) % Vec<T>::kN;
    if (member < around) {
      const int k = member < head ? member : n - around + member;
      y[k] = static_cast<T>(zero ? 0.0f : grad(static_cast<float>(x[k]), k));
    }
  } else {
    for (int k = member; k < n; k += kTeam)
      y[k] = static_cast<T>(zero ? 0.0f : grad(static_cast<float>(x[k]), k));
  }
}

// ---- host ----------------------------------------------------------------------------------

// Parts of a row: as many as give every SM two CTAs, none narrower than kPartCols.
int32_t parts_of(int64_t rows, int64_t vocab, int32_t sms) {
  int32_t parts = 1;
  while (parts < kMaxParts && rows * parts < 2 * (int64_t)sms && vocab >= 2 * (int64_t)parts * kPartCols)
    parts *= 2;
  return parts;
}

// The CTAs of a call, and whether each of their warps has a row of its own: a CTA's joins and its
// beginning are too much for a short one.  (Rows in several parts are never short ones: a warp takes a
// whole row.)
struct Teams {
  bool warps;
  unsigned ctas;
};
Teams teams_of(const Rows& a, int32_t dtype, int64_t short_bytes) {
  const bool warps = a.parts == 1 && a.vocab * (int64_t)(dtype == ZO_BF16 ? 2 : 4) <= short_bytes;
  return Teams{warps, (unsigned)(warps ? (a.rows + kWarps - 1) / kWarps : a.rows * a.parts)};
}

bool elem_aligned(const void* p, int32_t dtype) {
  return reinterpret_cast<uintptr_t>(p) % (dtype == ZO_BF16 ? 2 : 4) == 0;
}
bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

zo_status check_logits(const void* x, int64_t ld, int64_t rows, int64_t vocab, int32_t dtype) {
  if (dtype != ZO_F32 && dtype != ZO_BF16) return refuse(ZO_ERR_DTYPE, "unknown dtype");
  if (rows < 0 || rows >= (int64_t(1) << 26) || vocab < 1 || vocab >= (int64_t(1) << 26) || ld < vocab ||
      ld >= (int64_t(1) << 40))
    return refuse(ZO_ERR_SHAPE,
                  "zo_preference: need 0 <= rows < 2^26, 1 <= vocab < 2^26 and vocab <= ld < 2^40");
  if (rows > 0 && !x) return refuse(ZO_ERR_INVALID_ARG, "zo_preference: null logits");
  if (!elem_aligned(x, dtype)) return refuse(ZO_ERR_ALIGN, "zo_preference: logits not aligned to their elements");
  return ZO_OK;
}

void set_parts(Rows* a, int32_t parts) {
  a->parts = parts;
  a->part_cols = (a->vocab + 8 * parts - 1) / (8 * parts) * 8;
}

}  // namespace

extern "C" {

int64_t zo_preference_workspace(int64_t rows, int64_t vocab) {
  if (check_logits(reinterpret_cast<const void*>(16), vocab, rows, vocab, ZO_F32) != ZO_OK) return 0;
  // (for any number of SMs up to 256: parts are halved until 2 x 256 CTAs)
  const int64_t parts = parts_of(rows, vocab, 256);
  return 256 + (rows * 4 + 255) / 256 * 256 + (parts > 1 ? rows * parts * (int64_t)sizeof(Sum) : 0);
}

zo_status zo_preference_forward(const void* logits, int64_t ldl, int64_t rows, int64_t vocab,
                                int32_t dtype, const int64_t* labels, const int64_t* offsets,
                                int64_t pairs, const float* ref_logps, int32_t kind, float beta,
                                float smoothing, float margin, int32_t average, float* loss,
                                float* losses, float* logps, float* lse, float* dlogp,
                                void* workspace, int64_t workspace_bytes, void* stream) {
  const zo_status st = check_logits(logits, ldl, rows, vocab, dtype);
  if (st != ZO_OK) return st;
  if (pairs < 1 || pairs >= (int64_t(1) << 24))
    return refuse(ZO_ERR_SHAPE, "zo_preference_forward: need 1 <= pairs < 2^24");
  if (kind < ZO_PREFERENCE_SIGMOID || kind > ZO_PREFERENCE_SQUARE || !(beta > 0.0f) ||
      !std::isfinite(beta) || !std::isfinite(margin) || !(smoothing >= 0.0f && smoothing < 0.5f) ||
      (smoothing != 0.0f && kind != ZO_PREFERENCE_SIGMOID) ||
      (margin != 0.0f && kind == ZO_PREFERENCE_SQUARE))
    return refuse(ZO_ERR_INVALID_ARG,
                  "zo_preference_forward: need a known kind, beta > 0, a finite margin (0 for SQUARE) "
                  "and a smoothing in [0, 0.5) (0 for others than SIGMOID)");
  if ((rows > 0 && !labels) || !offsets || !loss || !losses || !logps)
    return refuse(ZO_ERR_INVALID_ARG, "zo_preference_forward: null labels, offsets, loss, losses or logps");
  if (!aligned_to(labels, 8) || !aligned_to(offsets, 8) || !aligned_to(ref_logps, 4) ||
      !aligned_to(loss, 4) || !aligned_to(losses, 4) || !aligned_to(logps, 4) || !aligned_to(lse, 4) ||
      !aligned_to(dlogp, 4) || !aligned16(workspace))
    return refuse(ZO_ERR_ALIGN, "zo_preference_forward: a buffer is not aligned to its elements "
                                "(the workspace: to 16 bytes)");
  if (!workspace || workspace_bytes < zo_preference_workspace(rows, vocab))
    return refuse(ZO_ERR_INVALID_ARG, "zo_preference_forward: the workspace is missing or smaller "
                                      "than zo_preference_workspace(rows, vocab)");
  const int32_t sms = sm_count();
  if (sms <= 0) return refuse(ZO_ERR_CUDA, "zo_preference_forward: no usable CUDA device");
  const auto s = reinterpret_cast<cudaStream_t>(stream);
  Rows a{};
  a.x = logits;
  a.ld = ldl;
  a.vocab = (int32_t)vocab;
  a.rows = rows;
  a.labels = labels;
  a.offsets = offsets;
  a.pairs = pairs;
  set_parts(&a, parts_of(rows, vocab, sms < 256 ? sms : 256));
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  auto* ticket = reinterpret_cast<uint32_t*>(ws);
  auto* logp = reinterpret_cast<float*>(ws + 256);
  auto* partial = reinterpret_cast<Sum*>(ws + 256 + (rows * 4 + 255) / 256 * 256);
  const auto [warps, ctas] = teams_of(a, dtype, kShortForward);
  const unsigned grid = rows > 0 ? ctas : 1u;
  const Loss f{kind, average != 0, beta, smoothing, margin};
  const bool half = dtype == ZO_BF16;
  using B = __nv_bfloat16;
  const auto rows_fn = half ? (warps ? rows_kernel<B, 32> : rows_kernel<B, kThreads>)
                            : (warps ? rows_kernel<float, 32> : rows_kernel<float, kThreads>);
  ZO_CUDA(zo::launch_dependent(rows_fn, grid, kThreads, 0, s, 1, true, a, partial, logp, lse, dlogp, ticket),
          "preference: rows' kernel");
  ZO_CUDA(zo::launch_dependent(half ? pairs_kernel<__nv_bfloat16> : pairs_kernel<float>,
                               (unsigned)pairs, kPairThreads, 0, s, 1, true, a, f, partial, logp,
                               ref_logps, lse, dlogp, logps, losses, loss, ticket),
          "preference: pairs' kernel");
  return ZO_OK;
}

zo_status zo_preference_backward(const void* logits, int64_t ldl, int64_t rows, int64_t vocab,
                                 int32_t dtype, const int64_t* labels, const float* lse,
                                 const float* dlogp, const float* dloss, void* dlogits, int64_t ldd,
                                 void* stream) {
  const zo_status st = check_logits(logits, ldl, rows, vocab, dtype);
  if (st != ZO_OK) return st;
  if (ldd < vocab || ldd >= (int64_t(1) << 40))
    return refuse(ZO_ERR_SHAPE, "zo_preference_backward: need vocab <= ldd < 2^40");
  if (rows == 0) return ZO_OK;
  if (!labels || !lse || !dlogp || !dlogits)
    return refuse(ZO_ERR_INVALID_ARG, "zo_preference_backward: null labels, lse, dlogp or dlogits");
  if (logits == dlogits && ldl != ldd)
    return refuse(ZO_ERR_INVALID_ARG, "zo_preference_backward: in place, the strides have to agree");
  if (!aligned_to(labels, 8) || !aligned_to(lse, 4) || !aligned_to(dlogp, 4) || !aligned_to(dloss, 4) ||
      !elem_aligned(dlogits, dtype))
    return refuse(ZO_ERR_ALIGN, "zo_preference_backward: a buffer is not aligned to its elements");
  const int32_t sms = sm_count();
  if (sms <= 0) return refuse(ZO_ERR_CUDA, "zo_preference_backward: no usable CUDA device");
  Rows a{};
  a.x = logits;
  a.ld = ldl;
  a.vocab = (int32_t)vocab;
  a.rows = rows;
  a.labels = labels;
  set_parts(&a, (int32_t)std::max<int64_t>(parts_of(rows, vocab, sms), vocab / kGradCols));
  const auto s = reinterpret_cast<cudaStream_t>(stream);
  if (rows * a.parts > INT32_MAX)
    return refuse(ZO_ERR_SHAPE, "zo_preference_backward: too many logits for one call");
  const auto [warps, grid] = teams_of(a, dtype, kShortBackward);
  using B = __nv_bfloat16;
  if (dtype == ZO_BF16)
    ZO_CUDA(zo::launch_dependent(warps ? gradient_kernel<B, 32> : gradient_kernel<B, kThreads>, grid,
                                 kThreads, 0, s, 1, true, a, lse, dlogp, dloss, static_cast<B*>(dlogits), ldd),
            "preference: gradient kernel");
  else
    ZO_CUDA(zo::launch_dependent(warps ? gradient_kernel<float, 32> : gradient_kernel<float, kThreads>,
                                 grid, kThreads, 0, s, 1, true, a, lse, dlogp, dloss,
                                 static_cast<float*>(dlogits), ldd),
            "preference: gradient kernel");
  return ZO_OK;
}

}  // extern "C"
