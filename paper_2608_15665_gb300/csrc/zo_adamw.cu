// The AdamW step over many tensors at once: host runtime, C ABI (declared in include/zo.h) and
// the kernel, one launch for all tensors (two where the device counts the steps).
//
//   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2
//   W <- rnd((1 - lr wd) W - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps))
//
// Bound by HBM with fp32 states (50M bf16 elements, 22 bytes each: 159 us, 103% of the copy rate), by
// instruction issue with 8-bit ones (131M: 245 us, 79%): W is read and written, g read, the states
// read and written, once each.  A warp
// works on blocks of 256 neighbouring elements, eight to a lane; a CTA on a chunk of one tensor,
// found in a table of the chunks.
//
// States in 8 bits: m and r = sqrt(v) as e4m3 codes times 2^(E - 134), E = the biased fp32
// exponent of the largest |m| (r) of the block of 256, in one byte; so the block's largest is in
// [128, 256], and values down to 2^-17 of it keep a code (where the largest v is subnormal, E is 63).  r and not v: the codes reach over 17
// binades, v's spread is twice that of r.  Codes are rounded up or down at random, by 16 bits of
// the Philox stream an element, as v moves by a thousandth of itself a step and the codes are an
// eighth apart: to nearest, a running mean would never move.  The expectation is the running
// mean's; its noise settles where what a step adds, |dr| times a code's distance, is what the mean
// forgets: about 15% of r for Gaussian gradients and b2 = 0.999.  m and r take the same bits: the two errors are not used
// together.  A root above zero keeps a code above zero, or m / eps would be taken as the update.
// The moments' sums are products and sums each rounded on its own: the exponents are then the
// same as those of any other fp32 evaluation in this order.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>
#include <type_traits>
#include <unordered_set>
#include <vector>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "../../include/zo.h"
#include "zo_device.cuh"
#include "zo_host.h"
#include "zo_launch.cuh"

namespace {

using namespace zo::host;

constexpr uint32_t kTagAdamW = 6;
constexpr int kThreads = 128, kLane = 8;
constexpr int kBlock = 32 * kLane;               // elements of a power of two
constexpr int kRow = kThreads * kLane;           // a block of every warp
constexpr int kMaxUnits = 8;                     // such rows of a chunk, at most
constexpr int kCtas = 7;                         // of an SM
// 8 bits: a warp's ring of blocks in shared memory (W and G in fp32 at most)
constexpr int kStages = 2, kStageBytes = kBlock * 10;
constexpr int kRingBytes = kThreads / 32 * kStages * kStageBytes;
static_assert(kRingBytes <= 48 * 1024 && kCtas * kRingBytes <= 227 * 1024, "shared memory");
static_assert(kBlock == 256 && kRow % kBlock == 0 && kMaxUnits <= 32, "a chunk is whole blocks");

struct Tensor {
  void* W;
  const void* G;
  void *M, *V;                                   // fp32, or codes
  uint8_t *Em, *Ev;                              // exponents (8 bits)
  int64_t n, cols, ldw, ldg;                     // elements; of a row, and the rows' strides
  int32_t kind;                                  // bit 0: W is bf16; bit 1: G is bf16
  int32_t wide;                                  // contiguous, and aligned to a lane's accesses
};

// What a step is made of: the update is rate m / (sqrt(v) spread + eps).
struct Now {                                     // what goes by the step's number
  float rate, spread;                            // -lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  uint32_t t;
};
struct Step {
  float b1, one_b1, b2, one_b2, keep, eps;
  float none;                                    // -0: what a product is added to
  uint32_t key[20];                              // of Philox's rounds
};
__host__ __device__ inline Now now_of(int64_t t, double lr, double b1, double b2) {
  return Now{(float)(lr / expm1((double)t * log(b1))),
             (float)(1.0 / sqrt(-expm1((double)t * log(b2)))), (uint32_t)t};
}

// Philox4x32-10 of zo_device.cuh with the rounds' keys given: they are the same for all threads.
__device__ __forceinline__ uint4 random_words(uint4 c, const uint32_t (&key)[20]) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ key[2 * r], (uint32_t)b,
                   (uint32_t)(a >> 32) ^ c.w ^ key[2 * r + 1], (uint32_t)a);
  }
  return c;
}

// One more step: its number and bias corrections.
__global__ void adamw_count_kernel(int64_t* count, double lr, double b1, double b2, Now* out) {
  zo::pdl_wait();
  int64_t t = *count;
  t = t < 0 ? 1 : t + 1;
  *count = t;
  *out = now_of(t, lr, b1, b2);
}

__device__ __forceinline__ uint32_t smem_u32(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

// Eight values of a lane as they lie in memory.
template <typename T>
struct Raw {
  static constexpr int kWords = 2 * (int)sizeof(T);
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (sizeof(T) == 1) {
      const uint2 a = __ldcs(reinterpret_cast<const uint2*>(p));
      w[0] = a.x;
      w[1] = a.y;
    } else {
#pragma unroll
      for (int q = 0; q < kWords; q += 4) {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p) + q / 4);
        w[q] = a.x;
        w[q + 1] = a.y;
        w[q + 2] = a.z;
        w[q + 3] = a.w;
      }
    }
  }
  // to shared memory, asynchronously, and from there
  static __device__ __forceinline__ void fetch(uint8_t* to, const T* p) {
    if constexpr (sizeof(T) == 1) {
      asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(to)), "l"(p) : "memory");
    } else {
#pragma unroll
      for (int q = 0; q < kWords / 4; ++q)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to + 512 * q)),
                     "l"(p + q * (16 / sizeof(T)))
                     : "memory");
    }
  }
  __device__ __forceinline__ void take(const uint8_t* from) {
    if constexpr (sizeof(T) == 1) {
      const uint2 a = *reinterpret_cast<const uint2*>(from);
      w[0] = a.x;
      w[1] = a.y;
    } else {
#pragma unroll
      for (int q = 0; q < kWords; q += 4) {
        const uint4 a = *reinterpret_cast<const uint4*>(from + 128 * q);
        w[q] = a.x;
        w[q + 1] = a.y;
        w[q + 2] = a.z;
        w[q + 3] = a.w;
      }
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (sizeof(T) == 1) {
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
      for (int q = 0; q < kWords; q += 4)
        reinterpret_cast<uint4*>(p)[q / 4] = make_uint4(w[q], w[q + 1], w[q + 2], w[q + 3]);
    }
  }
  // element by element, `n` of them from place e0 on, in rows of `cols` elements `ld` apart
  __device__ __forceinline__ void gather(const T* p, int64_t e0, int n, int64_t cols, int64_t ld) {
#pragma unroll
    for (int q = 0; q < kWords; ++q) w[q] = 0u;
    if (n == 0) return;
    int64_t row = cols == ld ? 0 : e0 / cols, col = e0 - row * cols;
#pragma unroll
    for (int e = 0; e < kLane; ++e) {
      if (e < n) {
        const T x = p[row * ld + col];
        uint32_t bits;
        if constexpr (sizeof(T) == 4) bits = __float_as_uint(x);
        else if constexpr (sizeof(T) == 2) bits = __bfloat16_as_ushort(x);
        else bits = x;
        w[e / kPer] |= bits << (kBits * (e % kPer));
      }
      step(row, col, cols, ld);
    }
  }
  __device__ __forceinline__ void scatter(T* p, int64_t e0, int n, int64_t cols, int64_t ld) const {
    if (n == 0) return;
    int64_t row = cols == ld ? 0 : e0 / cols, col = e0 - row * cols;
#pragma unroll
    for (int e = 0; e < kLane; ++e) {
      if (e < n) {
        const uint32_t bits = w[e / kPer] >> (kBits * (e % kPer));
        if constexpr (sizeof(T) == 4) p[row * ld + col] = __uint_as_float(bits);
        else if constexpr (sizeof(T) == 2)
          p[row * ld + col] = __ushort_as_bfloat16((unsigned short)bits);
        else p[row * ld + col] = (T)bits;
      }
      step(row, col, cols, ld);
    }
  }

 private:
  static constexpr int kBits = 8 * (int)sizeof(T), kPer = 32 / kBits;
  static __device__ __forceinline__ void step(int64_t& row, int64_t& col, int64_t cols, int64_t ld) {
    if (++col == cols && cols != ld) {
      col = 0;
      ++row;
    }
  }
};

template <typename T>
__device__ __forceinline__ void unpack(const Raw<T>& r, float (&x)[kLane]) {
#pragma unroll
  for (int e = 0; e < kLane; ++e) {
    if constexpr (sizeof(T) == 4) x[e] = __uint_as_float(r.w[e]);
    else x[e] = __uint_as_float(e & 1 ? r.w[e / 2] & 0xFFFF0000u : r.w[e / 2] << 16);
  }
}
template <typename T>
__device__ __forceinline__ void pack(const float (&x)[kLane], Raw<T>& r) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < kLane; ++e) r.w[e] = __float_as_uint(x[e]);
  } else {
#pragma unroll
    for (int e = 0; e < kLane; e += 2) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[e], x[e + 1]);
      r.w[e / 2] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
}

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// ---- 8-bit states ------------------------------------------------------------------------
// The kernel's instructions are what this path has to save: at HBM's rate an SM has 55 issue slots
// an element.  So products and sums go two to an instruction, random bits and codes move by byte
// permutations, and what is rare (a number that is not finite, a root whose code is 0) is found by a
// maximum over the block and mended apart.
__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }

// Eight e4m3 codes times 2^(E - 134).
__device__ __forceinline__ void decode(const Raw<uint8_t>& r, uint32_t E, float (&x)[kLane]) {
  const float2 s = both(power((int)max(E, 40u) - 134));
#pragma unroll
  for (int q = 0; q < kLane / 2; ++q) {
    const __half2 h = __nv_cvt_fp8x2_to_halfraw2(
        (__nv_fp8x2_storage_t)(r.w[q / 2] >> (16 * (q & 1))), __NV_E4M3);
    const float2 f = zo::mul2(__half22float2(h), s);
    x[2 * q] = f.x;
    x[2 * q + 1] = f.y;
  }
}

// Codes of x of a block whose largest finite |x| is `top` (bits, 2^(E - 127) its power of two).
// x 2^(134 - E) 2^-120 is laid out like the code: its exponent field, and its subnormal numbers,
// begin where e4m3's do.  So the code is the fp32 bits without the last 20, rounded up where
// these and the random bits carry; all of it is formed four bits further left, where the code is
// the topmost byte below the sign.  (The product rounds subnormals at 2^-20 of a code's step.)
// odd: the block holds something not finite, which becomes NaN.
template <bool kSigned>
__device__ __forceinline__ void encode(const float (&x)[kLane], uint32_t E, bool odd,
                                       const uint4& random, Raw<uint8_t>& r) {
  const int e40 = max((int)E, 40);
  const float2 s = both(power(14 - min(e40, 140)));
  const uint32_t rw[4] = {random.x, random.y, random.z, random.w};
  uint32_t c[kLane];
  float y[kLane];
#pragma unroll
  for (int e = 0; e < kLane; e += 2) {
    float2 v = make_float2(x[e], x[e + 1]);
    if (e40 > 140) v = zo::mul2(v, both(power(140 - e40)));     // (their power leaves fp32's range)
    v = zo::mul2(v, s);
    y[e] = v.x;
    y[e + 1] = v.y;
  }
#pragma unroll
  for (int e = 0; e < kLane; ++e) {
    const uint32_t add = __byte_perm(rw[e / 2], 0, e & 1 ? 0x4324 : 0x4104);
    const uint32_t bits = (__float_as_uint(y[e]) << 4) + add;
    if constexpr (kSigned) c[e] = (bits & 0x7FFFFFFFu) | (__float_as_uint(x[e]) & 0x80000000u);
    else c[e] = bits;
  }
  if constexpr (!kSigned) {
    uint32_t least = c[0];
#pragma unroll
    for (int e = 1; e < kLane; ++e) least = min(least, c[e]);
    if (least < 0x01000000u) {                       // above zero stays above zero
#pragma unroll
      for (int e = 0; e < kLane; ++e)
        if (x[e] > 0.0f) c[e] = max(c[e], 0x01000000u);
    }
  }
  if (odd) {
#pragma unroll
    for (int e = 0; e < kLane; ++e)
      if (!(fabsf(x[e]) < __int_as_float(0x7F800000)))
        c[e] = 0x7F000000u | (__float_as_uint(x[e]) & 0x80000000u);
  }
#pragma unroll
  for (int q = 0; q < 2; ++q)
    r.w[q] = __byte_perm(__byte_perm(c[4 * q], c[4 * q + 1], 0x0073),
                         __byte_perm(c[4 * q + 2], c[4 * q + 3], 0x0073), 0x5410);
}

// The largest finite |x| of the warp's block, as bits; odd: there are others.  kSigned = false: x has
// no negative values, and NaN and infinity are the largest bits.
template <bool kSigned>
__device__ __forceinline__ uint32_t largest(const float (&x)[kLane], bool* odd) {
  uint32_t top;
  if constexpr (kSigned) {
    // (a NaN is no maximum, but it and infinity spoil a sum of zeros)
    float most = 0.0f;
    float2 zeros = both(0.0f);
#pragma unroll
    for (int e = 0; e < kLane; e += 2) {
      most = fmaxf(fmaxf(most, fabsf(x[e])), fabsf(x[e + 1]));
      zeros = zo::fma2(make_float2(x[e], x[e + 1]), both(0.0f), zeros);
    }
    *odd = __any_sync(0xffffffffu, zeros.x + zeros.y != 0.0f);
    top = __reduce_max_sync(0xffffffffu, __float_as_uint(most));
  } else {
    top = __float_as_uint(x[0]);
#pragma unroll
    for (int e = 1; e < kLane; ++e) top = max(top, __float_as_uint(x[e]));
    top = __reduce_max_sync(0xffffffffu, top);
    *odd = top >= 0x7F800000u;
  }
  if (*odd) {
    top = 0;
#pragma unroll
    for (int e = 0; e < kLane; ++e) {
      const uint32_t b = __float_as_uint(x[e]) & 0x7FFFFFFFu;
      if (b < 0x7F800000u) top = max(top, b);
    }
    top = __reduce_max_sync(0xffffffffu, top);
  }
  return top;
}

__device__ __forceinline__ float root_of(float v) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// Square roots rounded to nearest, of 2^-102 <= v < infinity (smaller ones may come out too small, by
// less than 2^-65): the hardware's reciprocal root y, s = v y, and one Newton step by the residual,
// s + (v - s^2) y / 2 (Markstein, IBM J. Res. Dev. 34, 1990).  So a state's codes are those of any
// other fp32 evaluation.  (Infinity gives NaN, which its code would be in any case.)
__device__ __forceinline__ float2 rounded_roots(float2 v) {
  const float2 u = zo::add2(v, both(0x1p-126f));      // (0 has no reciprocal root; others keep theirs)
  float2 y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(u.x));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(u.y));
  const float2 s = zo::mul2(v, y);
  const float2 rest = zo::fma2(zo::mul2(s, both(-1.0f)), s, v);
  return zo::fma2(rest, zo::mul2(y, both(0.5f)), s);
}
// Roots of any v, subnormal ones too, rounded to nearest.  (Infinity gives NaN here as well.)
template <bool kEight>
__device__ __forceinline__ float exact_root(float v) {
  return kEight ? __fsqrt_rn(v) + (v - v) : __fsqrt_rn(v);
}
__device__ __forceinline__ float reciprocal(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// A lane's eight elements, from e0 on, of which the first `count` are the tensor's.
template <bool kEight, typename W, typename G>
struct Unit {
  using S = std::conditional_t<kEight, uint8_t, float>;
  Raw<W> w;
  Raw<G> g;
  Raw<S> m, v;
  uint32_t em, ev;
  int64_t e0;
  int count;

  __device__ __forceinline__ void at(const Tensor& t, int64_t first) {
    e0 = first;
    count = (int)max((int64_t)0, min((int64_t)kLane, t.n - e0));
  }
  __device__ __forceinline__ void load(const Tensor& t, int64_t first) {
    at(t, first);
    const W* pw = static_cast<const W*>(t.W);
    const G* pg = static_cast<const G*>(t.G);
    const S *pm = static_cast<const S*>(t.M), *pv = static_cast<const S*>(t.V);
    if (t.wide && count == kLane) {
      w.load(pw + e0);
      g.load(pg + e0);
      m.load(pm + e0);
      v.load(pv + e0);
    } else {
      w.gather(pw, e0, count, t.cols, t.ldw);
      g.gather(pg, e0, count, t.cols, t.ldg);
      m.gather(pm, e0, count, t.cols, t.cols);
      v.gather(pv, e0, count, t.cols, t.cols);
    }
    if constexpr (kEight) {
      const bool any = __shfl_sync(0xffffffffu, count, 0) > 0;
      // (bytes of a line that other SMs write: from L2)
      em = any ? __ldcg(t.Em + e0 / kBlock) : 0u;
      ev = any ? __ldcg(t.Ev + e0 / kBlock) : 0u;
    }
  }
  // Through a warp's stage of shared memory: a lane takes what it has fetched itself.
  static constexpr int g_at() { return 32 * kLane * (int)sizeof(W); }
  static constexpr int m_at() { return g_at() + 32 * kLane * (int)sizeof(G); }
  static __device__ __forceinline__ void fetch(const W* pw, const G* pg, const S* pm, const S* pv,
                                               uint8_t* stage) {
    const int lane = threadIdx.x & 31;
    Raw<W>::fetch(stage + 16 * lane, pw);
    Raw<G>::fetch(stage + g_at() + 16 * lane, pg);
    Raw<S>::fetch(stage + m_at() + 8 * lane, pm);
    Raw<S>::fetch(stage + m_at() + 256 + 8 * lane, pv);
  }
  __device__ __forceinline__ void take(const uint8_t* stage, uint32_t e_m, uint32_t e_v) {
    const int lane = threadIdx.x & 31;
    w.take(stage + 16 * lane);
    g.take(stage + g_at() + 16 * lane);
    m.take(stage + m_at() + 8 * lane);
    v.take(stage + m_at() + 256 + 8 * lane);
    em = e_m;
    ev = e_v;
  }

  // word: of the lane's eight elements in the stream of random words
  template <bool kExact>
  __device__ __forceinline__ void compute(uint32_t word, uint32_t index, const Step& st, const Now& now) {
    float x[kLane], y[kLane], a[kLane], b[kLane];
    unpack(g, y);
    if constexpr (kEight) {
      decode(m, em, a);
      decode(v, ev, b);
    } else {
      unpack(m, a);
      unpack(v, b);
    }
    unpack(w, x);
    const float2 rate = both(now.rate), spread = both(now.spread), keep = both(st.keep);
    const float2 b1 = both(st.b1), c1 = both(st.one_b1), b2 = both(st.b2), c2 = both(st.one_b2);
    const float2 none = both(st.none);
#pragma unroll
    for (int e = 0; e < kLane; e += 2) {
      const float2 gr = make_float2(y[e], y[e + 1]);
      float2 m2 = make_float2(a[e], a[e + 1]), v2 = make_float2(b[e], b[e + 1]);
      if constexpr (kEight) v2 = zo::mul2(v2, v2);
      // (products that a sum follows: as fused operations with a zero that the compiler does not
      // know, or it would fuse the sum instead)
      m2 = zo::add2(zo::fma2(b1, m2, none), zo::fma2(c1, gr, none));
      v2 = zo::add2(zo::fma2(b2, v2, none), zo::fma2(c2, zo::mul2(gr, gr), none));
      const float2 root = kExact   ? make_float2(exact_root<kEight>(v2.x), exact_root<kEight>(v2.y))
                          : kEight ? rounded_roots(v2)
                                   : make_float2(root_of(v2.x), root_of(v2.y));
      const float2 den = zo::fma2(root, spread, both(st.eps));
      const float2 move = zo::mul2(zo::mul2(rate, m2), make_float2(reciprocal(den.x), reciprocal(den.y)));
      const float2 to = zo::fma2(keep, make_float2(x[e], x[e + 1]), move);
      x[e] = to.x, x[e + 1] = to.y;
      y[e] = root.x, y[e + 1] = root.y;
      a[e] = m2.x, a[e + 1] = m2.y;
      b[e] = v2.x, b[e + 1] = v2.y;
    }
    pack(x, w);
    if constexpr (kEight) {
      bool odd_m, odd_v;
      const uint32_t tm = largest<true>(a, &odd_m), tv = largest<false>(b, &odd_v);
      // 2^k <= r < 2^(k + 1) where 2^2k <= v < 2^(2k + 2); of a subnormal v, r < 2^-63 gets the power
      // of two of the numbers above it, which leaves it 14 binades of codes (down to 2^-77, where v
      // ends at 2^-149)
      em = tm >> 23;
      ev = tv != 0u ? ((tv >> 23) + 127u) >> 1 : 0u;
      const uint4 random = random_words(
          make_uint4(word, index, now.t, kTagAdamW << 24), st.key);
      encode<true>(a, em, odd_m, random, m);
      encode<false>(y, ev, odd_v, random, v);
    } else {
      pack(a, m);
      pack(b, v);
    }
  }

  template <bool kExact>
  __device__ __forceinline__ void finish(const Tensor& t, uint32_t index, const Step& st, const Now& now) {
    compute<kExact>((uint32_t)(e0 / kLane), index, st, now);
    if constexpr (kEight) {
      const bool any = __shfl_sync(0xffffffffu, count, 0) > 0;
      if (any && (threadIdx.x & 31) == 0) {
        t.Em[e0 / kBlock] = (uint8_t)em;
        t.Ev[e0 / kBlock] = (uint8_t)ev;
      }
    }
    W* pw = static_cast<W*>(t.W);
    S *pm = static_cast<S*>(t.M), *pv = static_cast<S*>(t.V);
    if (t.wide && count == kLane) {
      w.store(pw + e0);
      m.store(pm + e0);
      v.store(pv + e0);
    } else {
      w.scatter(pw, e0, count, t.cols, t.ldw);
      m.scatter(pm, e0, count, t.cols, t.cols);
      v.scatter(pv, e0, count, t.cols, t.cols);
    }
  }
};

// `units` blocks of every warp, kRow elements apart.  In 8 bits, where a block's arithmetic takes
// as long as its loads, whole blocks of aligned tensors come through shared memory, the next one's
// loads under this one's arithmetic: with loads into registers 24 warps an SM waited half of their
// time (131M elements, bf16: 386 us; through shared memory 247 with three blocks ahead and 24 warps,
// 229 with two and 28, 245 with roots rounded to nearest: 460 instructions a block, 2.9 a cycle,
// the FMA and the ALU pipe each busy half of the time and in turn in the warps' way).
template <bool kEight, bool kExact, typename W, typename G>
__device__ __forceinline__ void run_chunk(const Tensor& t, int64_t first, int units, uint32_t index,
                                          const Step& st, const Now& now) {
  int64_t e0 = first + (int64_t)threadIdx.x * kLane;
  int k = 0;
  Unit<kEight, W, G> u;
  if constexpr (kEight) {
    extern __shared__ __align__(16) uint8_t ring[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* const mine = ring + warp * kStages * kStageBytes;
    const int64_t begin = first + (int64_t)warp * kBlock;
    // this warp's whole blocks
    const int whole = !t.wide || t.n < begin + kBlock ? 0
                      : (int)min((int64_t)units, (t.n - begin - kBlock) / kRow + 1);
    uint32_t em = 0, ev = 0;                     // lane l: of block l
    const int64_t block = begin / kBlock + (int64_t)lane * (kRow / kBlock);
    if (lane < whole) {
      em = __ldcg(t.Em + block);
      ev = __ldcg(t.Ev + block);
    }
    using U = Unit<kEight, W, G>;
    W* const pw = static_cast<W*>(t.W) + e0;
    const G* const pg = static_cast<const G*>(t.G) + e0;
    uint8_t *const pm = static_cast<uint8_t*>(t.M) + e0, *const pv = static_cast<uint8_t*>(t.V) + e0;
    const uint32_t word = (uint32_t)(e0 / kLane);
    const auto fetch = [&](int q) {
      const int o = q * kRow;
      if (q < whole) U::fetch(pw + o, pg + o, pm + o, pv + o, mine + q % kStages * kStageBytes);
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int q = 0; q < kStages - 1; ++q) fetch(q);
    for (; k < whole; ++k) {
      fetch(k + kStages - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      u.take(mine + k % kStages * kStageBytes, __shfl_sync(0xffffffffu, em, k),
             __shfl_sync(0xffffffffu, ev, k));
      u.template compute<kExact>(word + (uint32_t)(k * (kRow / kLane)), index, st, now);
      const int o = k * kRow;
      u.w.store(pw + o);
      u.m.store(pm + o);
      u.v.store(pv + o);
      if (lane == k) em = u.em, ev = u.ev;
    }
    if (lane < whole) {
      t.Em[block] = (uint8_t)em;
      t.Ev[block] = (uint8_t)ev;
    }
  }
  for (; k < units; ++k) {
    u.load(t, e0 + (int64_t)k * kRow);
    u.template finish<kExact>(t, index, st, now);
  }
}

// chunks: (tensor, number of the chunk in it).  kExact: for an eps so small that the hardware's roots of
// small v would show beside it.
template <bool kEight, bool kExact>
__global__ void __launch_bounds__(kThreads, kEight ? kCtas : 8)
adamw_kernel(const Tensor* __restrict__ tensors, const int2* __restrict__ chunks, int units,
             const __grid_constant__ Step st, Now now, const Now* __restrict__ counted) {
  const int2 at = chunks[blockIdx.x];
  const Tensor t = tensors[at.x];
  zo::pdl_wait();
  zo::pdl_trigger();
  if (counted) now = *counted;
  const int64_t first = (int64_t)at.y * units * kRow;
  using B = __nv_bfloat16;
  switch (t.kind) {
    case 0: run_chunk<kEight, kExact, float, float>(t, first, units, (uint32_t)at.x, st, now); break;
    case 1: run_chunk<kEight, kExact, B, float>(t, first, units, (uint32_t)at.x, st, now); break;
    case 2: run_chunk<kEight, kExact, float, B>(t, first, units, (uint32_t)at.x, st, now); break;
    default: run_chunk<kEight, kExact, B, B>(t, first, units, (uint32_t)at.x, st, now); break;
  }
}

// ---- host ----------------------------------------------------------------------------------

zo_status check_tensor(const zo_adamw_tensor& t, int32_t bits) {
  if ((t.dtype != ZO_F32 && t.dtype != ZO_BF16) || (t.grad_dtype != ZO_F32 && t.grad_dtype != ZO_BF16))
    return refuse(ZO_ERR_DTYPE, "unknown dtype in zo_adamw_tensor");
  if (t.m < 0 || t.n < 0 || t.m >= (int64_t(1) << 34) || t.n >= (int64_t(1) << 34) ||
      (t.n > 0 && t.m > (int64_t(1) << 34) / t.n) || t.ldw < t.n || t.ldg < t.n ||
      t.ldw >= (int64_t(1) << 40) || t.ldg >= (int64_t(1) << 40))
    return refuse(ZO_ERR_SHAPE, "zo_adamw_tensor: need 0 <= m, n; m n <= 2^34; n <= ldw, ldg < 2^40");
  if (t.m * t.n == 0) return ZO_OK;
  if (!t.W || !t.G || !t.M || !t.V || (bits == 8 && (!t.Em || !t.Ev)))
    return refuse(ZO_ERR_INVALID_ARG, "null W, G, M or V (with 8 bits: Em or Ev) in zo_adamw_tensor");
  const auto aligned = [](const void* p, int bytes) {
    return reinterpret_cast<uintptr_t>(p) % bytes == 0;
  };
  if (!aligned(t.W, t.dtype == ZO_BF16 ? 2 : 4) || !aligned(t.G, t.grad_dtype == ZO_BF16 ? 2 : 4) ||
      (bits == 32 && (!aligned(t.M, 4) || !aligned(t.V, 4))))
    return refuse(ZO_ERR_ALIGN, "zo_adamw_tensor: a buffer is not aligned to its elements");
  return ZO_OK;
}

zo_status check_tensors(const zo_adamw_tensor* ts, int32_t n, int32_t bits) {
  if (!ts || n <= 0) return refuse(ZO_ERR_INVALID_ARG, "zo_adamw: need at least one tensor");
  if (bits != 8 && bits != 32)
    return refuse(ZO_ERR_UNSUPPORTED, "zo_adamw: states are held in 8 or in 32 bits");
  int64_t chunks = 0;
  for (int32_t i = 0; i < n; ++i) {
    const zo_status st = check_tensor(ts[i], bits);
    if (st != ZO_OK) return st;
    chunks += (ts[i].m * ts[i].n + kRow - 1) / kRow;
  }
  if (chunks > INT_MAX) return refuse(ZO_ERR_SHAPE, "zo_adamw: too many elements for one context");
  return ZO_OK;
}

// Whatever a step writes is written by one tensor alone.
zo_status check_distinct(const zo_adamw_tensor* ts, int32_t n, int32_t bits) {
  std::unordered_set<const void*> seen;
  for (int32_t i = 0; i < n; ++i) {
    if (ts[i].m * ts[i].n == 0) continue;
    const void* own[5] = {ts[i].W, ts[i].M, ts[i].V, ts[i].Em, ts[i].Ev};
    for (int k = 0; k < (bits == 8 ? 5 : 3); ++k)
      if (!seen.insert(own[k]).second)
        return refuse(ZO_ERR_INVALID_ARG, "zo_adamw_create: a buffer that a step writes is given twice");
  }
  return ZO_OK;
}

struct Layout {
  int64_t tensors_at = 0, chunks_at = 0, bytes = 0, chunks = 0;
  int32_t units = 1;
};
int64_t round_up(int64_t v) { return (v + 255) / 256 * 256; }
int64_t chunks_of(const zo_adamw_tensor* ts, int32_t n, int64_t units) {
  int64_t chunks = 0;
  for (int32_t i = 0; i < n; ++i) chunks += (ts[i].m * ts[i].n + units * kRow - 1) / (units * kRow);
  return chunks;
}
// 8 bits: chunks as long as leave some of them to every CTA that a GPU of 152 SMs holds.
Layout layout(const zo_adamw_tensor* ts, int32_t n, int32_t bits) {
  Layout L;
  while (bits == 8 && L.units < kMaxUnits && chunks_of(ts, n, 2 * L.units) >= 4 * 152 * kCtas) L.units *= 2;
  L.chunks = chunks_of(ts, n, L.units);
  L.tensors_at = 256;                                      // Now
  L.chunks_at = round_up(L.tensors_at + (int64_t)sizeof(Tensor) * n);
  L.bytes = round_up(L.chunks_at + (int64_t)sizeof(int2) * L.chunks);
  return L;
}

}  // namespace

struct zo_adamw_ctx {
  int device = 0;
  cudaStream_t stream = nullptr;
  Layout plan;
  uint8_t* ws = nullptr;
  int32_t bits = 32;
  uint64_t seed = 0;
  int64_t launches = 0;
};

extern "C" {

int64_t zo_adamw_workspace(const zo_adamw_tensor* tensors, int32_t n_tensors, int32_t bits) {
  return check_tensors(tensors, n_tensors, bits) == ZO_OK ? layout(tensors, n_tensors, bits).bytes : 0;
}

zo_status zo_adamw_create(zo_adamw_ctx** out, const zo_adamw_tensor* tensors, int32_t n_tensors,
                          int32_t bits, uint64_t seed, void* workspace, int64_t workspace_bytes,
                          void* stream) {
  if (!out) return ZO_ERR_INVALID_ARG;
  *out = nullptr;
  try {
    zo_status st = check_tensors(tensors, n_tensors, bits);
    if (st == ZO_OK) st = check_distinct(tensors, n_tensors, bits);
    if (st != ZO_OK) return st;
    const Layout L = layout(tensors, n_tensors, bits);
    if (!workspace || workspace_bytes < L.bytes)
      return refuse(ZO_ERR_INVALID_ARG,
                    "zo_adamw_create: the workspace is missing or smaller than zo_adamw_workspace");
    if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
      return refuse(ZO_ERR_ALIGN, "zo_adamw_create: the workspace must be 256-byte aligned");
    int dev = 0, major = 0, minor = 0;
    ZO_CUDA(cudaGetDevice(&dev), "cudaGetDevice");
    ZO_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev), "device");
    ZO_CUDA(cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev), "device");
    if (major != 10 || minor != 3)
      return refuse(ZO_ERR_CUDA, "this library is built for sm_103a (GB300) only");
    std::unique_ptr<zo_adamw_ctx> c(new zo_adamw_ctx());
    c->device = dev;
    c->stream = reinterpret_cast<cudaStream_t>(stream);
    c->plan = L;
    c->ws = static_cast<uint8_t*>(workspace);
    c->bits = bits;
    c->seed = seed;
    std::vector<uint8_t> image((size_t)L.bytes, 0);
    auto* ts = reinterpret_cast<Tensor*>(image.data() + L.tensors_at);
    auto* chunks = reinterpret_cast<int2*>(image.data() + L.chunks_at);
    for (int32_t i = 0; i < n_tensors; ++i) {
      const zo_adamw_tensor& s = tensors[i];
      Tensor& d = ts[i];
      d.W = s.W;
      d.G = s.G;
      d.M = s.M;
      d.V = s.V;
      d.Em = s.Em;
      d.Ev = s.Ev;
      d.n = s.m * s.n;
      // one row is contiguous, and so are rows without a gap
      const bool flat_w = s.m <= 1 || s.ldw == s.n, flat_g = s.m <= 1 || s.ldg == s.n;
      d.cols = flat_w && flat_g ? d.n : s.n;
      d.ldw = flat_w ? d.cols : s.ldw;
      d.ldg = flat_g ? d.cols : s.ldg;
      d.kind = (s.dtype == ZO_BF16 ? 1 : 0) | (s.grad_dtype == ZO_BF16 ? 2 : 0);
      const auto to16 = [](const void* p) { return aligned16(p); };
      d.wide = flat_w && flat_g && to16(s.W) && to16(s.G) && to16(s.M) && to16(s.V);
      for (int64_t k = 0; k * L.units * kRow < d.n; ++k) *chunks++ = make_int2(i, (int)k);
    }
    ZO_CUDA(cudaMemcpyAsync(c->ws, image.data(), image.size(), cudaMemcpyHostToDevice, c->stream),
            "upload tables");
    // (a copy from pageable memory may be asynchronous where the GPU reads the host's page tables)
    ZO_CUDA(cudaStreamSynchronize(c->stream), "stream synchronize");
    *out = c.release();
    return ZO_OK;
  } catch (const std::bad_alloc&) {
    return refuse(ZO_ERR_NOMEM, "zo_adamw_create: out of host memory");
  }
}

zo_status zo_adamw_destroy(zo_adamw_ctx* c) {
  if (!c) return ZO_OK;
  DeviceGuard guard(c->device);
  const cudaError_t e = cudaStreamSynchronize(c->stream);
  delete c;
  if (e != cudaSuccess) return cuda_fail(e, "zo_adamw_destroy");
  return ZO_OK;
}

zo_status zo_adamw_step(zo_adamw_ctx* c, int64_t t, int64_t* count, double lr, double beta1,
                        double beta2, double eps, double weight_decay) {
  if (!c) return ZO_ERR_INVALID_ARG;
  if ((count == nullptr) != (t >= 1) || t < 0)
    return refuse(ZO_ERR_INVALID_ARG, "zo_adamw_step: need t >= 1, or t = 0 and a count");
  if (reinterpret_cast<uintptr_t>(count) % 8 != 0)
    return refuse(ZO_ERR_ALIGN, "zo_adamw_step: the count is not aligned to its type");
  if (!std::isfinite(lr) || !std::isfinite(weight_decay) || !(eps >= 0.0) || !std::isfinite(eps) ||
      !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
    return refuse(ZO_ERR_INVALID_ARG,
                  "zo_adamw_step: need finite scalars, eps >= 0 and betas in [0, 1)");
  if (c->plan.chunks == 0 && !count) return ZO_OK;
  DeviceGuard guard(c->device);
  Step st{};
  st.b1 = (float)beta1;
  st.one_b1 = (float)(1.0 - beta1);
  st.b2 = (float)beta2;
  st.one_b2 = (float)(1.0 - beta2);
  st.keep = (float)(1.0 - lr * weight_decay);
  st.eps = (float)eps;
  st.none = -0.0f;
  for (uint32_t r = 0; r < 10; ++r) {
    st.key[2 * r] = (uint32_t)c->seed + r * 0x9E3779B9u;
    st.key[2 * r + 1] = (uint32_t)(c->seed >> 32) + r * 0xBB67AE85u;
  }
  auto* counted = reinterpret_cast<Now*>(c->ws);
  Now now{};
  if (count) {
    ZO_CUDA(zo::launch_dependent(adamw_count_kernel, 1u, 1, 0, c->stream, 1, true, count, lr,
                                 beta1, beta2, counted),
            "AdamW count kernel");
    ++c->launches;
  } else {
    now = now_of(t, lr, beta1, beta2);
  }
  if (c->plan.chunks == 0) return ZO_OK;
  const auto* ts = reinterpret_cast<const Tensor*>(c->ws + c->plan.tensors_at);
  const auto* chunks = reinterpret_cast<const int2*>(c->ws + c->plan.chunks_at);
  // The fast roots of subnormal v are off by up to 2^-63, which the bias correction multiplies by
  // 1 / sqrt(1 - b2) at most: below 2^-25 of eps, else the exact ones (131M bf16 elements: fp32 states
  // 406 us and 412 with exact roots, 8 bits 244 and 272).
  const bool exact = eps < 0x1p-38 / std::sqrt(1.0 - beta2);
  const auto kernel = c->bits == 8 ? (exact ? adamw_kernel<true, true> : adamw_kernel<true, false>)
                                   : (exact ? adamw_kernel<false, true> : adamw_kernel<false, false>);
  ZO_CUDA(zo::launch_dependent(kernel, (unsigned)c->plan.chunks, kThreads,
                               c->bits == 8 ? kRingBytes : 0, c->stream, 1, true, ts, chunks,
                               c->plan.units, st, now, count ? counted : nullptr),
          "AdamW kernel");
  ++c->launches;
  return ZO_OK;
}

int64_t zo_adamw_launches(const zo_adamw_ctx* c) { return c ? c->launches : 0; }

}  // extern "C"
