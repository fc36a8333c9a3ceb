// The gated linear block's kernels, built from their sources with waits that can be told to run
// out: probe_lose_*(mode) chooses which waits of the kernels' roles report that nothing came, while
// copies and products go on as ever.  Their last waits, for what is in flight (without an abort flag),
// are the real ones, with a shorter limit.  Run by tests/test_gpu_gated_waits.py.
//   0 none; 1 every role's; 2 the loading warps' from the ring's second round on; 3 the product warps' of
//   every third CTA in the ring's odd rounds; 4 some lanes of the storing warps' in every fourth pair;
//   5 the storing warps' in the accumulators' odd rounds; 6 the loading warps' of the pairs' second CTAs
//   from the second round on; 7 one storing warp's in every sixteenth CTA; 8 the storing warps' without an
//   abort flag (the kernel for few tokens)
#pragma once

#include <cstdio>

#include "zo_sm100.cuh"

namespace zo {
namespace sm100 {
static __device__ int lose_mode;
__device__ __forceinline__ bool loses(uint32_t parity, bool role) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, mode = lose_mode;
  const unsigned b = blockIdx.x;
  if (!role) return mode == 8 && warp >= 2;
  switch (mode) {
    case 1: return true;
    case 2: return warp == 0 && parity == 0;
    case 3: return warp == 1 && b % 3 == 0 && parity == 1;
    case 4: return warp >= 2 && lane % 5 == 3 && b % 8 < 2;
    case 5: return warp >= 2 && parity == 1;
    case 6: return warp == 0 && b % 2 == 1 && parity == 0;
    case 7: return warp == 5 && b % 16 == 3;
    default: return false;
  }
}
__device__ __forceinline__ bool losing_wait(uint64_t* bar, uint32_t parity, const volatile int* abort,
                                            long long limit) {
  constexpr long long kShort = 100000000LL;      // ~50 ms
  return !loses(parity, abort != nullptr) &&
         mbar_wait_bounded(bar, parity, abort, abort || limit < kShort ? limit : kShort);
}
}  // namespace sm100
}  // namespace zo

#define mbar_wait_bounded losing_wait

#define PROBE_SETTER(name)                                                          \
  extern "C" __attribute__((visibility("default"))) int name(int mode) {            \
    return (int)cudaMemcpyToSymbol(zo::sm100::lose_mode, &mode, sizeof(mode));      \
  }
