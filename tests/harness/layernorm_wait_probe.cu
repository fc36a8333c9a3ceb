// The layer norm's entry points, built from their sources with waits that can be told to run out:
// probe_lose(mode) chooses which threads' waits for a row report that nothing came, while the
// copies come as ever.  The kernels' last waits, for copies in flight (without an abort flag), are
// the real ones.  Run by tests/test_gpu_layernorm_waits.py.
//   0 none; 1 every thread's; 2 those of threads 3, 8, 13, ...; 3 thread 0's; 4 thread 0's from the
//   ring's second round on; 5 the odd threads' in the ring's odd rounds
#include <cstdio>

#include "zo_sm100.cuh"

namespace zo {
namespace sm100 {
__device__ int lose_mode;
__device__ __forceinline__ bool loses(uint32_t parity) {
  const int t = threadIdx.x, mode = lose_mode;
  return mode == 1 || (mode == 2 && t % 5 == 3) || (mode == 3 && t == 0) ||
         (mode == 4 && t == 0 && parity == 1) || (mode == 5 && t % 2 == 1 && parity == 1);
}
__device__ __forceinline__ bool losing_try(uint64_t* bar, uint32_t parity) {
  return !loses(parity) && mbar_try_wait(bar, parity);
}
__device__ __forceinline__ bool losing_wait(uint64_t* bar, uint32_t parity, const volatile int* abort,
                                            long long limit) {
  return !(abort && loses(parity)) && mbar_wait_bounded(bar, parity, abort, limit);
}
}  // namespace sm100
void set_last_error(const char* msg) { std::fprintf(stderr, "%s\n", msg); }
}  // namespace zo

#define mbar_try_wait losing_try
#define mbar_wait_bounded losing_wait
#include "zo_firstorder.cu"
#include "zo_layernorm.cu"
#include "zo_layernorm_backward.cu"

extern "C" __attribute__((visibility("default"))) int probe_lose(int mode) {
  return (int)cudaMemcpyToSymbol(zo::sm100::lose_mode, &mode, sizeof(mode));
}
