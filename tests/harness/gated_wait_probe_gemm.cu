// The products on SM pairs with waits that can be told to run out (gated_wait_probe.cuh).
#include "gated_wait_probe.cuh"

#include "zo_gated_gemm.cu"

PROBE_SETTER(probe_lose_gemm)

// columns of a tile's half, or minus the tokens of a turned tile
extern "C" __attribute__((visibility("default"))) int probe_plan(long long T, long long D, long long F) {
  const zo::GatedPlan p = zo::gated_plan(T, D, F, zo::gated_max_pairs());
  return p.side ? p.side : -p.tokens;
}
extern "C" __attribute__((visibility("default"))) int probe_parts(long long T, long long D, long long F) {
  return zo::gated_parts(T, D, F);
}
