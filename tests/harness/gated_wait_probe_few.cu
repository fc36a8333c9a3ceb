// The kernel for few tokens with waits that can be told to run out (gated_wait_probe.cuh).
#include "gated_wait_probe.cuh"

#include "zo_gated_few.cu"

PROBE_SETTER(probe_lose_few)

namespace zo {
void set_last_error(const char* msg) { std::fprintf(stderr, "%s\n", msg); }
}  // namespace zo
