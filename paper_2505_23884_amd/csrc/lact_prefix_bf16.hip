// Attention over pages with shared prefixes: the kernels over a bf16 cache.
#include "lact_prefix.h"

namespace lact {
hipError_t launch_prefix_bf16(const PrefixArgs& a, hipStream_t s) { return run<__bf16, __bf16>(a, s); }
}  // namespace lact
