// Attention over pages with shared prefixes: the kernels over a cache of e4m3 numbers.
#include "lact_prefix.h"

namespace lact {
hipError_t launch_prefix_e4m3(const PrefixArgs& a, hipStream_t s) { return run<__bf16, Code>(a, s); }
}  // namespace lact
