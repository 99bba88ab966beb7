// Attention over pages with shared prefixes: the kernels over a cache of e4m3 numbers, with fp32 queries.
#include "lact_prefix.h"

namespace lact {
hipError_t launch_prefix_e4m3_fp32(const PrefixArgs& a, hipStream_t s) { return run<float, Code>(a, s); }
}  // namespace lact
