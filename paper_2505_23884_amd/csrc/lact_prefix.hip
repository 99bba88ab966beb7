// Attention over pages with shared prefixes: the plan of a call, and the
// kernels over an fp32 cache (a file of its own for each kind, since they take
// long to compile).
#include <algorithm>

#include "lact_prefix.h"

namespace lact {

void prefix_plan(PrefixArgs& a, bool bf16, bool codes) {
  const bool fp32 = !bf16 && !codes, pairs = codes && a.d <= 64 && a.Hkv % 2 == 0;
  const int rows16 = fp32 ? kRows32 : pairs ? kPairs16 : kRows16, rows32 = pairs ? kPairs32 : kRows32;
  const int64_t rows = (int64_t)a.T * a.G;
  a.shape = rows > 32 * (int64_t)a.B || (fp32 && a.d > 128) ? kRows128 : rows > 16 * (int64_t)a.B ? rows32 : rows16;
  const int64_t keys = (int64_t)a.max_pages * a.page, jobs = row_jobs(a, a.shape, a.B);
  const int64_t most = std::max<int64_t>(1, (keys + kKT - 1) / kKT / (2 * kWaves));
  a.psplits = a.pjobs = 0;
  if (a.P) {
    // (32 rows of prefixes go with 16 of sequences, or 32 of an fp32 cache)
    a.pshape = rows > 32 * (int64_t)a.P || a.shape == kRows128 || (a.shape == rows32 && !fp32) ? kRows128 : rows32;
    const int64_t pk = (int64_t)a.p_pages * a.page, pjobs = row_jobs(a, a.pshape, a.P);
    const int64_t pmost = std::max<int64_t>(1, pk / kKT / (2 * kWaves));
    // both roles' keys a workgroup about alike
    const double work = (double)pjobs * pk + (double)jobs * keys, each = work / 512;
    a.psplits = (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)(pk / std::max(each, 1.0) + 0.5), pmost, 64}));
    a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)(keys / std::max(each, 1.0) + 0.5), most, 32}));
    a.pjobs = (int)(pjobs * a.psplits);
    return;
  }
  if (a.shape != kRows128) {
    a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({(1024 + jobs - 1) / jobs, most, 32}));
    return;
  }
  double best = 0;
  for (int s = 1; s <= std::min<int64_t>(most, 16); ++s) {
    const double t = (double)((jobs * s + 511) / 512) / s * (s > 1 ? 1.08 + 0.02 * s : 1.0);
    if (s == 1 || t < best) {
      best = t;
      a.splits = s;
    }
  }
}

hipError_t launch_prefix(const PrefixArgs& a, bool bf16, hipStream_t s) {
  if (a.codes) return bf16 ? launch_prefix_e4m3(a, s) : launch_prefix_e4m3_fp32(a, s);
  return bf16 ? launch_prefix_bf16(a, s) : run<float, float>(a, s);
}

}  // namespace lact
