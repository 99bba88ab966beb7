// Attention over pages with shared prefixes: the plan of a call, and the
// kernels over an fp32 cache (a file of its own for each kind, since they take
// long to compile).
#include <algorithm>

#include "lact_prefix.h"

namespace lact {

// The time that `wgs` workgroups of `us` each take, two a CU where there are as
// many: a pair takes 1.43 times one alone (12 chunks of 160 tokens behind 8192 keys,
// the prefix in 1, 2, 3, 4 and 6 parts: 256, 180, 199, 162 and 173 us; 234, 167, 190, 142 and 151
// by this with 0.0286 us a key, and 5 a part for the sums; 32 sequences of 5 tokens, heads of 64
// in 8 bits, 2 to 8 parts: 52, 46, 43, 54, 52, 51 us). Where registers leave one a CU (an
// fp32 cache, heads over 128) the rounds are twice as many as this has them.
double span(int64_t wgs, double us) {
  const int64_t full = wgs / 512, rest = wgs % 512;
  return (full * 1.43 + (rest > 256 ? 1.43 : rest ? 1.0 : 0.0)) * us;
}

// The parts of `keys` keys for `jobs` workgroups a part, from 1 to `most`: what
// a workgroup does before its first key takes as long as some 6 us of them, and
// each part's sums of `rows` rows are written and read.
int best_parts(int64_t jobs, int64_t keys, double us_per_key, int64_t rows, int d, int most, bool joined) {
  const double sums = (double)rows * (d + 2) * 8 / 4.5e6;   // us
  int best = 1;
  double least = 0;
  for (int s = 1; s <= most; ++s) {
    const double t = span(jobs * s, 6.0 + us_per_key * (double)keys / s) + (s > 1 || joined ? 4.0 + (sums + 0.1) * s : 0.0);
    if (s == 1 || t < least) {
      least = t;
      best = s;
    }
  }
  return best;
}

void prefix_plan(PrefixArgs& a, bool bf16, bool codes) {
  const bool fp32 = !bf16 && !codes, pairs = codes && a.d <= 64 && a.Hkv % 2 == 0;
  const int rows16 = fp32 ? kRows32 : pairs ? kPairs16 : kRows16;
  const int64_t rows = (int64_t)a.T * a.G;
  // (fp32 queries over e4m3 numbers: 32 rows at most, as run() has it)
  const int many = codes && !bf16 ? kRows32 : kRows128;
  a.shape = rows > 32 * (int64_t)a.B || (fp32 && a.d > 128) ? many : rows > 16 * (int64_t)a.B ? kRows32 : rows16;
  // workgroups a part: as many as there would be if the tokens were spread evenly
  auto jobs = [&](int shape, int n) {
    const int R = shape_rows(shape);
    return (rows / n + (rows % n != 0) + R - 1) / R * n * (shape == kPairs16 ? a.Hkv / 2 : a.Hkv);
  };
  auto keys = [&](int64_t pages) { return std::min<int64_t>(pages * a.page, (int64_t)a.win + a.sinks + rows / a.G / a.B); };
  auto rate = [&](int shape) { return (shape == kRows128 ? 0.029 : 0.018) * (a.d > 128 ? 2 : 1) * (fp32 ? 3 : 1); };
  // (parts that leave each role half of the 2^24 workgroups that one launch holds, or one part)
  auto most = [&](int64_t k, int64_t limit, int shape, int n) {
    return (int)std::max<int64_t>(1, std::min({k / (4 * kKT), limit, (1 << 23) / row_jobs(a, shape, n, 1)}));
  };
  a.psplits = a.pjobs = 0;
  const int64_t own = keys(a.max_pages);
  // (beside a prefix they have half the room)
  a.splits = best_parts(jobs(a.shape, a.B) * (a.P ? 2 : 1), own, rate(a.shape), (int64_t)a.T * a.H, a.d,
                        most(own, 32, a.shape, a.B), a.P > 0);
  if (!a.P) return;
  // (32 rows of prefixes go with 16 of sequences, or 32 of an fp32 cache)
  a.pshape = rows > 32 * (int64_t)a.P || a.shape == kRows128 || (a.shape == kRows32 && !fp32) ? many : kRows32;
  const int64_t shared = keys(a.p_pages);
  a.psplits = best_parts(jobs(a.pshape, a.P), shared, rate(a.pshape), (int64_t)a.T * a.H, a.d,
                         most(shared, 64, a.pshape, a.P), true);
  a.pjobs = (int)row_jobs(a, a.pshape, a.P, a.psplits);
}

int64_t prefix_jobs(const PrefixArgs& a) { return a.pjobs + row_jobs(a, a.shape, a.B, a.splits); }

hipError_t launch_prefix(const PrefixArgs& a, bool bf16, hipStream_t s) {
  if (a.codes) return bf16 ? launch_prefix_e4m3(a, s) : launch_prefix_e4m3_fp32(a, s);
  return bf16 ? launch_prefix_bf16(a, s) : run<float, float>(a, s);
}

}  // namespace lact
