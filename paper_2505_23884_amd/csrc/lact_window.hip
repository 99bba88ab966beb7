// Softmax attention with a sliding window and first tokens that stay visible
// (sinks), and its reverse.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(c q_i . k_j - lse_i) over the visible j
//   dv_j = sum_i p_ij do_i,  ds_ij = p_ij (do_i . v_j - delta_i),
//   delta_i = do_i . o_i,  dq_i = c sum_j ds_ij k_j,  dk_j = c sum_i ds_ij q_i
//
// Bound by the matrix cores: 4 d flops a visible pair forward, 10 d in the
// reverse; memory traffic is q, k, v and o once where the tiles of one head
// share an L2. Only tiles of keys that some query of the workgroup sees are
// visited, and only those at the edges of the window, at the diagonal and at
// the sequence's end are masked element by element.
#include <algorithm>
#include <type_traits>

#include "lact_attn.h"
#include "lact_internal.h"

namespace lact {
namespace {

using namespace attn;

// Consecutive work on one XCD: workgroups go round the 8 XCDs in turn, so
// workgroup b takes item (b % 8) * (n / 8) + ..., and the tiles of one head
// meet their keys in one L2.
__device__ __forceinline__ int xcd_order(int b, int n) {
  const int x = b & 7, per = n >> 3, extra = n & 7;
  return x * per + (x < extra ? x : extra) + (b >> 3);
}

// Item p of a list of n in which each eighth, and so each XCD's share of a
// head, holds items from all along it: every eighth one, then the next ones.
// Work that shrinks towards the end of a sequence spreads over the XCDs, and
// each share ends with its shortest items.
__device__ __forceinline__ int spread(int p, int n) {
  const int full = n >> 3, extra = n & 7;   // residues below `extra` have full + 1 items
  if (p < extra * (full + 1)) return p / (full + 1) + 8 * (p % (full + 1));
  p -= extra * (full + 1);
  return extra + p / max(full, 1) + 8 * (p % max(full, 1));
}

template <typename T>
__device__ __forceinline__ T* row_of(const AttnView& v, int b, int h, int64_t t) {
  return reinterpret_cast<T*>(v.p) + b * v.sb + h * v.sh + t * v.st;
}

__device__ __forceinline__ int length_of(const WindowArgs& a, int b) {
  return a.len ? min(max(a.len[b], 0), a.n_kv) : a.n_kv;
}

// Rows of few keys (16-bit I/O): those that see at most this many. What the
// reverse does for their sake (k_window_dq) goes by each row's own count, so it
// is the same in dq and dk, whichever kernels run and whatever rows stand beside.
constexpr int kFewKeys = 128;

// The number of keys that position p of a sequence of len sees.
__device__ __forceinline__ int keys_of(const WindowArgs& a, int len, int p) {
  const int hi = min(p + a.look, len - 1), lo = max(0, p - a.win + 1);
  return max(0, hi - lo + 1) + max(0, min(min(a.sinks, hi + 1), lo));
}
// Which of 32 queries see few keys, for the kernel that holds queries by rows.
struct FewKeys {
  int below, above;   // queries i .. i + 31 of below <= i <= above all see more
  __device__ __forceinline__ FewKeys(const WindowArgs& a, int len) {
    // they share the keys from the last one's window to the first one's end
    const bool never = a.look >= kFewKeys + 32 - a.win && len > kFewKeys;   // (look + win may be 2^31)
    below = never ? kFewKeys - a.look - a.q_start : (1 << 30);
    above = len + a.win - (kFewKeys + 33) - a.q_start;
  }
  __device__ __forceinline__ bool any(int i) const { return (i < below) | (i > above); }
  // What the rounding to bf16 leaves of the rows of an accumulator (below_bf16)
  // whose queries, from i on, see few keys.
  static __device__ __forceinline__ f32x16 below_bf16_of(const WindowArgs& a, int len, int i, const f32x16& s) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));   // nothing of this is worked out ahead of a loop, for it hardly ever runs
    const uint32_t few = (uint32_t)__ballot(keys_of(a, len, a.q_start + i + (lane & 31)) <= kFewKeys) >> (lane >> 5) * 4;
    f32x16 r = below_bf16(s);
#pragma unroll
    for (int e = 0; e < 16; ++e) r[e] = few >> (8 * (e >> 2) + (e & 3)) & 1 ? r[e] : 0.0f;
    return r;
  }
};

// Keys a tile: those of a lone wave (of NW = 1) leave room for three more waves' at DP = 128.
template <typename T, int DP, int NW> constexpr int key_tile() {
  return sizeof(T) == 2 && DP <= (NW > 1 ? 128 : 64) ? 64 : 32;
}

// ------------------------------------------------------------------ forward
// A workgroup of NW waves owns 32 NW queries of one head, a wave 32 of them;
// keys and values pass through LDS in two stages. Or (NW = 1) KS waves share
// 32 queries, each with every KS-th tile in LDS of its own, and join their sums.
// Scores are held transposed (lact_attn.h), so the softmax needs one exchange
// between lanes a tile.
//
// 128 queries share each tile that comes from L2, and 64 keys a step leave two
// workgroups a CU (D = 128; four at 64): one's vector work and LDS reads run
// beside the other's products. bf16, heads of 128: [1, 16, 16384], window 2048:
// 337 to 424 us by the card's clock, 0.76 to 0.61 PF; [2, 40, 3120], all keys:
// 468 to 592, 0.85 to 0.67 (a library product of 8192 x 8192 x 8192: 1.15).
// Heads of 64, [2, 32 / 8, 8192], causal: 0.76. Matrix instructions take 31 % of
// the cycles (1.9 GHz), vector ones 37 % and a quarter more for exponentials.
// Weaving the halves of a tile in one wave (one's scores beside the other's
// weights) was slower by 4 %, a higher priority for matrix work changed nothing.
template <typename T, int DP, int NW, int KS, int OCC>
__global__ __launch_bounds__(64 * NW * KS, OCC) void k_window_fwd(const WindowArgs a) {
  constexpr int KT = key_tile<T, DP, NW>(), QB = 32 * NW, NT = 64 * NW;
  using L = Tile<T, DP>;
  constexpr int BYTES = KT * L::PITCH;
  __shared__ __attribute__((aligned(1024))) uint8_t smem_[KS * 4 * BYTES];
  __shared__ uint32_t mask_[2 * KS];
  __shared__ int found_[KS];
  const int wave_ = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wave = KS > 1 ? 0 : wave_, ks_ = KS > 1 ? wave_ : 0;   // of the queries; of the keys
  uint8_t* const smem = smem_ + ks_ * 4 * BYTES;
  uint32_t* const mask = mask_ + 2 * ks_;
  int* const found = found_ + ks_;
  const int ntile = (a.n_q + QB - 1) / QB;
  const int w = xcd_order(blockIdx.x, gridDim.x);
  const int bh = w / ntile, qt = ntile - 1 - w % ntile;   // the longest rows of a causal head first
  const int b = bh / a.H, h = bh % a.H, hk = h / a.G;
  const int len = length_of(a, b);
  const int r0 = qt * QB, i = r0 + 32 * wave + (lane & 31);
  const int last = min(a.n_q, len - a.q_start) - 1;       // the last query of the sequence
  const int p = a.q_start + i;
  const bool live = i <= last;
  const KeyTiles kt(a, len, a.q_start + r0, a.q_start + min(r0 + QB - 1, last), KT);
  const int wa = a.q_start + r0 + 32 * wave, wb = a.q_start + min(r0 + 32 * wave + 31, last);
  const int jhi = live ? min(p + a.look, len - 1) : -1;

  u32x4 q[L::KS];
  load_row<T, DP>(q, row_of<T>(a.q, b, h, min(i, a.n_q - 1)), live, a.d);
  Softmax<DP / 32> st;
  st.init();
  const float c = a.scale * kLog2e;
  const int n = kt.count();
  const int ldk = (int)(a.k.st * sizeof(T)), ldv = (int)(a.v.st * sizeof(T));
  using Cp = Copy<T, DP, KT, NT>;
  auto copy = [&](int x) __attribute__((always_inline)) {
    const int k0 = kt.tile(x) * KT;
    uint8_t* to = smem + (x / KS & 1) * 2 * BYTES;
    Cp::rows(to, row_of<T>(a.k, b, hk, k0), ldk, len - k0, a.d);
    Cp::rows(to + BYTES, row_of<T>(a.v, b, hk, k0), ldv, len - k0, a.d);
  };
  const int pa = a.q_start + r0, pb = a.q_start + min(r0 + QB - 1, last);
  if (Cp::thread() == 0) *found = -1;
  if (ks_ < n) copy(ks_);
  Cp::sync();
  for (int x = ks_; x < n; x += KS) {
    uint8_t* ks = smem + (x / KS & 1) * 2 * BYTES;
    const int k0 = kt.tile(x) * KT;
    uint64_t bad = 0;   // keys whose values were scrubbed
    if (sees(a, len, pa, pb, k0, KT) != 2 && __builtin_expect(Cp::holds_nonfinite(ks + BYTES, x, found), 0))
      bad = Cp::scrub(ks + BYTES, mask);
    if (x + KS < n) copy(x + KS);
    const Sight sight(a, p, jhi, k0);
    auto step = [&](auto rb) __attribute__((always_inline)) {
      constexpr int RB = decltype(rb)::value;
      const int what = sees(a, len, wa, wb, k0 + RB, 32);
      if (what) softmax_step<T, DP, RB>(st, q, ks, ks + BYTES, c, what == 1, [&](int r) { return sight.see(r); });
    };
    step(std::integral_constant<int, 0>{});
    if constexpr (KT == 64) step(std::integral_constant<int, 32>{});
#pragma unroll 1
    for (; __builtin_expect(bad != 0, 0); bad &= bad - 1) {
      const int j = __builtin_ctzll(bad);
      add_nonfinite<T, DP / 32>(st.o, row_of<T>(a.v, b, hk, k0 + j), sight.see(j - 4 * (lane >> 5)), 0, a.d);
    }
    Cp::sync();
  }
  if constexpr (KS > 1) {   // the waves' sums to the first
    float* to = reinterpret_cast<float*>(smem_) + lane;
    constexpr int PER = DP / 2 + 2;
    static_assert(PER * 64 * 4 <= 4 * BYTES, "sums of a wave");
    __syncthreads();
    if (ks_) st.put(to + ks_ * PER * 64);
    __syncthreads();
    if (ks_) return;
    for (int w = 1; w < KS; ++w) st.join(to + w * PER * 64);
  }
  const float l = half_sum(st.l);
  const bool none = !live || l == 0.0f;   // a row that sees nothing: 0, lse -inf
  if (i < a.n_q) {
    if (a.lse && lane < 32)
      a.lse[(int64_t)bh * a.n_q + i] = none ? neg_inf() : (st.m + __builtin_amdgcn_logf(l)) * kLn2;
  }
  store_row<T, DP / 32>(row_of<T>(a.o, b, h, min(i, a.n_q - 1)), st.o, 1.0f / l, 0, a.d, i < a.n_q, none);
}

// ------------------------------------------------------------------ reverse
// The sums of W waves to the first of them (true), in order, through LDS
// (W - 1 times 4 KiB of floats a block).
template <int W, int NB>
__device__ __forceinline__ bool join_waves(f32x16 (&acc)[NB], float* lds, int w) {
  float* at = lds + (threadIdx.x & 63);
  __syncthreads();
  if (w)
#pragma unroll
    for (int x = 0; x < NB; ++x)
#pragma unroll
      for (int e = 0; e < 16; ++e) at[((w - 1) * NB * 16 + x * 16 + e) * 64] = acc[x][e];
  __syncthreads();
  if (w) return false;
  for (int y = 0; y < W - 1; ++y)
#pragma unroll
    for (int x = 0; x < NB; ++x)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[x][e] += at[(y * NB * 16 + x * 16 + e) * 64];
  return true;
}

// The sum of x y over the lane's half of a row (load_row).
template <typename T, int N>
__device__ __forceinline__ float dot_half(const u32x4 (&x)[N], const u32x4 (&y)[N]) {
  float sum = 0.0f;
#pragma unroll
  for (int c = 0; c < N; ++c)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 2)
        sum += __uint_as_float(x[c][k] << 16) * __uint_as_float(y[c][k] << 16) +
               __uint_as_float(x[c][k] & 0xffff0000u) * __uint_as_float(y[c][k] & 0xffff0000u);
      else
        sum += __uint_as_float(x[c][k]) * __uint_as_float(y[c][k]);
    }
  return sum;
}

// dq: queries stay in registers with their cotangents, keys and values pass
// through LDS as in the forward (NW, KS as there). Leaves -lse / scale and -delta of its queries
// for dk and dv, whose accumulators start from them. Three products a pair with
// one exponential: [1, 16 / 4, 8192, 128] bf16, window 2048, 4 sinks: 214 to 231
// us by the card's clock, 0.84 to 0.78 PF. Registers: what spills at heads of 128
// (44) stays out of the products; fp32 heads of 256 spill 173, read back among
// theirs too.
template <typename T, int DP, int NW, int KS, int OCC>
__global__ __launch_bounds__(64 * NW * KS, OCC) void k_window_dq(const WindowBwdArgs g) {
  const WindowArgs& a = g.f;
  constexpr int KT = key_tile<T, DP, NW>(), QB = 32 * NW, NT = 64 * NW;
  using L = Tile<T, DP>;
  constexpr int BYTES = KT * L::PITCH;
  __shared__ __attribute__((aligned(1024))) uint8_t smem_[KS * 4 * BYTES];
  __shared__ uint32_t mask_[2 * KS];
  __shared__ int found_[KS];
  const int wave_ = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = KS > 1 ? 0 : wave_, ks_ = KS > 1 ? wave_ : 0;   // of the queries; of the keys
  uint8_t* const smem = smem_ + ks_ * 4 * BYTES;
  uint32_t* const mask = mask_ + 2 * ks_;
  int* const found = found_ + ks_;
  const int ntile = (a.n_q + QB - 1) / QB;
  const int w = xcd_order(blockIdx.x, gridDim.x);
  const int bh = w / ntile, qt = ntile - 1 - w % ntile;
  const int b = bh / a.H, h = bh % a.H, hk = h / a.G;
  const int len = length_of(a, b);
  const int r0 = qt * QB, i = r0 + 32 * wave + (lane & 31), ic = min(i, a.n_q - 1);
  const int last = min(a.n_q, len - a.q_start) - 1;
  const int p = a.q_start + i;
  const bool live = i <= last;
  const KeyTiles kt(a, len, a.q_start + r0, a.q_start + min(r0 + QB - 1, last), KT);
  const int wa = a.q_start + r0 + 32 * wave, wb = a.q_start + min(r0 + 32 * wave + 31, last);
  const int jhi = live ? min(p + a.look, len - 1) : -1;

  u32x4 q[L::KS], go[L::KS];
  load_row<T, DP>(q, row_of<T>(a.q, b, h, ic), live, a.d);
  load_row<T, DP>(go, row_of<T>(g.dout, b, h, ic), live, a.d);
  const int64_t at = (int64_t)bh * a.n_q + ic;
  float nlse = live ? a.lse[at] : neg_inf(), ndelta;
  nlse = nlse == neg_inf() ? neg_inf() : -nlse / a.scale;   // an empty row's too: weights exp2(-inf) = 0
  {
    u32x4 o[L::KS];
    load_row<T, DP>(o, row_of<T>(a.o, b, h, ic), live, a.d);
    ndelta = -half_sum(dot_half<T>(o, go));
  }
  const float nlse2 = nlse * a.scale * kLog2e;
  const float c = a.scale * kLog2e;
  const int n = kt.count();
  const int ldk = (int)(a.k.st * sizeof(T)), ldv = (int)(a.v.st * sizeof(T));
  using Cp = Copy<T, DP, KT, NT>;
  auto copy = [&](int x) __attribute__((always_inline)) {
    const int k0 = kt.tile(x) * KT;
    uint8_t* to = smem + (x / KS & 1) * 2 * BYTES;
    Cp::rows(to, row_of<T>(a.k, b, hk, k0), ldk, len - k0, a.d);
    Cp::rows(to + BYTES, row_of<T>(a.v, b, hk, k0), ldv, len - k0, a.d);
  };
  const int pa = a.q_start + r0, pb = a.q_start + min(r0 + QB - 1, last);
  // The cotangents of the scores of rows RB .. of the tile; with `Sum` the weights are added to `whole`.
  float whole = 0.0f;
  auto scores = [&](const uint8_t* ks, int k0, auto rb, bool masked, uint64_t bad, f32x16& s, auto with_sum)
      __attribute__((always_inline)) {
    constexpr int RB = decltype(rb)::value;
    constexpr bool Sum = decltype(with_sum)::value;
    f32x16 dp, w;
    mma_dot<T, DP, RB>(s, ks, q);
    mma_dot<T, DP, RB>(dp, ks + BYTES, go);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, nlse2));
      s[e] = w[e] * (dp[e] + ndelta);
    }
    if (masked) {
      if (__builtin_expect(bad != 0, 0))   // keys that held an infinity or NaN
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (bad >> (RB + 8 * (e >> 2) + 4 * half + (e & 3)) & 1) s[e] = __builtin_nanf("");
      const Sight sight(a, p, jhi, k0);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const bool see = sight.see(RB + 8 * (e >> 2) + (e & 3));
        s[e] = see ? s[e] : 0.0f;
        if (Sum) w[e] = see ? w[e] : 0.0f;
      }
    }
    if (Sum)
#pragma unroll
      for (int e = 0; e < 16; ++e) whole += w[e];
  };
  // use(tile, k0, RB, masked, bad) for each 32 keys that the wave sees something of
  auto over_tiles = [&](auto use) __attribute__((always_inline)) {
    if (Cp::thread() == 0) *found = -1;
    if (ks_ < n) copy(ks_);
    Cp::sync();
    for (int x = ks_; x < n; x += KS) {
      uint8_t* ks = smem + (x / KS & 1) * 2 * BYTES;
      const int k0 = kt.tile(x) * KT;
      uint64_t bad = 0;
      if (sees(a, len, pa, pb, k0, KT) != 2 && __builtin_expect(Cp::holds_nonfinite(ks, x, found), 0))
        bad = Cp::scrub(ks, mask);
      if (x + KS < n) copy(x + KS);
      auto part = [&](auto rb) __attribute__((always_inline)) {
        const int what = sees(a, len, wa, wb, k0 + rb, 32);
        if (what) use(ks, k0, rb, what == 1 || bad != 0, bad);
      };
      part(std::integral_constant<int, 0>{});
      if constexpr (KT == 64) part(std::integral_constant<int, 32>{});
      Cp::sync();
    }
  };
  // the lane's query, some of the wave's and some of the workgroup's
  const bool few = sizeof(T) == 2 && live && keys_of(a, len, p) <= kFewKeys, few_wave = __any(few);
  const bool few_block = sizeof(T) == 2 && (NW > 1 ? __syncthreads_or(few) : few_wave);
  if (few_block) {
    // delta from a rounded o is off by 2^-8 of its terms, which shows in rows
    // of few keys (their o is large): the cotangents of a row's scores sum to
    // zero, so a pass over its keys finds what is missing. Where lse is of more
    // keys than these (split over calls) the weights here sum to less than 1 and
    // the cotangents need not cancel: such rows keep delta as it is, also those
    // whose scores are so large that the weights' own error passes 2^-12.
    float rest = 0.0f;
    over_tiles([&](const uint8_t* ks, int k0, auto rb, bool masked, uint64_t bad) __attribute__((always_inline)) {
      f32x16 s;
      scores(ks, k0, rb, masked, bad, s, std::true_type{});
#pragma unroll
      for (int e = 0; e < 16; ++e) rest += s[e];
    });
    if constexpr (KS > 1) {
      float* all = reinterpret_cast<float*>(smem_) + lane;
      __syncthreads();
      all[2 * ks_ * 64] = rest;
      all[(2 * ks_ + 1) * 64] = whole;
      __syncthreads();
      rest = whole = 0.0f;
      for (int w = 0; w < KS; ++w) {
        rest += all[2 * w * 64];
        whole += all[(2 * w + 1) * 64];
      }
      __syncthreads();
    }
    rest = half_sum(rest);
    const bool all_keys = fabsf(half_sum(whole) - 1.0f) < 0x1p-12f;
    if (few && all_keys && __builtin_isfinite(rest)) ndelta -= rest;   // (an infinite key that weighs nothing leaves the row its delta)
  }
  if (i < a.n_q && lane < 32 && ks_ == 0) {
    g.nlse[at] = nlse;
    g.ndelta[at] = ndelta;
  }
  f32x16 dq[DP / 32];
#pragma unroll
  for (int x = 0; x < DP / 32; ++x) dq[x] = f32x16{};
  // The rounding of the cotangents to 16 bits makes the error of dq and dk 1.4
  // times that of a form which rounds its outputs only, of however many keys. A
  // second product, of what it leaves, makes it 1.0. Rows of few keys take it: in
  // long calls they are the first ones and cost nothing that shows; a window of
  // 128 costs 9 % of the training call ([1, 16 / 4, 8192, 128]: 164 to 179 us).
  auto products = [&](auto rest) __attribute__((always_inline)) {
    over_tiles([&](const uint8_t* ks, int k0, auto rb, bool masked, uint64_t bad) __attribute__((always_inline)) {
      constexpr int RB = decltype(rb)::value;
      f32x16 s;
      scores(ks, k0, rb, masked, bad, s, std::false_type{});
      mma_rows<T, DP, DP / 32, RB>(dq, RowsB<T>(s), ks, 0);
      if (decltype(rest)::value && few_wave) {
        s = below_bf16(s);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = few ? s[e] : 0.0f;
        mma_rows<T, DP, DP / 32, RB>(dq, RowsB<T>(s), ks, 0);
      }
    });
  };
  if (few_block) products(std::integral_constant<bool, sizeof(T) == 2>{});
  else products(std::false_type{});
  if constexpr (KS > 1) {
    static_assert(DP / 2 * 64 * 4 <= 4 * BYTES, "sums of a wave");
    if (!join_waves<KS, DP / 32>(dq, reinterpret_cast<float*>(smem_), ks_)) return;
  }
  store_row<T, DP / 32>(row_of<T>(g.dq, b, h, ic), dq, a.scale, 0, a.d, i < a.n_q, !live);
}

// The job of workgroup `id` of `n`: first the tiles without sinks of every
// (batch, key head), then the parts of the others, which are short and fill
// the gaps that the former leave.
struct DkvJob {
  int bk, tile, part, head_part, slot;   // slot < 0: the sums go to dk and dv
  int qa, qb;                            // queries [qa, qb)
  __device__ __forceinline__ DkvJob(const WindowArgs& a, const DkvPlan& pl, int id, int n) {
    const int plain = (pl.ntile - pl.st) * pl.np_a * pl.gs, sinks = pl.st * pl.np_s * pl.gs;
    const int n1 = n / (plain + sinks) * plain;
    const bool sink = id >= n1;
    const int per = sink ? sinks : plain, w = sink ? xcd_order(id - n1, n - n1) : xcd_order(id, n1);
    bk = w / per;
    int x = spread(w % per, per);
    head_part = x % pl.gs;
    x /= pl.gs;
    const int np = sink ? pl.np_s : pl.np_a;
    tile = x / np + (sink ? 0 : pl.st);
    part = x % np;
    const int before = sink || pl.np_s * pl.gs <= 1 ? 0 : sinks;
    slot = np * pl.gs > 1 ? before + (((sink ? tile : tile - pl.st) * np) + part) * pl.gs + head_part : -1;
  }
  __device__ __forceinline__ void queries(const WindowArgs& a, const DkvPlan& pl, int len) {
    const bool sink = tile < pl.st;
    const int np = sink ? pl.np_s : pl.np_a, ch = sink ? pl.ch_s : pl.ch_a;
    const int k0 = tile * pl.kb, k1 = min(k0 + pl.kb, len) - 1;   // keys k0 .. k1
    const int last = min(a.n_q, len - a.q_start);                  // queries of the sequence
    // j <= p + look and (p < j + win or j < sinks), p = q_start + i
    const int ia = max(0, k0 - a.look - a.q_start);
    int ib = k0 < a.sinks ? last : min(last, k1 + a.win - a.q_start);
    if (k0 > k1) ib = ia;
    qa = ia + part * ch;
    qb = part == np - 1 ? ib : min(ib, qa + ch);
  }
};

// dk and dv: 32 keys and values a wave stay in registers, queries and
// cotangents pass through LDS, over every head that shares the keys. DO
// columns of dk and dv a workgroup (DP, or less where both would not fit the
// registers: the scores are then computed again for each part). NW waves with
// 32 keys each share a step's queries, or (NW = 1) QS waves share 32 keys, each
// with every QS-th step's queries in LDS of its own, and add their sums. Two
// waves a SIMD where 256 registers hold one ([1, 16 / 4, 4096, 64] fp32, window
// 1024, training: 770 us, with one 791).
template <typename T, int DP, int DO, int QT, int NW, int QS>
__global__ __launch_bounds__(64 * NW * QS, (DP == 64 && NW > 1 ? 2 : 1)) void k_window_dkv(const WindowBwdArgs g) {
  const WindowArgs& a = g.f;
  constexpr int KB = 32 * NW, NT = 64 * NW, NB = DO / 32;
  using L = Tile<T, DP>;
  constexpr int BYTES = QT * L::PITCH, STAGE = 2 * BYTES + 1024;   // tiles start at multiples of their pitch
  static_assert(2 * QT * 4 <= 1024, "lse2 and delta of a step");
  __shared__ __attribute__((aligned(1024))) uint8_t smem_[QS * 2 * STAGE];
  __shared__ uint32_t mask_[2 * QS];
  __shared__ int found_[QS];
  const int wave_ = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = QS > 1 ? 0 : wave_, qs_ = QS > 1 ? wave_ : 0;   // of the keys; of the queries
  uint8_t* const smem = smem_ + qs_ * 2 * STAGE;
  uint32_t* const mask = mask_ + 2 * qs_;
  int* const found = found_ + qs_;
  constexpr int ND = DP / DO;
  const int dsel = blockIdx.x % ND;
  DkvJob job(a, g.plan, blockIdx.x / ND, gridDim.x / ND);
  const int bk = job.bk, b = bk / a.Hkv, hk = bk % a.Hkv;
  const int len = length_of(a, b);
  const FewKeys few(a, len);
  job.queries(a, g.plan, len);
  const int kw = job.tile * KB + 32 * wave, j = kw + (lane & 31), jc = min(j, a.n_kv - 1);
  const bool live = j < len;
  const int iend = min(a.n_q, len - a.q_start);   // queries past it are padding
  // the queries of the job that see key j
  const int ilo = max(j - a.look - a.q_start, 0);
  const int ihi = !live ? -1 : min(job.qb - 1, j < a.sinks ? iend - 1 : min(iend - 1, j + a.win - 1 - a.q_start));

  u32x4 kf[L::KS], vf[L::KS];
  load_row<T, DP>(kf, row_of<T>(a.k, b, hk, jc), live, a.d);
  load_row<T, DP>(vf, row_of<T>(a.v, b, hk, jc), live, a.d);
  f32x16 dk[NB], dv[NB];
#pragma unroll
  for (int x = 0; x < NB; ++x) dk[x] = dv[x] = f32x16{};
  const float c = a.scale * kLog2e;
  const int steps = job.qb > job.qa ? (job.qb - job.qa + QT - 1) / QT : 0;
  const int gh = a.G / g.plan.gs, n = steps * gh;
  const int ldq = (int)(a.q.st * sizeof(T)), ldo = (int)(g.dout.st * sizeof(T));
  using Cp = Copy<T, DP, QT, NT>;
  using Cp2 = Copy<T, DP, 2 * QT, NT>;   // queries and cotangents as one tile
  typedef __attribute__((address_space(3))) void lds_void;
  auto copy = [&](int x) __attribute__((always_inline)) {
    const int h = hk * a.G + job.head_part * gh + x / steps, i0 = job.qa + (x % steps) * QT;
    uint8_t* to = smem + (x / QS & 1) * STAGE;
    Cp::rows(to, row_of<T>(a.q, b, h, i0), ldq, job.qb - i0, a.d);
    Cp::rows(to + BYTES, row_of<T>(g.dout, b, h, i0), ldo, job.qb - i0, a.d);
    if (wave == 0) {   // nlse and ndelta of the queries; past the last one zeros (masked)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const float* from = (y ? g.ndelta : g.nlse) + ((int64_t)b * a.H + h) * a.n_q + i0;
        const __amdgpu_buffer_rsrc_t rsrc =
            __builtin_amdgcn_make_buffer_rsrc((void*)from, (short)0, min(QT, job.qb - i0) * 4, kBufFlags);
        if (lane < QT)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(to + 2 * BYTES + y * QT * 4), 4, lane * 4, 0, 0, 0);
      }
    }
  };
  const int kb0 = job.tile * KB, kb1 = kb0 + KB - 1;
  // queries i0 .. against the keys k0 .. k1: nothing (0), something (1) or all (2)
  auto seen = [&](int i0, int count, int k0, int k1) __attribute__((always_inline)) {
    const int pa = a.q_start + i0, pe = a.q_start + min(i0 + count, min(job.qb, iend)) - 1;
    if (pa > pe || k0 >= len || k0 > pe + a.look || (k0 >= a.sinks && k1 <= pa - a.win)) return 0;
    return pe - pa == count - 1 && k1 < len && k1 <= pa + a.look && (k0 > pe - a.win || k1 < a.sinks) ? 2 : 1;
  };
  auto step = [&](const uint8_t* qs, int i0, auto rb, bool masked, uint64_t badq, uint64_t bado)
      __attribute__((always_inline)) {
    constexpr int RB = decltype(rb)::value;
    const uint8_t* os = qs + BYTES;
    f32x16 s, dp;
    mma_dot<T, DP, RB>(s, qs, kf);
    mma_dot<T, DP, RB>(dp, os, vf);
    // nlse and ndelta of rows 8e + 4 half ..
    u32x4 rows[8];
    {
      const uint32_t at = lds_addr(qs + 2 * BYTES) + RB * 4 + 16 * half;
      const uint32_t ad[8] = {at, at + 32, at + 64, at + 96, at + 4 * QT, at + 4 * QT + 32, at + 4 * QT + 64, at + 4 * QT + 96};
      read_rows8<0>(rows, ad);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = __builtin_amdgcn_exp2f((s[e] + __uint_as_float(rows[e >> 2][e & 3])) * c);
      dp[e] = s[e] * (dp[e] + __uint_as_float(rows[4 + (e >> 2)][e & 3]));
    }
    if (masked) {
      if (__builtin_expect((badq | bado) != 0, 0))   // queries, or cotangents, that held an infinity or NaN
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int r = RB + 8 * (e >> 2) + 4 * half + (e & 3);
          if (badq >> r & 1) s[e] = __builtin_nanf("");
          if ((badq | bado) >> r & 1) dp[e] = __builtin_nanf("");
        }
      // the queries ilo .. ihi see the lane's key
      const int at = i0 + RB + 4 * half, lo = ihi < ilo ? (1 << 30) : ilo - at;
      const uint32_t span = (uint32_t)max(ihi - ilo, 0);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const bool see = (uint32_t)(8 * (e >> 2) + (e & 3) - lo) <= span;
        s[e] = see ? s[e] : 0.0f;
        dp[e] = see ? dp[e] : 0.0f;
      }
    }
    mma_rows<T, DP, NB, RB>(dv, RowsB<T>(s), os, dsel * NB);
    if constexpr (sizeof(T) == 2) {
      if (__builtin_expect(few.any(i0 + RB), 0))
        mma_rows<T, DP, NB, RB>(dk, RowsB<T>(FewKeys::below_bf16_of(a, len, i0 + RB, dp)), qs, dsel * NB);
    }
    mma_rows<T, DP, NB, RB>(dk, RowsB<T>(dp), qs, dsel * NB);
  };
  if (Cp::thread() == 0) *found = -1;
  if (qs_ < n) copy(qs_);
  Cp::sync();
  for (int x = qs_; x < n; x += QS) {
    uint8_t* qs = smem + (x / QS & 1) * STAGE;
    const int i0 = job.qa + (x % steps) * QT;
    uint64_t badq = 0, bado = 0;
    if (seen(i0, QT, kb0, kb1) != 2 &&
        __builtin_expect(Cp2::holds_nonfinite(qs, x, found), 0)) {
      badq = Cp::scrub(qs, mask);
      bado = Cp::scrub(qs + BYTES, mask);
    }
    if (x + QS < n) copy(x + QS);
    auto part = [&](auto rb) __attribute__((always_inline)) {
      const int what = seen(i0 + rb, 32, kw, kw + 31);
      if (what) step(qs, i0, rb, what == 1 || (badq | bado) != 0, badq, bado);
    };
    part(std::integral_constant<int, 0>{});
    if constexpr (QT == 64) part(std::integral_constant<int, 32>{});
#pragma unroll 1
    for (; __builtin_expect(bado != 0, 0); bado &= bado - 1) {   // dv takes the cotangents' infinities and NaN
      const int i = i0 + __builtin_ctzll(bado), h = hk * a.G + job.head_part * gh + x / steps;
      add_nonfinite<T, NB>(dv, row_of<T>(g.dout, b, h, i), i >= ilo && i <= ihi, dsel * DO, a.d);
    }
    Cp::sync();
  }
  if constexpr (QS > 1) {
    static_assert((QS - 1) * NB * 16 * 64 * 4 <= QS * 2 * STAGE, "sums of the waves");
    join_waves<QS, NB>(dk, reinterpret_cast<float*>(smem_), qs_);
    if (!join_waves<QS, NB>(dv, reinterpret_cast<float*>(smem_), qs_)) return;
  }
  if (job.slot < 0) {
    store_row<T, NB>(row_of<T>(g.dk, b, hk, jc), dk, a.scale, dsel * DO, a.d, j < a.n_kv, !live);
    store_row<T, NB>(row_of<T>(g.dv, b, hk, jc), dv, 1.0f, dsel * DO, a.d, j < a.n_kv, !live);
  } else {
    float* part = g.part + ((int64_t)bk * g.plan.slots() + job.slot) * 2 * KB * a.d + (int64_t)(32 * wave + (lane & 31)) * a.d;
    store_row<float, NB>(part, dk, a.scale, dsel * DO, a.d, true, !live);
    store_row<float, NB>(part + (int64_t)KB * a.d, dv, 1.0f, dsel * DO, a.d, true, !live);
  }
}

// The same for 16-bit I/O and DP <= 128, two waves a SIMD: QH waves share the
// 32 keys of a wave above, each with 64 / QH queries of a step and its own
// sums (added at the end), so that one's vector work runs beside the other's
// matrix products. The values wait in LDS instead of registers. Four products
// a pair, 40 KB of fragments from LDS for 32 matrix instructions: bound by
// those reads and their waits ([1, 16 / 4, 8192, 128], window 2048, 4 sinks:
// 421 to 462 us by the card's clock, 0.57 to 0.52 PF, matrix cores busy 24 %; 9
// registers spill).
template <int DP, int QH>
__global__ __launch_bounds__(256 * QH, 2) void k_window_dkv16(const WindowBwdArgs g) {
  typedef __bf16 T;
  const WindowArgs& a = g.f;
  constexpr int KB = 128, NT = 256 * QH, QT = 64, NB = DP / 32, QW = QT / QH;
  using L = Tile<T, DP>;
  constexpr int BYTES = QT * L::PITCH, STAGE = 2 * BYTES + 1024, VB = KB * L::PITCH;
  constexpr int RING = DP > 64 ? 3 : 2;   // stages: copies run RING - 1 steps ahead
  __shared__ __attribute__((aligned(1024))) uint8_t smem[VB + RING * STAGE];
  __shared__ uint32_t mask[2];
  __shared__ int found;
  uint8_t* const ring = smem + VB;
  DkvJob job(a, g.plan, blockIdx.x, gridDim.x);
  const int bk = job.bk, b = bk / a.Hkv, hk = bk % a.Hkv;
  const int len = length_of(a, b);
  const FewKeys few(a, len);
  job.queries(a, g.plan, len);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int kg = wave & 3, qh = wave >> 2;
  const int kw = job.tile * KB + 32 * kg, j = kw + (lane & 31), jc = min(j, a.n_kv - 1);
  const bool live = j < len;
  const int iend = min(a.n_q, len - a.q_start);   // queries past it are padding
  const int ilo = max(j - a.look - a.q_start, 0);  // the queries of the job that see key j: ilo .. ihi
  const int ihi = !live ? -1 : min(job.qb - 1, j < a.sinks ? iend - 1 : min(iend - 1, j + a.win - 1 - a.q_start));
  const uint32_t span = (uint32_t)max(ihi - ilo, 0);
  const int first = ihi < ilo ? (1 << 30) : ilo - 4 * half;

  u32x4 kf[L::KS];
  load_row<T, DP>(kf, row_of<T>(a.k, b, hk, jc), live, a.d);
  f32x16 dk[NB], dv[NB];
#pragma unroll
  for (int x = 0; x < NB; ++x) dk[x] = dv[x] = f32x16{};
  const float c = a.scale * kLog2e;
  const int steps = job.qb > job.qa ? (job.qb - job.qa + QT - 1) / QT : 0;
  const int gh = a.G / g.plan.gs, n = steps * gh, h0 = hk * a.G + job.head_part * gh;
  const int ldq = (int)(a.q.st * sizeof(T)), ldo = (int)(g.dout.st * sizeof(T));
  using Cp = Copy<T, DP, QT, NT>;
  typedef __attribute__((address_space(3))) void lds_void;
  int ch = h0, ci = job.qa;   // head and first query of the next copy
  auto copy = [&](int stage) __attribute__((always_inline)) {
    uint8_t* to = ring + stage * STAGE;
    Cp::template rows<(DP > 64)>(to, row_of<T>(a.q, b, ch, ci), ldq, job.qb - ci, a.d);
    Cp::template rows<(DP > 64)>(to + BYTES, row_of<T>(g.dout, b, ch, ci), ldo, job.qb - ci, a.d);
    if (wave < 2) {   // nlse and ndelta of the queries; past the last one zeros (masked)
      const float* from = (wave ? g.ndelta : g.nlse) + ((int64_t)b * a.H + ch) * a.n_q + ci;
      const __amdgpu_buffer_rsrc_t rsrc =
          __builtin_amdgcn_make_buffer_rsrc((void*)from, (short)0, min(QT, job.qb - ci) * 4, kBufFlags);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(to + 2 * BYTES + wave * QT * 4), 4, lane * 4, 0, 0, 0);
    }
    ci += QT;
    if (ci >= job.qb) {
      ci = job.qa;
      ++ch;
    }
  };
  // queries i0 .. against the keys k0 .. k1: nothing (0), something (1) or all (2)
  auto seen = [&](int i0, int count, int k0, int k1) __attribute__((always_inline)) {
    const int pa = a.q_start + i0, pe = a.q_start + min(i0 + count, min(job.qb, iend)) - 1;
    if (pa > pe || k0 >= len || k0 > pe + a.look || (k0 >= a.sinks && k1 <= pa - a.win)) return 0;
    return pe - pa == count - 1 && k1 < len && k1 <= pa + a.look && (k0 > pe - a.win || k1 < a.sinks) ? 2 : 1;
  };
  if (threadIdx.x == 0) found = -1;
  if (n > 0) {
    Copy<T, DP, KB, NT>::rows(smem, row_of<T>(a.v, b, hk, job.tile * KB), (int)(a.v.st * sizeof(T)),
                              len - job.tile * KB, a.d);
    for (int x = 0; x < RING - 1 && x < n; ++x) copy(x);
  }
  __syncthreads();
  int i0 = job.qa, h = h0, stage = 0, to = RING - 1;
  for (int x = 0; x < n; ++x) {
    uint8_t* qs = ring + stage * STAGE;
    uint8_t* os = qs + BYTES;
    uint64_t bado = 0;
    if (seen(i0, QT, job.tile * KB, job.tile * KB + KB - 1) != 2 &&
        __builtin_expect((Copy<T, DP, 2 * QT, NT>::holds_nonfinite(qs, x, &found)), 0)) {
      const uint64_t badq = Cp::scrub(qs, mask);
      bado = Cp::scrub(os, mask);
      // a query's infinity or NaN makes its weights NaN, a cotangent's their cotangents
      float* rows = reinterpret_cast<float*>(qs + 2 * BYTES);
      if (threadIdx.x < QT) {
        if (badq >> threadIdx.x & 1) rows[threadIdx.x] = __builtin_nanf("");
        if (bado >> threadIdx.x & 1) rows[QT + threadIdx.x] = __builtin_nanf("");
      }
      __syncthreads();
    }
    if (x + RING - 1 < n) copy(to);
#pragma unroll
    for (int rb = 0; rb < QW; rb += 32) {
      const int r0 = qh * QW + rb;   // the 32 queries of the step
      const int what = seen(i0 + r0, 32, kw, kw + 31);
      if (!what) continue;
      const uint8_t *qt = qs + r0 * L::PITCH, *ot = os + r0 * L::PITCH;
      // the accumulators start from nlse and ndelta of rows 8e + 4 half ..
      const uint32_t at = lds_addr(qs + 2 * BYTES) + r0 * 4 + 16 * half;
      const uint32_t ad[4] = {at, at + 32, at + 64, at + 96};
      f32x16 s, d;
      auto start = [&](f32x16& acc, auto off) __attribute__((always_inline)) {
        u32x4 r[4];
        read_rows4<decltype(off)::value>(r, ad);
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] = __uint_as_float(r[e >> 2][e & 3]);
      };
      start(s, std::integral_constant<int, 0>{});
      mma_dot_add<T, DP, 0>(s, qt, kf);
      start(d, std::integral_constant<int, 4 * QT>{});
      mma_dot_lds<DP>(d, ot, smem + 32 * kg * L::PITCH);
      if (what == 1) {
        const int lo = first - i0 - r0;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const bool see = (uint32_t)(8 * (e >> 2) + (e & 3) - lo) <= span;
          s[e] = see ? s[e] : neg_inf();
          d[e] = see ? d[e] : 0.0f;
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = __builtin_amdgcn_exp2f(s[e] * c);
        d[e] *= s[e];
      }
      mma_rows<T, DP, NB, 0>(dv, RowsB<T>(s), ot, 0);
      // (of dv, whose weights' rounding nothing of the kind corrects, the same would
      // cost 4 % of a long call, by registers)
      if (__builtin_expect(few.any(i0 + r0), 0))
        mma_rows<T, DP, NB, 0>(dk, RowsB<T>(FewKeys::below_bf16_of(a, len, i0 + r0, d)), qt, 0);
      mma_rows<T, DP, NB, 0>(dk, RowsB<T>(d), qt, 0);
    }
#pragma unroll 1
    for (; __builtin_expect(bado != 0, 0); bado &= bado - 1) {   // dv takes the cotangents' infinities and NaN
      const int r = __builtin_ctzll(bado), i = i0 + r;
      add_nonfinite<T, NB>(dv, row_of<T>(g.dout, b, h, i), r / QW == qh && i >= ilo && i <= ihi, 0, a.d);
    }
    i0 += QT;
    if (i0 >= job.qb) {
      i0 = job.qa;
      ++h;
    }
    stage = stage + 1 == RING ? 0 : stage + 1;
    to = to + 1 == RING ? 0 : to + 1;
    // the next step's copies are done; those of the steps behind it go on
    if (RING == 3 && x + 2 < n) {
      if (wave < 2) wait_loads<2 * Cp::N + 1>();
      else wait_loads<2 * Cp::N>();
    } else {
      wait_loads<0>();
    }
    barrier_only();
  }
  if constexpr (QH == 2) {   // the second wave's sums to the first
    static_assert(4 * NB * 16 * 64 * 4 <= VB + RING * STAGE, "sums of four waves");
    float* to = reinterpret_cast<float*>(smem) + kg * NB * 16 * 64;
    join_waves<2, NB>(dk, to, qh);
    if (!join_waves<2, NB>(dv, to, qh)) return;
  }
  if (job.slot < 0) {
    store_row<T, NB>(row_of<T>(g.dk, b, hk, jc), dk, a.scale, 0, a.d, j < a.n_kv, !live);
    store_row<T, NB>(row_of<T>(g.dv, b, hk, jc), dv, 1.0f, 0, a.d, j < a.n_kv, !live);
  } else {
    float* part = g.part + ((int64_t)bk * g.plan.slots() + job.slot) * 2 * KB * a.d + (int64_t)(32 * kg + (lane & 31)) * a.d;
    store_row<float, NB>(part, dk, a.scale, 0, a.d, true, !live);
    store_row<float, NB>(part + (int64_t)KB * a.d, dv, 1.0f, 0, a.d, true, !live);
  }
}

// dk and dv of the tiles whose sums came in parts, in the order of the parts:
// four elements a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_window_dkv_sum(const WindowBwdArgs g) {
  const WindowArgs& a = g.f;
  const DkvPlan& pl = g.plan;
  const bool ps = pl.np_s * pl.gs > 1, pa = pl.np_a * pl.gs > 1;
  const int t0 = ps ? 0 : pl.st, t1 = pa ? pl.ntile : pl.st;      // tiles in parts: [t0, t1)
  const int64_t per = (int64_t)(t1 - t0) * pl.kb * (a.d / 4);     // work per (batch, key head)
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (x >= per * a.B * a.Hkv) return;
  const int bk = (int)(x / per), b = bk / a.Hkv, hk = bk % a.Hkv;
  const int64_t y = x - bk * per;
  const int e = (int)(y % (a.d / 4)) * 4, row = (int)(y / (a.d / 4)) % pl.kb, t = t0 + (int)(y / (a.d / 4)) / pl.kb;
  const int64_t j = (int64_t)t * pl.kb + row;
  if (j >= a.n_kv) return;
  const bool sink = t < pl.st;
  const int np = (sink ? pl.np_s : pl.np_a) * pl.gs;
  const int slot = sink ? t * np : (ps ? pl.st * pl.np_s * pl.gs : 0) + (t - pl.st) * np;
  const float* part = g.part + ((int64_t)bk * pl.slots() + slot) * 2 * pl.kb * a.d + (int64_t)row * a.d + e;
  f32x4 k = {}, v = {};
  for (int s = 0; s < np; ++s) {
    k += *reinterpret_cast<const f32x4*>(part + (int64_t)s * 2 * pl.kb * a.d);
    v += *reinterpret_cast<const f32x4*>(part + (int64_t)(s * 2 + 1) * pl.kb * a.d);
  }
  T *ok = row_of<T>(g.dk, b, hk, j) + e, *ov = row_of<T>(g.dv, b, hk, j) + e;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<u32x2*>(ok) = u32x2{pack_bf16(k[0], k[1]), pack_bf16(k[2], k[3])};
    *reinterpret_cast<u32x2*>(ov) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  } else {
    *reinterpret_cast<f32x4*>(ok) = k;
    *reinterpret_cast<f32x4*>(ov) = v;
  }
}

int cdiv(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Waves that may share 32 queries (or keys): as many as have room in LDS for
// tiles of their own.
constexpr int sharers(bool bf16, int DP) { return DP <= (bf16 ? 128 : 64) ? 4 : bf16 || DP <= 128 ? 2 : 1; }

// Where workgroups of 128 of n rows would leave CUs idle, workgroups of 32 whose
// waves take turns at the other side's tiles and join their sums: more CUs and
// a shorter chain of tiles. Their LDS holds one workgroup a CU, so past 64
// times four of them they come in rounds, each a W-th as long; fp32's longer
// products forgive more of these. (Heads of more than 128 in bf16 have two such
// waves and would gain past their limit of 48 too.) This and workgroups of 128,
// in us:
//   training  [1, 2, 256, 64] fp32, window 64 (4 workgroups of 128)      43   94
//             [1, 8 / 4, 2048, 64] fp32, window 512 (128)               165  260
//             [1, 12 / 4, 2048, 64] fp32, window 512 (192)              238  262
//             [3, 4 / 2, 1264, 80] fp32, window 348 (120)               309  346
//   forward   [1, 8 / 4, 1024, 128] bf16, window 512 (64)                16   25
//             [1, 8 / 4, 1536, 128] bf16, window 512 (96)                27   25
//             [1, 8 / 4, 2048, 64] bf16, window 512 (128)                19   19
//             [1, 12 / 4, 2048, 64] bf16, window 512 (192)               27   18
//             [1, 4 / 2, 1024, 256] bf16, window 512 (32)                34   50
//             [1, 4 / 2, 2048, 256] bf16, window 512 (64)                36   51
//   dq        [1, 8 / 4, 1024, 128] bf16, window 512 (64)                17   28
//             [1, 8 / 4, 1536, 128] bf16, window 512 (96)                30   29
//             [1, 8 / 4, 1024, 64] bf16, window 512 (64)                 13   22
//             [1, 8 / 4, 1536, 64] bf16, window 512 (96)                 23   22
//             [1, 4 / 2, 1024, 256] bf16, window 512 (32)                29   49
//             [1, 4 / 2, 2048, 256] bf16, window 512 (64)                30   49
bool few_blocks(const WindowArgs& a, bool bf16, int n) {
  const int W = sharers(bf16, a.d <= 64 ? 64 : a.d <= 128 ? 128 : 256);
  return W > 1 && (int64_t)a.B * a.H * cdiv(n, 128) < (bf16 ? 24 : 64) * W;
}

template <typename T, int DP>
hipError_t fwd(const WindowArgs& a, hipStream_t s) {
  // waves a SIMD, by what the registers hold (fp32 at DP = 128: 314 us for
  // [1, 16 / 4, 4096, 128], window 1024; with one wave 380)
  constexpr int OCC = DP > 128 ? 1 : sizeof(T) == 4 || DP > 64 ? 2 : 4, W = sharers(sizeof(T) == 2, DP);
  const int64_t bh = (int64_t)a.B * a.H;
  if (W > 1 && few_blocks(a, sizeof(T) == 2, a.n_q))
    k_window_fwd<T, DP, (W > 1 ? 1 : 4), W, (W > 1 ? 1 : OCC)><<<(unsigned)(bh * cdiv(a.n_q, 32)), 64 * W, 0, s>>>(a);
  else
    k_window_fwd<T, DP, 4, 1, OCC><<<(unsigned)(bh * cdiv(a.n_q, 128)), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T, int DP>
hipError_t bwd(const WindowBwdArgs& g, hipStream_t s) {
  const WindowArgs& a = g.f;
  constexpr bool H16 = sizeof(T) == 2;
  constexpr int DO = DP <= 128 ? DP : H16 ? 128 : 64, QT = 32, W = sharers(H16, DP);
  const int64_t bh = (int64_t)a.B * a.H, bk = (int64_t)a.B * a.Hkv;
  if (a.n_q > 0) {
    if (W > 1 && few_blocks(a, H16, a.n_q))
      k_window_dq<T, DP, (W > 1 ? 1 : 4), W, 1><<<(unsigned)(bh * cdiv(a.n_q, 32)), 64 * W, 0, s>>>(g);
    else
      k_window_dq<T, DP, 4, 1, (H16 && DP <= 128 ? 2 : 1)><<<(unsigned)(bh * cdiv(a.n_q, 128)), 256, 0, s>>>(g);
  }
  if (a.n_kv > 0) {
    if constexpr (H16 && DP <= 128)
      k_window_dkv16<DP, DP / 64><<<(unsigned)(bk * g.plan.jobs()), 256 * (DP / 64), 0, s>>>(g);
    else if (W > 1 && g.plan.kb == 32)
      k_window_dkv<T, DP, DO, QT, (W > 1 ? 1 : 4), W><<<(unsigned)(bk * g.plan.jobs() * (DP / DO)), 64 * W, 0, s>>>(g);
    else
      k_window_dkv<T, DP, DO, QT, 4, 1><<<(unsigned)(bk * g.plan.jobs() * (DP / DO)), 256, 0, s>>>(g);
    const DkvPlan& pl = g.plan;
    const bool ps = pl.np_s * pl.gs > 1 && pl.st > 0, pa = pl.np_a * pl.gs > 1;
    const int t0 = pl.np_s * pl.gs > 1 ? 0 : pl.st, t1 = pa ? pl.ntile : pl.st;
    if (ps || pa) {
      const int64_t n = (int64_t)(t1 - t0) * pl.kb * (a.d / 4) * bk;
      if (n > 0) k_window_dkv_sum<T><<<(unsigned)((n + 255) / 256), 256, 0, s>>>(g);
    }
  }
  return hipGetLastError();
}

}  // namespace

// Tiles of sinks are seen by every later query, the others by a window of
// them: the former are cut into parts of a quarter of the latter's queries
// ([1, 16 / 4, 8192, 128], window 2048, sinks 4: 12 jobs of a whole window's
// size beside 256 others take another round, 720 us; without sinks 400), and
// all of them, by heads first, where the tiles alone would leave CUs idle.
DkvPlan window_dkv_plan(const WindowArgs& a, bool bf16) {
  DkvPlan p{};
  // (16-bit of up to 128 columns has kernels of 128 keys only)
  const bool few = (!bf16 || a.d > 128) && few_blocks(a, bf16, a.n_kv);
  p.kb = few ? 32 : 128;
  p.ntile = cdiv(a.n_kv, p.kb);
  const int n_q = std::max(a.n_q, 1);
  const int reach = (int)std::min<int64_t>(n_q, (int64_t)a.win + a.look + p.kb);   // queries that see a tile
  auto parts = [&](int ch, int* np, int* out) {   // parts of about `ch` queries, at most 64
    *np = std::min(cdiv(n_q, std::max(ch, 1)), 64);
    *out = cdiv(cdiv(n_q, *np), 64) * 64;
  };
  p.np_s = p.np_a = p.gs = 1;
  p.ch_s = p.ch_a = cdiv(n_q, 64) * 64;
  const int64_t tiles = (int64_t)a.B * a.Hkv * p.ntile;
  if (reach < n_q) {
    p.st = cdiv(std::min(a.sinks, a.n_kv), p.kb);
    parts(std::max(256, cdiv(reach, 256) * 64), &p.np_s, &p.ch_s);
    const int64_t enough = 2048 / std::max<int64_t>((int64_t)a.B * a.Hkv * p.st, 1);   // many sink tiles need no parts
    if (p.np_s > enough) parts(cdiv(n_q, std::max<int64_t>(enough, 1)), &p.np_s, &p.ch_s);
  }
  while (tiles * p.gs < (few ? 512 : 256) && p.gs < a.G) {
    int f = 2;
    while (a.G / p.gs % f) ++f;   // the least factor of what is left of the group
    p.gs *= f;
  }
  if (tiles * p.gs < 128 && reach > 512) {
    const int want = (int)std::min<int64_t>(256 / (tiles * p.gs), reach / 256);
    if (want > 1) {
      p.np_a = want;
      p.ch_a = cdiv(cdiv(reach, want), 64) * 64;
      if (p.st) parts(p.ch_a, &p.np_s, &p.ch_s);
    }
  }
  return p;
}

hipError_t launch_window_fwd(const WindowArgs& a, bool bf16, hipStream_t s) {
  if (a.n_q == 0) return hipSuccess;
  if (bf16) return a.d <= 64 ? fwd<__bf16, 64>(a, s) : a.d <= 128 ? fwd<__bf16, 128>(a, s) : fwd<__bf16, 256>(a, s);
  return a.d <= 64 ? fwd<float, 64>(a, s) : a.d <= 128 ? fwd<float, 128>(a, s) : fwd<float, 256>(a, s);
}

hipError_t launch_window_bwd(const WindowBwdArgs& g, bool bf16, hipStream_t s) {
  const int d = g.f.d;
  if (bf16) return d <= 64 ? bwd<__bf16, 64>(g, s) : d <= 128 ? bwd<__bf16, 128>(g, s) : bwd<__bf16, 256>(g, s);
  return d <= 64 ? bwd<float, 64>(g, s) : d <= 128 ? bwd<float, 128>(g, s) : bwd<float, 256>(g, s);
}

}  // namespace lact
