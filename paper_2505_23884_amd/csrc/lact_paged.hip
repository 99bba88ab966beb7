// Attention of new tokens over a cache of pages, and the writes of their keys
// and values into it.
//
// A "row" is one (token, head of a group) pair: the heads that share keys
// stand beside each other in one 32-column tile, so keys and values are read
// once for all of them. Bound by HBM for one or few tokens a sequence (the
// keys and values of the visible positions), by the matrix cores for long
// chunks. Two shapes of a workgroup of four waves:
//   narrow  32 rows; the waves take turns at the tiles of keys, each through
//           LDS of its own, and join their sums at the end: every wave keeps
//           a tile of loads in flight;
//   wide    128 rows, 32 a wave; the tiles pass through LDS for all waves,
//           copied there without registers between.
// Measured, bf16, heads of 128, 16 over 4: decoding of 64 sequences of up to
// 16384 tokens, 1.59 GB, 323 to 349 us by the card's clock, 4.9 to 4.6 TB/s (a
// large copy moves 4.9); one token over a window of 2048, 8.4 us and 4 for the
// joining of 20 parts; six chunks of up to 700 tokens over 4096 to 8192, 201 GF,
// 314 to 354 us, 0.64 to 0.57 PF (matrix cores busy 26 % of the cycles, vector
// instructions 28 %, the rest waits for LDS and for the slots' addresses); 63
// tokens and a chunk of 700, each over 8192, 302 us, where the tokens alone take
// 231 and the chunk 95. Heads of 256 spill 99 registers of the narrow kernel, in
// its loop too: 32 sequences of up to 16384, 1.58 GB, 502 us or 3.1 TB/s.
// Where the row tiles alone would leave the chip idle, the tiles of keys are
// cut into `splits` parts; each leaves its maximum, sum and unnormalised
// output, and k_paged_join adds them in order.
//
// Lengths, offsets and page numbers are device data: they are clamped to the
// tensors here, and a page outside the cache holds nothing (its positions are
// masked, its slots not written).
#include <algorithm>
#include <type_traits>

#include "lact_attn.h"
#include "lact_internal.h"

namespace lact {
namespace {

using namespace attn;

constexpr int kWaves = 4;
constexpr int kKT = 32;   // keys a tile

// The rows of sequence b: `rows` of them, of tokens t0 .., the first at position p0.
struct Seq {
  int b, t0, rows, p0, len;
};

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

template <class Args>
__device__ __forceinline__ int seq_len(const Args& a, int b) {
  return clampi(a.len[b], 0, a.max_pages * a.page);
}

// Row tile `t` of R rows. Up to 64 sequences stand a lane each, in the order of
// the keys they see, most first: what is left for the end, or comes as a
// second workgroup to a CU, is short. More than that stand in their own order,
// sequence b from tile cu[b] G / R + b on (rounded down, so that each has room
// for its last partial tile). Tiles past the last one are empty.
__device__ __forceinline__ bool find_rows(const PagedArgs& a, int t, int R, Seq& s, int& r0) {
  int count, k;
  if (a.B <= 64) {
    const int lane = threadIdx.x & 63, b = min(lane, a.B - 1);
    const int t0 = clampi(a.cu[b], 0, a.T), t1 = a.cu[b + 1], len = seq_len(a, b);
    const int n = lane < a.B ? clampi(t1, t0, a.T) - t0 : 0, tiles = (int)(((int64_t)n * a.G + R - 1) / R);
    const int keys = min(len, a.win);
    int start = 0;
    for (int j = 0; j < a.B; ++j) {
      const int kj = __builtin_amdgcn_readlane(keys, j), nj = __builtin_amdgcn_readlane(tiles, j);
      start += (kj > keys) | ((kj == keys) & (j < lane)) ? nj : 0;
    }
    const uint64_t mine = __ballot(t >= start && t - start < tiles);
    if (!mine) return false;
    s.b = __builtin_ctzll(mine);
    s.t0 = __builtin_amdgcn_readlane(t0, s.b);
    s.len = __builtin_amdgcn_readlane(len, s.b);
    count = __builtin_amdgcn_readlane(n, s.b);
    k = t - __builtin_amdgcn_readlane(start, s.b);
  } else {
    int lo = 0, hi = a.B - 1;
    auto first = [&](int b) { return (int)((int64_t)clampi(a.cu[b], 0, a.T) * a.G / R) + b; };
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first(mid) <= t) lo = mid;
      else hi = mid - 1;
    }
    s.b = lo;
    s.t0 = clampi(a.cu[lo], 0, a.T);
    s.len = seq_len(a, lo);
    count = clampi(a.cu[lo + 1], s.t0, a.T) - s.t0;
    k = t - first(lo);
  }
  s.rows = count * a.G;
  s.p0 = s.len - count;
  if (k < 0 || (int64_t)k * R >= s.rows) return false;
  r0 = k * R;
  return true;
}

__device__ __forceinline__ int page_of(int key, uint32_t mul, uint32_t shift) {
  return (int)((__umulhi((uint32_t)key, mul) + (uint32_t)key) >> shift);
}

// Where lane l's key k0 + l lies: its offset in elements, < 0 if it is past
// the length or its page is no page of the cache.
template <class Args>
__device__ __forceinline__ int64_t slot_of(const Args& a, const int32_t* table, int key, int len) {
  if (key < 0 || key >= len) return -1;
  const int pi = page_of(key, a.mul, a.shift), pg = table[pi];
  if (pg < 0 || pg >= a.pages) return -1;
  return pg * a.c.sb + (key - pi * a.page) * a.c.st;
}

__device__ __forceinline__ int64_t shfl64(int64_t x, int lane) {
  const int lo = __shfl((int)x, lane, 64), hi = __shfl((int)(x >> 32), lane, 64);
  return ((int64_t)hi << 32) | (uint32_t)lo;
}

// A tile of kKT keys and values through the registers of NT threads; `at` is
// each wave's slot_of() of the tile's keys (lane = key).
template <typename T, int DP, int NT>
struct PagedStage {
  using L = Tile<T, DP>;
  static constexpr int N = kKT * L::CPR / NT, STEP = NT / L::CPR;
  static_assert(N >= 1 && kKT * L::CPR % NT == 0 && NT % L::CPR == 0, "tile split");
  u32x4 k[N], v[N];
  __device__ __forceinline__ void load(const T* kb, const T* vb, int64_t at, int d) {
    const int row = threadIdx.x % NT / L::CPR, e = threadIdx.x % L::CPR * L::E;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t o = shfl64(at, row + i * STEP);
      const bool ok = o >= 0 && e < d;
      k[i] = ok ? *reinterpret_cast<const u32x4*>(kb + o + e) : u32x4{};
      v[i] = ok ? *reinterpret_cast<const u32x4*>(vb + o + e) : u32x4{};
    }
  }
  // an infinity or NaN among the values; the values without them
  __device__ __forceinline__ bool any_nonfinite() const {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < N; ++i) bad |= nonfinite<T>(v[i]);
    return bad;
  }
  __device__ __forceinline__ void scrub() {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) v[i][x] = finite_or_zero<T>(v[i][x]);
  }
  __device__ __forceinline__ void store(uint8_t* kt, uint8_t* vt) const {
    const int row = threadIdx.x % NT / L::CPR, c = threadIdx.x % L::CPR;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      *reinterpret_cast<u32x4*>(kt + L::off(row + i * STEP, c)) = k[i];
      *reinterpret_cast<u32x4*>(vt + L::off(row + i * STEP, c)) = v[i];
    }
  }
};

__device__ __forceinline__ void wave_fence() {   // LDS of one wave: its instructions run in order
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The infinities and NaN of a scrubbed tile (offsets `at` of its keys, a lane
// each) to the rows that see them: the sight counts from the lane's first row
// of the tile, key j is row j - 4 (lane / 32) there, which may be below 0.
template <typename T, int DP>
__device__ __forceinline__ void restore_nonfinite(Softmax<DP / 32>& st, const T* vb, int64_t at, int d,
                                                  const Sight& sight) {
#pragma unroll 1
  for (int j = 0; j < kKT; ++j) {
    const int64_t o = shfl64(at, j);
    if (o >= 0) add_nonfinite<T, DP / 32>(st.o, vb + o, sight.see(j - 4 * (int)((threadIdx.x >> 5) & 1)), 0, d);
  }
}

// What a workgroup and its lane work on.
struct RowOf {
  int token, head;      // of this lane's row
  bool ok;
  int p;                // its position
  __device__ __forceinline__ RowOf(const PagedArgs& a, const Seq& s, int hk, int r) {
    ok = r < s.rows;
    const int rc = ok ? r : s.rows - 1, t = rc / a.G;
    token = s.t0 + t;
    head = hk * a.G + rc - t * a.G;
    p = s.p0 + t;
  }
};

// The lane's output, or its part of it.
template <typename T, int DP>
__device__ __forceinline__ void finish(const PagedArgs& a, const RowOf& row, int split, Softmax<DP / 32>& st) {
  const int lane = threadIdx.x & 63;
  const float l = half_sum(st.l);
  if (a.splits == 1) {
    T* o = reinterpret_cast<T*>(a.o.p) + row.token * a.o.st + row.head * a.o.sh;
    store_row<T, DP / 32>(o, st.o, 1.0f / l, 0, a.d, row.ok, l == 0.0f);
    return;
  }
  const int64_t rows = (int64_t)a.T * a.H, at = rows * split + (int64_t)row.token * a.H + row.head;
  store_row<float, DP / 32>(a.part + at * a.d, st.o, 1.0f, 0, a.d, row.ok, false);
  if (row.ok && lane < 32)
    *reinterpret_cast<f32x2*>(a.part + (int64_t)a.splits * rows * a.d + at * 2) = f32x2{st.m, l};
}

// 16 bytes of zeros for the lanes of a copy that have nothing to read.
__device__ const uint32_t kZeros[4] = {0, 0, 0, 0};

template <typename T, int DP, int KT, int OCC>
__global__ __launch_bounds__(64 * kWaves, OCC) void k_paged_wide(const PagedArgs a) {
  using L = Tile<T, DP>;
  constexpr int BYTES = KT * L::PITCH, NT = 64 * kWaves;
  using Cp = Copy<T, DP, KT, NT>;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * BYTES];
  __shared__ uint32_t mask[2];
  __shared__ int found;
  Seq s;
  int r0;
  if (!find_rows(a, blockIdx.x / a.Hkv, 32 * kWaves, s, r0)) return;
  const int hk = blockIdx.x % a.Hkv, split = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const RowOf row(a, s, hk, r0 + 32 * wave + (lane & 31));
  const int rl = min(r0 + 32 * kWaves, s.rows) - 1, wr = r0 + 32 * wave, wl = min(wr + 32, s.rows) - 1;
  const int pa = s.p0 + r0 / a.G, pb = s.p0 + rl / a.G;
  const KeyTiles kt(a, s.len, pa, pb, KT);
  const int wa = s.p0 + wr / a.G, wb = wl >= wr ? s.p0 + wl / a.G : wa - 1;
  const int x0 = (int)((int64_t)kt.count() * split / a.splits), x1 = (int)((int64_t)kt.count() * (split + 1) / a.splits);
  const int32_t* table = a.table + (int64_t)s.b * a.max_pages;
  const T* kb = reinterpret_cast<const T*>(a.kc) + hk * a.c.sh;
  const T* vb = reinterpret_cast<const T*>(a.vc) + hk * a.c.sh;
  u32x4 q[L::KS];
  load_row<T, DP>(q, reinterpret_cast<const T*>(a.q.p) + row.token * a.q.st + row.head * a.q.sh, row.ok, a.d);
  Softmax<DP / 32> st;
  st.init();
  const float c = a.scale * kLog2e;
  const int jhi = row.ok ? row.p : -1;
  // slots (a lane a key) run two tiles ahead of the products, the copies one
  auto slot = [&](int x) __attribute__((always_inline)) {
    return x < x1 && lane < KT ? slot_of(a, table, kt.tile(x) * KT + lane, s.len) : (int64_t)-1;
  };
  auto copy = [&](int x, int64_t at) __attribute__((always_inline)) {
    uint8_t* to = smem + ((x - x0) & 1) * 2 * BYTES;
    typedef __attribute__((address_space(1))) const void gvoid;
    typedef __attribute__((address_space(3))) void lvoid;
#pragma unroll
    for (int i = 0; i < Cp::N; ++i) {
      const int r = threadIdx.x / L::CPR + i * Cp::STEP, e = ((threadIdx.x % L::CPR) ^ L::swz(r)) * L::E;
      const int64_t o = shfl64(at, r);
      const bool ok = o >= 0 && e < a.d;
      uint8_t* dst = to + (i * NT + wave * 64) * 16;
      __builtin_amdgcn_global_load_lds((gvoid*)(ok ? (const void*)(kb + o + e) : (const void*)kZeros), (lvoid*)dst, 16, 0, 0);
      __builtin_amdgcn_global_load_lds((gvoid*)(ok ? (const void*)(vb + o + e) : (const void*)kZeros),
                                       (lvoid*)(dst + BYTES), 16, 0, 0);
    }
  };
  int64_t here = slot(x0), next = slot(x0 + 1);
  if (threadIdx.x == 0) found = -1;
  if (x0 < x1) copy(x0, here);
  __syncthreads();
  for (int x = x0; x < x1; ++x) {
    uint8_t* ks = smem + ((x - x0) & 1) * 2 * BYTES;
    const int k0 = kt.tile(x) * KT;
    const uint64_t there = __ballot(here >= 0);
    const bool whole = there == (KT == 64 ? ~0ull : 0xffffffffull);
    uint64_t bad = 0;   // keys whose values were scrubbed
    if ((!whole || sees(a, s.len, pa, pb, k0, KT) != 2) &&
        __builtin_expect(Cp::holds_nonfinite(ks + BYTES, x, &found), 0))
      bad = Cp::scrub(ks + BYTES, mask);
    if (x + 1 < x1) copy(x + 1, next);
    const int64_t after = slot(x + 2);
    const Sight sight(a, row.p, jhi, k0);
    const uint64_t mine = there >> (4 * (lane >> 5));
    auto see = [&](int r) __attribute__((always_inline)) { return sight.see(r) && (mine >> r & 1); };
    auto step = [&](auto rb) __attribute__((always_inline)) {
      constexpr int RB = decltype(rb)::value;
      const int what = sees(a, s.len, wa, wb, k0 + RB, 32);
      if (what) softmax_step<T, DP, RB>(st, q, ks, ks + BYTES, c, what == 1 || !whole, see);
    };
    step(std::integral_constant<int, 0>{});
    if constexpr (KT == 64) step(std::integral_constant<int, 32>{});
#pragma unroll 1
    for (; __builtin_expect(bad != 0, 0); bad &= bad - 1) {
      const int j = __builtin_ctzll(bad);
      const int64_t o = shfl64(here, j);
      if (o >= 0) add_nonfinite<T, DP / 32>(st.o, vb + o, sight.see(j - 4 * (lane >> 5)), 0, a.d);
    }
    here = next;
    next = after;
    __syncthreads();
  }
  finish<T, DP>(a, row, split, st);
}

template <typename T, int DP>
__global__ __launch_bounds__(64 * kWaves) void k_paged_narrow(const PagedArgs a) {
  using L = Tile<T, DP>;
  constexpr int BYTES = kKT * L::PITCH, JOIN = 32 * (DP + 2) * 4;   // a wave's sums, when they are joined
  constexpr int WAVE = ((2 * BYTES > JOIN ? 2 * BYTES : JOIN) + 1023) / 1024 * 1024;   // tiles start at multiples of their pitch
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kWaves * WAVE];
  Seq s;
  int r0;
  if (!find_rows(a, blockIdx.x / a.Hkv, 32, s, r0)) return;
  const int hk = blockIdx.x % a.Hkv, split = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const RowOf row(a, s, hk, r0 + (lane & 31));
  const int rl = min(r0 + 32, s.rows) - 1;
  const int wa = s.p0 + r0 / a.G, wb = s.p0 + rl / a.G;
  const KeyTiles kt(a, s.len, wa, wb, kKT);
  const int x0 = (int)((int64_t)kt.count() * split / a.splits), x1 = (int)((int64_t)kt.count() * (split + 1) / a.splits);
  const int32_t* table = a.table + (int64_t)s.b * a.max_pages;
  const T* kb = reinterpret_cast<const T*>(a.kc) + hk * a.c.sh;
  const T* vb = reinterpret_cast<const T*>(a.vc) + hk * a.c.sh;
  u32x4 q[L::KS];
  load_row<T, DP>(q, reinterpret_cast<const T*>(a.q.p) + row.token * a.q.st + row.head * a.q.sh, row.ok, a.d);
  Softmax<DP / 32> st;
  st.init();
  const float c = a.scale * kLog2e;
  const int jhi = row.ok ? row.p : -1;
  uint8_t* ks = smem + wave * WAVE;
  PagedStage<T, DP, 64> sg;
  auto slot = [&](int x) __attribute__((always_inline)) { return x < x1 && lane < kKT ? slot_of(a, table, kt.tile(x) * kKT + lane, s.len) : -1; };
  int x = x0 + wave;
  int64_t at = slot(x);
  if (x < x1) sg.load(kb, vb, at, a.d);
  for (; x < x1; x += kWaves) {
    const int64_t here = at;
    const uint32_t there = (uint32_t)__ballot(here >= 0);
    at = slot(x + kWaves);
    const int k0 = kt.tile(x) * kKT;
    const int what = there == 0xffffffffu ? sees(a, s.len, wa, wb, k0, kKT) : 1;
    const bool scrubbed = what == 1 && __any(sg.any_nonfinite());
    if (__builtin_expect(scrubbed, 0)) sg.scrub();
    wave_fence();
    sg.store(ks, ks + BYTES);
    wave_fence();
    if (x + kWaves < x1) sg.load(kb, vb, at, a.d);
    const Sight sight(a, row.p, jhi, k0);
    const uint32_t mine = there >> (4 * (lane >> 5));
    auto see = [&](int r) __attribute__((always_inline)) { return sight.see(r) && (mine >> r & 1); };
    // memory bounds this kernel, so the weights keep their bits: decoding of 64
    // sequences 337 to 344 us, at heads of 64 164 to 172, of 256 478 to 502
    if (what) softmax_step<T, DP, 0, true>(st, q, ks, ks + BYTES, c, what == 1, see);
    if (__builtin_expect(scrubbed, 0)) restore_nonfinite<T, DP>(st, vb, here, a.d, sight);
  }
  // the waves' sums: each lane's [32][DP] and (m, l), added by all threads
  __syncthreads();
  float* mine = reinterpret_cast<float*>(smem + wave * WAVE);
  const float l = half_sum(st.l);
#pragma unroll
  for (int db = 0; db < DP / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4*>(mine + (lane & 31) * DP + 32 * db + 8 * g + 4 * (lane >> 5)) =
          f32x4{st.o[db][4 * g], st.o[db][4 * g + 1], st.o[db][4 * g + 2], st.o[db][4 * g + 3]};
  if (lane < 32) {
    mine[32 * DP + 2 * lane] = st.m;
    mine[32 * DP + 2 * lane + 1] = l;
  }
  __syncthreads();
  const int64_t rows = (int64_t)a.T * a.H;
  for (int x4 = threadIdx.x; x4 < 32 * (DP / 4); x4 += 64 * kWaves) {
    const int r = x4 / (DP / 4), e = x4 % (DP / 4) * 4;
    const RowOf out(a, s, hk, r0 + r);
    if (!out.ok || e >= a.d) continue;
    float m = neg_inf(), sum = 0.0f;
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, reinterpret_cast<const float*>(smem + w * WAVE)[32 * DP + 2 * r]);
    f32x4 o = {};
    for (int w = 0; w < kWaves; ++w) {
      const float* of = reinterpret_cast<const float*>(smem + w * WAVE);
      const float mw = of[32 * DP + 2 * r];
      const float f = mw == neg_inf() ? 0.0f : __builtin_amdgcn_exp2f(mw - m);
      sum += of[32 * DP + 2 * r + 1] * f;
      o += *reinterpret_cast<const f32x4*>(of + r * DP + e) * f;
    }
    if (a.splits == 1) {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      T* dst = reinterpret_cast<T*>(a.o.p) + out.token * a.o.st + out.head * a.o.sh + e;
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<u32x2*>(dst) = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
      else
        *reinterpret_cast<f32x4*>(dst) = o * inv;
    } else {
      const int64_t at_ = rows * split + (int64_t)out.token * a.H + out.head;
      *reinterpret_cast<f32x4*>(a.part + at_ * a.d + e) = o;
      if (e == 0) *reinterpret_cast<f32x2*>(a.part + (int64_t)a.splits * rows * a.d + at_ * 2) = f32x2{m, sum};
    }
  }
}

// The parts of each (token, head), joined in a fixed order; rows past the last
// sequence are left as they were. A row has G lanes of four elements, times W:
// the W-th parts from w on are added by lanes of their own, four loads in
// flight, and the W sums through LDS.
template <typename T>
__global__ __launch_bounds__(256) void k_paged_join(const PagedArgs a, int G, int W) {
  __shared__ f32x4 so[256];
  __shared__ f32x2 sm[256];
  const int lg = threadIdx.x & (G - 1), w = threadIdx.x / G & (W - 1);
  const int64_t rows = (int64_t)a.T * a.H, r = (int64_t)blockIdx.x * (256 / (G * W)) + threadIdx.x / (G * W);
  const int token = (int)(r / a.H), head = (int)(r % a.H), e = lg * 4;
  const bool ok = r < rows && token >= clampi(a.cu[0], 0, a.T) && token < clampi(a.cu[a.B], 0, a.T);
  const float* ml = a.part + (int64_t)a.splits * rows * a.d;
  float m = neg_inf(), sum = 0.0f;
  f32x4 o = {};
  auto add = [&](f32x2 x, f32x4 y) __attribute__((always_inline)) {
    const float up = fmaxf(m, x[0]);
    if (up == neg_inf()) return;
    const float f = __builtin_amdgcn_exp2f(m - up), g = __builtin_amdgcn_exp2f(x[0] - up);
    sum = sum * f + x[1] * g;
    o = o * f + y * g;
    m = up;
  };
  if (ok) {
    for (int s0 = w; s0 < a.splits; s0 += 4 * W) {
      f32x2 x[4];
      f32x4 y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s = s0 + i * W;
        x[i] = s < a.splits ? *reinterpret_cast<const f32x2*>(ml + (rows * s + r) * 2) : f32x2{neg_inf(), 0.0f};
        y[i] = s < a.splits && e < a.d ? *reinterpret_cast<const f32x4*>(a.part + (rows * s + r) * a.d + e) : f32x4{};
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) add(x[i], y[i]);
    }
  }
  if (W > 1) {
    so[threadIdx.x] = o;
    sm[threadIdx.x] = f32x2{m, sum};
    __syncthreads();
    if (w) return;
    for (int i = 1; i < W; ++i) add(sm[threadIdx.x + i * G], so[threadIdx.x + i * G]);
  }
  if (!ok || e >= a.d) return;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  T* dst = reinterpret_cast<T*>(a.o.p) + token * a.o.st + head * a.o.sh + e;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<u32x2*>(dst) = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
  else
    *reinterpret_cast<f32x4*>(dst) = o * inv;
}

// Keys and values of the new tokens into their slots, 16 bytes a thread. Bound
// by HBM: 8 chunks of up to 4000 tokens, 8 heads of 128, 210 MB in 33 us
// (partly from the caches).
template <typename T>
__global__ __launch_bounds__(256) void k_paged_append(const AppendArgs a) {
  constexpr int E = 16 / (int)sizeof(T);
  const int cpt = a.Hkv * (a.d / E);
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t token = x / cpt;
  if (token >= a.T) return;
  const int y = (int)(x - token * cpt), h = y / (a.d / E), e = (y - h * (a.d / E)) * E;
  int lo = 0, hi = a.B;   // the last sequence that starts at or before the token
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (mid < a.B && a.cu[mid] <= token) lo = mid;
    else hi = mid - 1;
  }
  const int t0 = a.cu[lo], t1 = min(a.cu[lo + 1], a.T);   // (as find_rows)
  if (token < t0 || token >= t1) return;
  const int len = clampi(a.len[lo], 0, a.max_pages * a.page);
  const int64_t pos = len - ((int64_t)t1 - token);
  if (pos < 0) return;
  const int pi = page_of((int)pos, a.mul, a.shift), pg = a.table[(int64_t)lo * a.max_pages + pi];
  if (pg < 0 || pg >= a.pages) return;
  const int64_t to = pg * a.c.sb + h * a.c.sh + ((int)pos - pi * a.page) * a.c.st + e;
  const u32x4 k = *reinterpret_cast<const u32x4*>(reinterpret_cast<const T*>(a.k.p) + token * a.k.st + h * a.k.sh + e);
  const u32x4 v = *reinterpret_cast<const u32x4*>(reinterpret_cast<const T*>(a.v.p) + token * a.v.st + h * a.v.sh + e);
  *reinterpret_cast<u32x4*>(reinterpret_cast<T*>(a.kc) + to) = k;
  *reinterpret_cast<u32x4*>(reinterpret_cast<T*>(a.vc) + to) = v;
}

int row_tiles(const PagedArgs& a, bool wide) { return (int)((int64_t)a.T * a.G / (wide ? 32 * kWaves : 32)) + a.B; }

template <typename T, int DP>
hipError_t run(const PagedArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(row_tiles(a, a.wide) * a.Hkv), (unsigned)a.splits);
  if constexpr (sizeof(T) == 4 && DP == 256) {
    k_paged_wide<T, DP, 32, 1><<<grid, 64 * kWaves, 0, s>>>(a);   // a wave's own tile would not fit
  } else {
    constexpr bool H = sizeof(T) == 2 && DP <= 128;
    if (a.wide) k_paged_wide<T, DP, H ? 64 : 32, H ? 2 : 1><<<grid, 64 * kWaves, 0, s>>>(a);
    else k_paged_narrow<T, DP><<<grid, 64 * kWaves, 0, s>>>(a);
  }
  if (a.splits > 1) {
    int G = 1, W = 1;
    while (G * 4 < a.d) G *= 2;
    const int64_t rows = (int64_t)a.T * a.H;
    // few rows: more lanes each, up to a workgroup a CU (a decoding token of 16
    // heads, 20 parts: 13.4 us one after the other, 4.1 us so)
    while (G * W < 256 && 4 * W < a.splits && rows * G * W < 256 * 256) W *= 2;
    const int per = 256 / (G * W);
    k_paged_join<T><<<(unsigned)((rows + per - 1) / per), 256, 0, s>>>(a, G, W);
  }
  return hipGetLastError();
}

}  // namespace

void paged_plan(PagedArgs& a, bool bf16) {
  // rows a sequence on average: more than one narrow tile's, and the keys
  // are better shared by four waves (16 / 4 heads of 128, 64 sequences of 4096:
  // 24 rows 118 us narrow and 117 wide, 36 rows 154 and 122, 72 rows 218 and 134;
  // of 16 sequences, which leave CUs idle, 24 rows 50 and 36)
  a.wide = (int64_t)a.T * a.G > 32 * (int64_t)a.B || (!bf16 && a.d > 128);
  const int64_t groups = (int64_t)row_tiles(a, a.wide) * a.Hkv;
  const int64_t most = std::max<int64_t>(1, ((int64_t)a.max_pages * a.page + kKT - 1) / kKT / (2 * kWaves));
  if (!a.wide) {
    a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({(1024 + groups - 1) / groups, most, 32}));
    return;
  }
  // The split that fills the rounds of 512 workgroups (two a CU) best; its sums
  // and their joining cost about a tenth (6 sequences of 4096 to 8192 tokens,
  // 350 to 700 new, 416 workgroups: unsplit 353 us, two or three parts 370).
  double best = 0;
  for (int s = 1; s <= std::min<int64_t>(most, 16); ++s) {
    const double t = (double)((groups * s + 511) / 512) / s * (s > 1 ? 1.08 + 0.02 * s : 1.0);
    if (s == 1 || t < best) {
      best = t;
      a.splits = s;
    }
  }
}

hipError_t launch_paged(const PagedArgs& a, bool bf16, hipStream_t s) {
  if (bf16) return a.d <= 64 ? run<__bf16, 64>(a, s) : a.d <= 128 ? run<__bf16, 128>(a, s) : run<__bf16, 256>(a, s);
  return a.d <= 64 ? run<float, 64>(a, s) : a.d <= 128 ? run<float, 128>(a, s) : run<float, 256>(a, s);
}

hipError_t launch_append(const AppendArgs& a, bool bf16, hipStream_t s) {
  const int64_t n = (int64_t)a.T * a.Hkv * (a.d / (bf16 ? 8 : 4));
  const unsigned blocks = (unsigned)((n + 255) / 256);
  if (bf16) k_paged_append<__bf16><<<blocks, 256, 0, s>>>(a);
  else k_paged_append<float><<<blocks, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lact
