// What the kernels over pages share (lact_paged.hip, lact_prefix.hip): which
// rows a workgroup has, where a key lies, and a tile of keys and values on its
// way through registers.
#pragma once

#include "lact_attn.h"
#include "lact_internal.h"

namespace lact {
namespace attn {

constexpr int kWaves = 4;

// The rows of sequence b: `rows` of them, of tokens t0 .., the first at position p0.
struct Seq {
  int b, t0, rows, p0, len;
};

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

template <class Args>
__device__ __forceinline__ int seq_len(const Args& a, int b) {
  return clampi(a.len[b], 0, a.max_pages * a.page);
}

// The sequences of a call, as find_rows() takes them: their count, the first
// token of each and the keys that it sees.
struct Sequences {
  const PagedArgs& a;
  __device__ __forceinline__ int count() const { return a.B; }
  __device__ __forceinline__ int first(int b) const { return clampi(a.cu[b], 0, a.T); }
  __device__ __forceinline__ int len(int b) const { return seq_len(a, b); }
};

// Row tile `t` of R rows. Up to 64 sequences stand a lane each, in the order of
// the keys they see, most first: what is left for the end, or comes as a
// second workgroup to a CU, is short. More than that stand in their own order,
// sequence b from tile first(b) G / R + b on (rounded down, so that each has room
// for its last partial tile). Tiles past the last one are empty.
template <class Src>
__device__ __forceinline__ bool find_rows(const PagedArgs& a, const Src& src, int t, int R, Seq& s, int& r0) {
  int count, k;
  const int B = src.count();
  if (B <= 64) {
    const int lane = threadIdx.x & 63, b = min(lane, B - 1);
    const int t0 = src.first(b), t1 = src.first(b + 1), len = src.len(b);
    const int n = lane < B ? max(t1, t0) - t0 : 0, tiles = (int)(((int64_t)n * a.G + R - 1) / R);
    const int keys = min(len, a.win);
    int start = 0;
    for (int j = 0; j < B; ++j) {
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
    int lo = 0, hi = B - 1;
    auto first = [&](int b) { return (int)((int64_t)src.first(b) * a.G / R) + b; };
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first(mid) <= t) lo = mid;
      else hi = mid - 1;
    }
    s.b = lo;
    s.t0 = src.first(lo);
    s.len = src.len(lo);
    count = max(src.first(lo + 1), s.t0) - s.t0;
    k = t - first(lo);
  }
  s.rows = count * a.G;
  s.p0 = s.len - count;
  if (k < 0 || (int64_t)k * R >= s.rows) return false;
  r0 = k * R;
  return true;
}
__device__ __forceinline__ bool find_rows(const PagedArgs& a, int t, int R, Seq& s, int& r0) {
  return find_rows(a, Sequences{a}, t, R, s, r0);
}

__device__ __forceinline__ int page_of(int key, uint32_t mul, uint32_t shift) {
  return (int)((__umulhi((uint32_t)key, mul) + (uint32_t)key) >> shift);
}

// The page and place in it of a key; false if it is past the length or its
// page is no page of the cache.
template <class Args>
__device__ __forceinline__ bool find_slot(const Args& a, const int32_t* table, int key, int len, int& pg, int& at) {
  if (key < 0 || key >= len) return false;
  const int pi = page_of(key, a.mul, a.shift);
  pg = table[pi];
  at = key - pi * a.page;
  return pg >= 0 && pg < a.pages;
}

// Where lane l's key k0 + l lies: its offset in elements, < 0 if there is none.
template <class Args>
__device__ __forceinline__ int64_t slot_of(const Args& a, const int32_t* table, int key, int len) {
  int pg, at;
  return find_slot(a, table, key, len, pg, at) ? pg * a.c.sb + at * a.c.st : -1;
}

__device__ __forceinline__ int64_t shfl64(int64_t x, int lane) {
  const int lo = __shfl((int)x, lane, 64), hi = __shfl((int)(x >> 32), lane, 64);
  return ((int64_t)hi << 32) | (uint32_t)lo;
}

constexpr int kKT = 32;   // keys a tile of a wave of its own

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

// 16 bytes of zeros for the lanes of a copy that have nothing to read.
__device__ const uint32_t kZeros[4] = {0, 0, 0, 0};

// Loads that lanes have nothing to read with go to zeros instead of around a
// branch, behind which the compiler could not tell what is in flight and would wait
// for all of it.
template <class X>
__device__ __forceinline__ X load_or_zeros(bool ok, const void* p) {
  typedef __attribute__((address_space(1))) const X global;   // (a choice of generic pointers would count as LDS too)
  return *(ok ? (global*)p : (global*)kZeros);
}
__device__ __forceinline__ u32x4 load16(bool ok, const void* p) { return load_or_zeros<u32x4>(ok, p); }
__device__ __forceinline__ u32x2 load8(bool ok, const void* p) { return load_or_zeros<u32x2>(ok, p); }
__device__ __forceinline__ uint32_t load4(bool ok, const void* p) { return load_or_zeros<uint32_t>(ok, p); }
__device__ __forceinline__ int load_byte(bool ok, const uint8_t* p) { return load_or_zeros<uint8_t>(ok, p); }

}  // namespace attn
}  // namespace lact
