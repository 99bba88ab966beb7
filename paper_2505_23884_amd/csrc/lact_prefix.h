// Attention of new tokens over pages of either kind of cache (the elements of
// the call, or e4m3 numbers), with or without prefixes that groups of
// sequences share.
//
// The softmax of a row over the keys of its group's prefix and over those of
// its own sequence are joined at the end,
//   o = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i,  m = max_i m_i,
// so the two are computed apart: the rows of a whole group stand beside each
// other over the prefix, whose keys and values are read once for all of them,
// and each sequence's over its own keys. Both are workgroups of one launch; the
// prefix's, which last longer, come first.
#pragma once

#include <type_traits>

#include "lact_codes.h"
#include "lact_paged.h"

namespace lact {
namespace {

using namespace attn;

struct Code;   // the cache's elements: e4m3 numbers (else those of the call)

// The keys that a role's rows see, in the positions of its own table: those of
// a sequence without the prefix's count from its end.
struct Band {
  int win, look, sinks;
};

// Where part `i` of n parts of `count` tiles begins (2^24 tiles of 32 at most, 64 parts).
__device__ __forceinline__ int share(int count, int i, int n) { return (int)((uint32_t)count * (uint32_t)i / (uint32_t)n); }

// What a workgroup works on: `rows` rows from token t0 on, from row r0, over
// part `split` of `splits` of the tiles of keys, to part `part` of the sums
// (< 0: to the output).
struct Job {
  const int32_t* table;
  int t0, rows, r0, len, split, splits, part;
  Band band;
};

// A lane's row.
struct Row {
  int token, head;
  bool ok;
  Row() = default;
  __device__ __forceinline__ Row(const PrefixArgs& a, const Job& j, int hk, int r) {
    ok = r < j.rows;
    const int rc = ok ? r : j.rows - 1, t = rc / a.G;
    token = j.t0 + t;
    head = hk * a.G + rc - t * a.G;
  }
};

// The offsets of a call's sequences, clamped, are brought to LDS first (those
// of up to kOffsets sequences; of more they are read where they lie): everything that
// a workgroup has to find then takes one round trip to memory, with the
// offsets, lengths and groups on their way together.
constexpr int kOffsets = 511;
struct Offsets {
  const PrefixArgs& a;
  const int* lds;
  __device__ __forceinline__ Offsets(const PrefixArgs& a_, int* to) : a(a_), lds(to) {
    if (a.B <= kOffsets)
      for (int i = threadIdx.x; i <= a.B; i += 64 * kWaves) to[i] = clampi(a.cu[i], 0, a.T);
  }
  __device__ __forceinline__ int operator()(int b) const { return a.B <= kOffsets ? lds[b] : clampi(a.cu[b], 0, a.T); }
};

// What a role's rows come from: sequences, or groups of them. Its count, and
// of item i the first token and the keys that it has.
struct Items {
  const PrefixArgs& a;
  const Offsets& off;
  bool groups;
  __device__ __forceinline__ int count() const { return groups ? a.P : a.B; }
  __device__ __forceinline__ int at(int i) const { return groups ? clampi(a.cu_seq[i], 0, a.B) : i; }
  __device__ __forceinline__ int first(int i) const { return off(at(i)); }
  __device__ __forceinline__ int len(int i) const { return groups ? clampi(a.plen[i], 0, a.p_pages * a.page) : seq_len(a, i); }
};

// Row tile `t` of R rows, as find_rows() has them: up to 64 items in the order
// of their keys, most first; of more, item i from tile first(i) G / R + i on.
template <bool GROUPS>
__device__ __forceinline__ bool find_tile(const PrefixArgs& a, const Offsets& off, int t, int R, Seq& s, int& r0) {
  const Items it{a, off, GROUPS};
  const int n = it.count();
  int count, k;
  if (n <= 64) {
    const int lane = threadIdx.x & 63, i = min(lane, n - 1);
    const int b0 = it.at(i), b1 = it.at(i + 1), len = it.len(i);   // (loads before the offsets are waited for)
    // rank by keys; the lane in its low bits makes each one's its own
    const int mine = min(len, a.win) >> 5 << 6 | (63 - lane);
    __syncthreads();
    const int t0 = off(b0), c = lane < n ? max(off(b1), t0) - t0 : 0, tiles = (int)(((int64_t)c * a.G + R - 1) / R);
    int start = 0;
    for (int j = 0; j < n; ++j) {
      const int nj = __builtin_amdgcn_readlane(tiles, j);
      start += __builtin_amdgcn_readlane(mine, j) > mine ? nj : 0;
    }
    const uint64_t found = __ballot(t >= start && t - start < tiles);
    if (!found) return false;
    s.b = __builtin_ctzll(found);
    s.t0 = __builtin_amdgcn_readlane(t0, s.b);
    s.len = __builtin_amdgcn_readlane(len, s.b);
    count = __builtin_amdgcn_readlane(c, s.b);
    k = t - __builtin_amdgcn_readlane(start, s.b);
  } else {
    __syncthreads();
    int lo = 0, hi = n - 1;
    auto first = [&](int i) { return (int)((int64_t)it.first(i) * a.G / R) + i; };
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first(mid) <= t) lo = mid;
      else hi = mid - 1;
    }
    s.b = lo;
    s.t0 = it.first(lo);
    s.len = it.len(lo);
    count = max(it.first(lo + 1), s.t0) - s.t0;
    k = t - first(lo);
  }
  s.rows = count * a.G;
  s.p0 = s.len - count;
  if (k < 0 || (int64_t)k * R >= s.rows) return false;
  r0 = k * R;
  return true;
}

// The position of a token among its sequence's own keys (< 0 for one that its
// sequence does not hold).
__device__ __forceinline__ int own_position(const PrefixArgs& a, const Offsets& off, int token) {
  int b = 0, hi = a.B - 1;
  while (b < hi) {
    const int mid = (b + hi + 1) >> 1;
    if (off(mid) <= token) b = mid;
    else hi = mid - 1;
  }
  return seq_len(a, b) - (off(b + 1) - token);
}

// The group of sequence b, or -1.
__device__ __forceinline__ int group_of(const PrefixArgs& a, int b) {
  if (!a.P) return -1;
  int lo = 0, hi = a.P - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.cu_seq[mid] <= b) lo = mid;
    else hi = mid - 1;
  }
  return a.cu_seq[lo] <= b && b < a.cu_seq[lo + 1] ? lo : -1;
}

// A key's page, as the table has it (not looked at: the load stays in flight),
// and its place there, < 0 if it is past the length.
struct Place {
  int page, at;
  Place() = default;
  // (only where there are keys: entry 0 of the table is read for those past them)
  __device__ __forceinline__ Place(const PrefixArgs& a, const int32_t* table, int key, int len) {
    const bool ok = key < len;
    const int pi = page_of(ok ? key : 0, a.mul, a.shift);
    page = table[pi];
    at = ok ? key - pi * a.page : -1;
  }
};

// Where it lies: offsets of its vectors and of its scales, `at` < 0 if there is none.
template <class C>
struct Slot {
  int64_t at;
  Slot() = default;
  __device__ __forceinline__ Slot(const PrefixArgs& a, const Place& p)
      : at(p.at >= 0 && p.page >= 0 && p.page < a.pages ? p.page * a.c.sb + p.at * a.c.st : -1) {}
};
template <>
struct Slot<Code> {
  int64_t at, scale;
  Slot() = default;
  __device__ __forceinline__ Slot(const PrefixArgs& a, const Place& p) {
    const bool ok = p.at >= 0 && p.page >= 0 && p.page < a.pages;
    at = ok ? p.page * a.c.sb + p.at * a.c.st : -1;
    scale = ok ? p.page * a.cs.sb + p.at * a.cs.st : 0;
  }
};

// Has the compiler wait here for what is loaded in these registers, so that a
// loop that uses them does not (it would wait for its own loads with them).
template <class X>
__device__ __forceinline__ void arrived(X& x) {
  if constexpr (std::is_array<X>::value) {
#pragma unroll
    for (auto& y : x) arrived(y);
  } else {
    asm volatile("" : "+v"(x));
  }
}

// The caches of one key head.
template <class C>
struct Heads {
  const C *k, *v;
  __device__ __forceinline__ Heads(const PrefixArgs& a, int hk)
      : k(static_cast<const C*>(a.kc) + hk * a.c.sh), v(static_cast<const C*>(a.vc) + hk * a.c.sh) {}
};
template <>
struct Heads<Code> {
  const uint8_t *k, *v, *ks, *vs;
  __device__ __forceinline__ Heads(const PrefixArgs& a, int hk)
      : k(static_cast<const uint8_t*>(a.kc) + hk * a.c.sh), v(static_cast<const uint8_t*>(a.vc) + hk * a.c.sh),
        ks(a.ks + hk * a.cs.sh), vs(a.vs + hk * a.cs.sh) {}
};

// A tile of KT keys and values in e4m3 numbers on its way from memory to LDS,
// as bf16, through the registers of NT threads. Each wave's lanes know where the
// tile's keys lie (lane = key).
template <int DP, int KT, int NT>
struct Stage {
  using L = Tile<__bf16, DP>;
  static constexpr int CPR = DP / 16;   // 16 numbers a load
  static constexpr int N = KT * CPR / NT, STEP = NT / CPR;
  static_assert(N >= 1 && KT * CPR % NT == 0, "tile split");
  u32x4 k[N], v[N];
  int kb, vb;   // scales of the lane's key
  static __device__ __forceinline__ int row(int i) { return threadIdx.x % NT / CPR + i * STEP; }
  __device__ __forceinline__ void load(const Heads<Code>& h, const Slot<Code>& s, int d) {
    const int e = threadIdx.x % CPR * 16;
    kb = load_byte(s.at >= 0, h.ks + s.scale);
    vb = load_byte(s.at >= 0, h.vs + s.scale);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t o = shfl64(s.at, row(i) & 63);
      const bool ok = o >= 0 && e < d;
      k[i] = load16(ok, h.k + o + e);
      v[i] = load16(ok, h.v + o + e);
    }
  }
  __device__ __forceinline__ void put(uint8_t* kt, uint8_t* vt) {
    const int c = threadIdx.x % CPR * 2;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row(i);
      const float ks = scale_of(__shfl(kb, r & 63, 64)), vs = scale_of(__shfl(vb, r & 63, 64));
      uint32_t w[8];
#pragma unroll
      for (int x = 0; x < 4; ++x) widen<__bf16>(k[i][x], ks, w + 2 * x);
      *reinterpret_cast<u32x4*>(kt + L::off(r, c)) = u32x4{w[0], w[1], w[2], w[3]};
      *reinterpret_cast<u32x4*>(kt + L::off(r, c + 1)) = u32x4{w[4], w[5], w[6], w[7]};
#pragma unroll
      for (int x = 0; x < 4; ++x) widen<__bf16>(v[i][x], vs, w + 2 * x);
      *reinterpret_cast<u32x4*>(vt + L::off(r, c)) = u32x4{w[0], w[1], w[2], w[3]};
      *reinterpret_cast<u32x4*>(vt + L::off(r, c + 1)) = u32x4{w[4], w[5], w[6], w[7]};
    }
  }
};

// The infinities and NaN of key j of a tile, whose values were scrubbed, to
// the rows that see it (as add_nonfinite()).
template <typename T, class C, int DP>
__device__ __forceinline__ void restore_key(Softmax<DP / 32>& st, const Heads<C>& h, const Slot<C>& s, int j, int d,
                                            const Sight& sight) {
  const int64_t o = shfl64(s.at, j);
  if (o < 0) return;
  const bool see = sight.see(j - 4 * (int)((threadIdx.x >> 5) & 1));
  if constexpr (std::is_same<C, Code>::value) {
    const uint8_t* row = h.v + o;
    const float scale = scale_of(h.vs[shfl64(s.scale, j)]);
    int half = (threadIdx.x >> 5) & 1;
    asm volatile("" : "+v"(half));   // (as add_nonfinite())
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int e = 32 * db + 8 * (i >> 2) + 4 * half + (i & 3);
        if (!see || e >= d) continue;
        uint32_t w[2];
        widen<__bf16>(row[e], scale, w);
        const float x = __uint_as_float(w[0] << 16);
        if (!(fabsf(x) < __builtin_inff())) st.o[db][i] += x;
      }
  } else {
    add_nonfinite<T, DP / 32>(st.o, h.v + o, see, 0, d);
  }
}

// What a lane's row sees: keys up to jhi of those that its position p sees.
// The positions of the wave's rows are wa .. wb, of the workgroup's pa .. pb
// (none: from 1 to 0).
struct Sights {
  int p, jhi, wa, wb, pa, pb;
};

// Rows of one sequence over its own keys: their positions follow each other.
__device__ __forceinline__ Sights own_sights(const PrefixArgs& a, const Job& j, int p0, const Row& row, int wr, int R) {
  Sights s;
  s.p = p0 + (row.token - j.t0);
  s.jhi = row.ok ? s.p : -1;
  const int rl = min(j.r0 + R, j.rows) - 1, wl = min(wr + min(R, 32), j.rows) - 1;
  s.pa = p0 + j.r0 / a.G;
  s.pb = p0 + rl / a.G;
  s.wa = p0 + wr / a.G;
  s.wb = wl >= wr ? p0 + wl / a.G : s.wa - 1;
  return s;
}

// Rows of a group over its prefix: the positions are those of their sequences,
// behind all keys. A row that its sequence does not hold stands before them.
// wa .. wb are those of the wave's rows (of which lane l has row l % N).
template <int N>
__device__ __forceinline__ Sights group_sights(const PrefixArgs& a, const Offsets& off, const Job& j, const Row& row) {
  Sights s;
  const int p = own_position(a, off, row.token);
  s.p = p < 0 ? -1 : j.len + p;
  s.jhi = row.ok && p >= 0 ? j.len - 1 : -1;
  int lo = row.ok ? s.p : 1 << 30, hi = row.ok ? s.p : -1;
#pragma unroll
  for (int x = 1; x < N; x *= 2) {
    lo = min(lo, __shfl_xor(lo, x, 64));
    hi = max(hi, __shfl_xor(hi, x, 64));
  }
  const bool some = __any(row.ok);
  s.pa = s.wa = some ? __builtin_amdgcn_readfirstlane(lo) : 1;
  s.pb = s.wb = some ? __builtin_amdgcn_readfirstlane(hi) : 0;
  return s;
}
// The same over the waves of a workgroup, through LDS (eight words).
__device__ __forceinline__ void join_sights(Sights& s, int* lds) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((threadIdx.x & 63) == 0) {
    lds[2 * wave] = s.wa <= s.wb ? s.wa : 1 << 30;
    lds[2 * wave + 1] = s.wa <= s.wb ? s.wb : -1;
  }
  __syncthreads();
  int lo = lds[0], hi = lds[1];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    lo = min(lo, lds[2 * w]);
    hi = max(hi, lds[2 * w + 1]);
  }
  s.pa = __builtin_amdgcn_readfirstlane(lo);
  s.pb = __builtin_amdgcn_readfirstlane(hi);
}

// Part `part` of a row's sums, or the output.
template <typename T>
__device__ __forceinline__ T* out_row(const PrefixArgs& a, const Row& row) {
  return reinterpret_cast<T*>(a.o.p) + row.token * a.o.st + row.head * a.o.sh;
}
__device__ __forceinline__ int64_t part_row(const PrefixArgs& a, int part, const Row& row) {
  return (int64_t)a.T * a.H * part + (int64_t)row.token * a.H + row.head;
}
__device__ __forceinline__ f32x2* part_sums(const PrefixArgs& a, int64_t row) {
  return reinterpret_cast<f32x2*>(a.part + (int64_t)(a.psplits + a.splits) * a.T * a.H * a.d) + row;
}

template <typename T, int DP>
struct Shapes {
  using L = Tile<T, DP>;
  static constexpr bool H = sizeof(T) == 2 && DP <= 128;
  static constexpr int KT = H ? 64 : 32, BYTES = KT * L::PITCH, WIDE = 4 * BYTES;
  static constexpr int JOIN = 32 * (DP + 2) * 4;
  static constexpr int WAVE = ((2 * kKT * L::PITCH > JOIN ? 2 * kKT * L::PITCH : JOIN) + 1023) / 1024 * 1024;
};

// 128 rows, 32 a wave; the tiles pass through LDS for all waves. The elements
// of the call are copied there without registers between, e4m3 numbers are
// widened on the way (once for all waves) and, having no copies in flight that LDS reads would
// wait for, are read a stretch ahead of the products. Bound by vector and matrix work that
// take turns (43 and 31 % of the cycles), 8 chunks of 1024 tokens over 8192 keys, 16 / 4 heads
// of 128: e4m3 0.69 PF, bf16 0.65; 64 keys a tile, since 32 cost 20 % more.
// WHOLE: bf16 weights in two parts, for the rows of groups whose sequences have few
// each (up to 32 on average, as the rows over their own keys then have them): 64 tokens
// behind 16384 bf16 keys 50 us for 49, 2 x 48 behind 30011 in 8 bits 78 for 70, heads of 256 117 for 111.
template <typename T, class C, int DP, bool WHOLE>
__device__ __forceinline__ void wide(const PrefixArgs& a, const Job& jb, const Row& row, const Sights& sg, int hk,
                                     uint8_t* smem, uint32_t* mask, int* found) {
  using L = Tile<T, DP>;
  constexpr bool CODES = std::is_same<C, Code>::value;
  constexpr int KT = Shapes<T, DP>::KT, BYTES = KT * L::PITCH, NT = 64 * kWaves;
  using Cp = Copy<T, DP, KT, NT>;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const KeyTiles kt(jb.band, jb.len, sg.pa, sg.pb, KT);
  const int x0 = share(kt.count(), jb.split, jb.splits), x1 = share(kt.count(), jb.split + 1, jb.splits);
  const Heads<C> hd(a, hk);
  u32x4 q[L::KS];
  load_row<T, DP>(q, reinterpret_cast<const T*>(a.q.p) + row.token * a.q.st + row.head * a.q.sh, row.ok, a.d);
  Softmax<DP / 32> st;
  st.init();
  const float c = a.scale * kLog2e;
  arrived(q);
  constexpr bool PIPED = CODES && DP <= 128;
  // (addresses as in mma_dot_add() and mma_rows(): chunks by flipping bits of the first one's)
  typedef __attribute__((address_space(3))) const u32x4 lds_u4;
  typedef __attribute__((address_space(3))) s16x4 lds_s4;
  const int sl = lane & 15, vrow = 4 * (lane >> 5) + (sl >> 2), vchunk = 2 * (lane >> 4 & 1) + (sl >> 1 & 1);
  const uint32_t kat = L::off(lane & 31, lane >> 5), vlo = L::off(vrow, vchunk) + ((sl & 1) << 3),
                 vhi = L::off(vrow + 8, vchunk) + ((sl & 1) << 3);
  auto read_keys = [&](u32x4 (&f)[L::KS], uint32_t t) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < L::KS; ++i) f[i] = *(lds_u4*)(uintptr_t)((t + kat) ^ (uint32_t)(i << 5));
  };
  auto read_values = [&](u32x2 (&f)[4 * L::DB], uint32_t t) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < L::DB; ++b)
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const uint32_t at = ((t + (h & 1 ? vhi : vlo)) ^ (uint32_t)(b << 6)) + (h >> 1) * 16 * L::PITCH;
        f[4 * b + h] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(uintptr_t)at));
      }
  };
  // pages (a lane a key) run two tiles ahead of the products, the copies one
  auto place = [&](int x) __attribute__((always_inline)) {
    Place p{};
    p.at = -1;
    if (x < x1) p = Place(a, jb.table, lane < KT ? kt.tile(x) * KT + lane : jb.len, jb.len);
    return p;
  };
  auto tile_of = [&](int x) __attribute__((always_inline)) { return smem + ((x - x0) & 1) * 2 * BYTES; };
  [[maybe_unused]] typename std::conditional<CODES, Stage<DP, KT, NT>, Softmax<1>>::type stage;
  auto copy = [&](int x, const Slot<C>& s) __attribute__((always_inline)) {
    if constexpr (CODES) {
      stage.load(hd, s, a.d);
    } else {
      uint8_t* to = tile_of(x);
      typedef __attribute__((address_space(1))) const void gvoid;
      typedef __attribute__((address_space(3))) void lvoid;
#pragma unroll
      for (int i = 0; i < Cp::N; ++i) {
        const int r = threadIdx.x / L::CPR + i * Cp::STEP, e = ((threadIdx.x % L::CPR) ^ L::swz(r)) * L::E;
        const int64_t o = shfl64(s.at, r);
        const bool ok = o >= 0 && e < a.d;
        uint8_t* dst = to + (i * NT + wave * 64) * 16;
        __builtin_amdgcn_global_load_lds((gvoid*)(ok ? (const void*)(hd.k + o + e) : (const void*)kZeros), (lvoid*)dst, 16,
                                         0, 0);
        __builtin_amdgcn_global_load_lds((gvoid*)(ok ? (const void*)(hd.v + o + e) : (const void*)kZeros),
                                         (lvoid*)(dst + BYTES), 16, 0, 0);
      }
    }
  };
  auto arrive = [&](int x) __attribute__((always_inline)) {
    if constexpr (CODES) stage.put(tile_of(x), tile_of(x) + BYTES);
  };
  Slot<C> here(a, place(x0));
  Place next = place(x0 + 1);
  if (threadIdx.x == 0) *found = -1;
  if (x0 < x1) {
    copy(x0, here);
    arrive(x0);
  }
  __syncthreads();
  for (int x = x0; x < x1; ++x) {
    uint8_t* ks = tile_of(x);
    const int k0 = kt.tile(x) * KT;
    const uint64_t there = __ballot(here.at >= 0);
    const bool whole = there == (KT == 64 ? ~0ull : 0xffffffffull);
    // (most tiles are seen by all rows, which is found out once)
    const bool inner = whole && sees(jb.band, jb.len, sg.pa, sg.pb, k0, KT) == 2;
    uint64_t bad = 0;   // keys whose values were scrubbed
    if (!inner && __builtin_expect(Cp::holds_nonfinite(ks + BYTES, x, found), 0)) bad = Cp::scrub(ks + BYTES, mask);
    const Slot<C> then(a, next);
    if (x + 1 < x1) copy(x + 1, then);
    next = place(x + 2);
    auto see = [&](int r) __attribute__((always_inline)) {
      const Sight sight(jb.band, sg.p, sg.jhi, k0);
      return sight.see(r) && (there >> (4 * (lane >> 5)) >> r & 1);
    };
    if constexpr (PIPED) {
      // keys of the first 32, then in turn: values of a step while its scores are
      // worked out, keys of the next one while its weights are
      u32x4 kf[L::KS];
      read_keys(kf, lds_addr(ks));
#pragma unroll
      for (int rb = 0; rb < KT; rb += 32) {
        const int what = inner ? 2 : sees(jb.band, jb.len, sg.wa, sg.wb, k0 + rb, 32);
        u32x2 vf[4 * L::DB];
        read_values(vf, lds_addr(ks) + BYTES + rb * L::PITCH);
        __builtin_amdgcn_sched_barrier(0);
        f32x16 s = {};
#pragma unroll
        for (int i = 0; i < L::KS; ++i) mma_chunk<T>(s, kf[i], q[i]);
        __builtin_amdgcn_sched_barrier(0);
        if (rb + 32 < KT) read_keys(kf, lds_addr(ks) + (rb + 32) * L::PITCH);
        __builtin_amdgcn_sched_barrier(0);
        if (!what) continue;
        if (!inner) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!see(rb + 8 * (i >> 2) + (i & 3))) s[i] = neg_inf();
        }
        float mx = neg_inf();
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[i]);
        if (__any(mx * c > st.m + 8.0f)) st.grow(half_max(mx) * c);
        const float m = st.m == neg_inf() ? 0.0f : st.m;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -m));
          sum += s[i];
        }
        st.l += sum;
        // (WHOLE: the first 8 bits and what they leave; e4m3 numbers have no infinities that need both above zero)
        f32x16 most = s;
        if constexpr (WHOLE) {
#pragma unroll
          for (int i = 0; i < 16; ++i) most[i] = __uint_as_float(__float_as_uint(s[i]) & 0xffff0000u);
          s -= most;
        }
        const RowsB<T> w(most), rest(s);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int b = 0; b < L::DB; ++b) {
            const u32x2 lo = vf[4 * b + 2 * h], hi = vf[4 * b + 2 * h + 1];
            mma_chunk<T>(st.o[b], u32x4{lo[0], lo[1], hi[0], hi[1]}, w.v[h]);
            if constexpr (WHOLE) mma_chunk<T>(st.o[b], u32x4{lo[0], lo[1], hi[0], hi[1]}, rest.v[h]);
          }
      }
    } else {
      auto step = [&](auto rb) __attribute__((always_inline)) {
        constexpr int RB = decltype(rb)::value;
        const int what = inner ? 2 : sees(jb.band, jb.len, sg.wa, sg.wb, k0 + RB, 32);
        if (what) softmax_step<T, DP, RB, WHOLE>(st, q, ks, ks + BYTES, c, !inner, see);
      };
      step(std::integral_constant<int, 0>{});
      if constexpr (KT == 64) step(std::integral_constant<int, 32>{});
    }
#pragma unroll 1
    for (; __builtin_expect(bad != 0, 0); bad &= bad - 1)
      restore_key<T, C, DP>(st, hd, here, __builtin_ctzll(bad), a.d, Sight(jb.band, sg.p, sg.jhi, k0));
    if (x + 1 < x1) arrive(x + 1);
    here = then;
    __syncthreads();
  }
  const float l = half_sum(st.l);
  if (jb.part < 0) {
    store_row<T, DP / 32>(out_row<T>(a, row), st.o, 1.0f / l, 0, a.d, row.ok, l == 0.0f);
    return;
  }
  const int64_t to = part_row(a, jb.part, row);
  store_row<float, DP / 32>(a.part + to * a.d, st.o, 1.0f, 0, a.d, row.ok, false);
  if (row.ok && lane < 32) *part_sums(a, to) = f32x2{st.m, l};
}

// 32 rows over an fp32 cache; the waves take turns at the tiles of keys, each through LDS of its
// own, and join their sums at the end.
template <int DP>
__device__ __forceinline__ void narrow(const PrefixArgs& a, const Job& jb, const Row& row, const Sights& sg, int hk,
                                       uint8_t* smem) {
  using L = Tile<float, DP>;
  constexpr int BYTES = kKT * L::PITCH, WAVE = Shapes<float, DP>::WAVE;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const KeyTiles kt(jb.band, jb.len, sg.wa, sg.wb, kKT);
  const int x0 = share(kt.count(), jb.split, jb.splits), x1 = share(kt.count(), jb.split + 1, jb.splits);
  const Heads<float> hd(a, hk);
  u32x4 q[L::KS];
  load_row<float, DP>(q, reinterpret_cast<const float*>(a.q.p) + row.token * a.q.st + row.head * a.q.sh, row.ok, a.d);
  Softmax<DP / 32> st;
  st.init();
  const float c = a.scale * kLog2e;
  uint8_t* ks = smem + wave * WAVE;
  PagedStage<float, DP, 64> stage;
  auto place = [&](int x) __attribute__((always_inline)) {
    Place p{};
    p.at = -1;
    if (x < x1) p = Place(a, jb.table, lane < kKT ? kt.tile(x) * kKT + lane : jb.len, jb.len);
    return p;
  };
  int x = x0 + wave;
  Slot<float> at(a, place(x));
  Place next = place(x + kWaves);
  if (x < x1) stage.load(hd.k, hd.v, at.at, a.d);
  for (; x < x1; x += kWaves) {
    const Slot<float> here = at;
    const uint32_t there = (uint32_t)__ballot(here.at >= 0);
    at = Slot<float>(a, next);
    const int k0 = kt.tile(x) * kKT;
    const int what = there == 0xffffffffu ? sees(jb.band, jb.len, sg.wa, sg.wb, k0, kKT) : 1;
    const bool scrubbed = what == 1 && __any(stage.any_nonfinite());
    if (__builtin_expect(scrubbed, 0)) stage.scrub();
    wave_fence();
    stage.store(ks, ks + BYTES);
    wave_fence();
    if (x + kWaves < x1) stage.load(hd.k, hd.v, at.at, a.d);
    next = place(x + 2 * kWaves);
    const Sight sight(jb.band, sg.p, sg.jhi, k0);
    const uint32_t mine = there >> (4 * (lane >> 5));
    auto see = [&](int r) __attribute__((always_inline)) { return sight.see(r) && (mine >> r & 1); };
    if (what) softmax_step<float, DP, 0>(st, q, ks, ks + BYTES, c, what == 1, see);
    if (__builtin_expect(scrubbed, 0)) restore_nonfinite<float, DP>(st, hd.v, here.at, a.d, sight);
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
  for (int x4 = threadIdx.x; x4 < 32 * (DP / 4); x4 += 64 * kWaves) {
    const int r = x4 / (DP / 4), e = x4 % (DP / 4) * 4;
    const Row out(a, jb, hk, jb.r0 + r);
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
    if (jb.part < 0) {
      *reinterpret_cast<f32x4*>(out_row<float>(a, out) + e) = o * (sum == 0.0f ? 0.0f : 1.0f / sum);
    } else {
      const int64_t to = part_row(a, jb.part, out);
      *reinterpret_cast<f32x4*>(a.part + to * a.d + e) = o;
      if (e == 0) *part_sums(a, to) = f32x2{m, sum};
    }
  }
}

// 16 NR rows over tiles of 32 keys by four waves in turn, for caches of 16 or
// 8 bits. Scores are held transposed (keys x queries) in 16 x 16 tiles: lane l
// has query l % 16 and, of each 16 keys, those from 4 (l / 16) on; a contraction
// over 32 keys then takes its weights as they are, with the keys in the order
//   slot 8 g + j: key 4 g + j (j < 4), 16 + 4 g + j - 4 (j >= 4)   (g = l / 16).
// Keys and values pass through LDS as they lie in the cache; e4m3 numbers are
// widened behind its reads (for the values, the transposing ones) and both
// scales are multiplied into scores and weights, in fp32. 16 bytes of a key are
// its elements of one step of the scores' contraction, or of two for e4m3
// numbers, and the queries' operands have the same order.
//
// With fp32 queries (over e4m3 numbers, which are numbers of bf16) queries and
// weights are three bf16 parts each, which hold all their bits. (A weight times a
// value's power of two below 2^-126 may count as zero.)
//
// Bound by HBM: decoding of 64 sequences of up to 16384 over 16 / 4 heads of 128, e4m3, 803 MB,
// 160 to 166 us (4.8 to 5 TB/s), with fp32 queries 167 (with 32-row tiles and numbers
// widened before LDS 186 and 690), heads of 256 in 300; a token over a window of 2048, 8.3 us.
//
// HP key heads stand beside each other in a workgroup's tiles: two of 64 e4m3
// numbers, which share lines of memory where heads lie behind slots (decoding of 64
// sequences of up to 16384, heads of 64: 149 us one by one, 96 in pairs).
template <typename T, class C, int DP, int NR, int HP>
struct Slim {
  static constexpr bool CODES = std::is_same<C, Code>::value;
  static constexpr int ES = CODES ? 1 : 2, CH = 16 / ES;       // bytes an element, elements a chunk of 16 bytes
  static constexpr int CPH = DP / CH, LK = CPH / 4;            // chunks of a head's key, and of that a lane
  static constexpr int PITCH = HP * DP * ES, CPR = HP * CPH, NY = NR * HP;
  static constexpr int ST = DP / 32, DB = DP / 16;
  static constexpr int NQ = sizeof(T) == 4 ? 3 : 1, NP = sizeof(T) == 4 ? 3 : 2;
  static constexpr int VB = 32 * PITCH, WAVE = 2 * VB + 256 * HP, SUMS = NY * (4 * DB + 2) * 256;
  // 32 fp32 queries of 128 in their three parts are 96 registers (67 and more spilled): they stay in LDS, behind the
  // waves' tiles (6 chunks of 200 tokens over 4096 to 8192, 16 / 4 heads of 128: 186 us for 387).
  static constexpr bool QLDS = NQ == 3 && NY == 2 && DP >= 128;
  static constexpr int QUERIES = QLDS ? NY * NQ * ST * 1024 : 0;
  static constexpr int SMEM = kWaves * WAVE + QUERIES > 2 * SUMS ? kWaves * WAVE + QUERIES : 2 * SUMS;
  static_assert(CPH >= 4, "four chunks a head at least");

  // The row of LDS that a key's values have, and its chunks' order: the 16
  // lanes of a transposing read (8 rows of one chunk, or 4 rows of two), and 8
  // of a write (one chunk of 8 keys), meet different banks.
  static __device__ __forceinline__ int row_of(int key) {
    return CODES ? ((key & 12) << 1) | ((key & 16) >> 2) | (key & 3) : key;
  }
  static __device__ __forceinline__ int swz(int row) {
    if constexpr (CODES) return CPR >= 16 ? row & 15 : CPR == 8 ? row >> 1 & 7 : row >> 2 & 3;
    else return CPR >= 16 ? (row & 7) << 1 : (row >> 1 & 3) << 1;
  }
  static __device__ __forceinline__ int off(int row, int chunk) { return row * PITCH + ((chunk ^ swz(row)) << 4); }

  typedef __attribute__((ext_vector_type(2))) int i32x2;
  typedef __attribute__((address_space(3))) i32x2 lds_i2;
  typedef __attribute__((address_space(3))) s16x4 lds_s4;

  // Values of columns 16 db + l % 16 in the contraction's order.
  static __device__ __forceinline__ bf16x8 columns(const uint8_t* vt, int db) {
    const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
    u32x4 r;
    if constexpr (CODES) {
      const int row = 8 * g + (n >> 1);
      const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2*)(vt + off(row, db) + ((n & 1) << 3)));
      widen<__bf16>((uint32_t)x[0], 1.0f, reinterpret_cast<uint32_t*>(&r));
      widen<__bf16>((uint32_t)x[1], 1.0f, reinterpret_cast<uint32_t*>(&r) + 2);
    } else {
      const int row = 4 * g + (n >> 2), c = 2 * db + (n >> 1 & 1), at = (n & 1) << 3;
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(vt + off(row, c) + at));
      const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(vt + off(row + 16, c) + at));
      const u32x2 lo = __builtin_bit_cast(u32x2, x), hi = __builtin_bit_cast(u32x2, y);
      r = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
    return __builtin_bit_cast(bf16x8, r);
  }
  // A chunk of a key as the operand of its step h.
  static __device__ __forceinline__ bf16x8 rows(const u32x4& k, int h) {
    if constexpr (CODES) {
      uint32_t w[4];
      widen<__bf16>(k[2 * h], 1.0f, w);
      widen<__bf16>(k[2 * h + 1], 1.0f, w + 2);
      return __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
    } else {
      return __builtin_bit_cast(bf16x8, k);
    }
  }
  // The first element of a query's part in step s.
  static __device__ __forceinline__ int query_at(int s) {
    const int g = (threadIdx.x & 63) >> 4;
    return CODES ? 16 * (g + 4 * (s >> 1)) + 8 * (s & 1) : 32 * s + 8 * g;
  }

  // Eight numbers in N parts of bf16 each, whose sum is the number to 2^-16 (two) or 2^-24 (three): of a query's
  // elements the first 8 bits of what is left each time, of WEIGHTS the bf16 next below it, so that all parts of one
  // above zero are above zero, and an infinity times them stays one. The last part is rounded.
  template <int N, bool WEIGHTS>
  static __device__ __forceinline__ void parts(const float (&x)[8], bf16x8 (&to)[N]) {
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float a = rest[2 * i], b = rest[2 * i + 1];
        if (k + 1 < N) {
          a = __uint_as_float((WEIGHTS ? __builtin_elementwise_sub_sat(__float_as_uint(a), 1u) : __float_as_uint(a)) & 0xffff0000u);
          b = __uint_as_float((WEIGHTS ? __builtin_elementwise_sub_sat(__float_as_uint(b), 1u) : __float_as_uint(b)) & 0xffff0000u);
          rest[2 * i] -= a;
          rest[2 * i + 1] -= b;
          w[i] = (__float_as_uint(a) >> 16) | __float_as_uint(b);
        } else {
          w[i] = pack_bf16(a, b);
        }
      }
      to[k] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
    }
  }

  struct Sums {
    f32x4 o[NY][DB];
    float m[NY], l[NY];
    __device__ __forceinline__ void put(float* to) const {
      to += threadIdx.x & 63;
#pragma unroll
      for (int y = 0; y < NY; ++y) {
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) to[((y * DB + b) * 4 + i) * 64] = o[y][b][i];
        to[(NY * DB * 4 + 2 * y) * 64] = m[y];
        to[(NY * DB * 4 + 2 * y + 1) * 64] = l[y];
      }
    }
    __device__ __forceinline__ void join(const float* from) {
      from += threadIdx.x & 63;
#pragma unroll
      for (int y = 0; y < NY; ++y) {
        const float m2 = from[(NY * DB * 4 + 2 * y) * 64], up = fmaxf(m[y], m2);
        const float f = m[y] == up ? 1.0f : __builtin_amdgcn_exp2f(m[y] - up);
        const float g = m2 == up ? 1.0f : __builtin_amdgcn_exp2f(m2 - up);
        m[y] = up;
        l[y] = l[y] * f + from[(NY * DB * 4 + 2 * y + 1) * 64] * g;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[y][b][i] = o[y][b][i] * f + from[((y * DB + b) * 4 + i) * 64] * g;
      }
    }
  };

  // A tile on its way to LDS, whole rows by neighbouring lanes: memory gives
  // lines of 128 bytes, and parts of them by separate loads at three quarters of
  // the rate (decoding of 64 sequences of up to 16384, heads of 128: 233 us where the
  // lanes of a key took 64 bytes of it a load). Lanes know where key l % 32 lies.
  struct Tile32 {
    static constexpr int N = CPR / 2, STEP = 64 / CPR;
    u32x4 k[N], v[N];
    int scale[HP];                 // bytes of the lane's key (lanes 0 to 31) or value, of each head
    __device__ __forceinline__ void load(const PrefixArgs& a, const Heads<C>& h, const Slot<C>& s) {
      const int lane = threadIdx.x & 63, c = lane % CPR, e = c % CPH * CH;
      const int64_t more = e + (HP > 1 ? c / CPH * a.c.sh : 0);
      if constexpr (CODES) {
#pragma unroll
        for (int y = 0; y < HP; ++y) scale[y] = load_byte(s.at >= 0, (lane < 32 ? h.ks : h.vs) + s.scale + y * a.cs.sh);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int64_t o = shfl64(s.at, lane / CPR + i * STEP);
        const bool ok = o >= 0 && e < a.d;
        k[i] = load16(ok, h.k + o + more);
        v[i] = load16(ok, h.v + o + more);
      }
    }
    __device__ __forceinline__ bool any_nonfinite() const {
      bool bad = false;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (CODES) {
          uint32_t x = 0;
#pragma unroll
          for (int w = 0; w < 4; ++w) x |= (v[i][w] & 0x7f7f7f7fu) + 0x01010101u;
          bad |= (x & 0x80808080u) != 0;
        } else {
          bad |= nonfinite<__bf16>(v[i]);
        }
      }
      return bad;
    }
    __device__ __forceinline__ void scrub() {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if constexpr (CODES) {
            const uint32_t x = v[i][w], nan = ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
            v[i][w] = x & ~(nan | (nan - (nan >> 7)));
          } else {
            v[i][w] = finite_or_zero<__bf16>(v[i][w]);
          }
        }
    }
    __device__ __forceinline__ void put(uint8_t* kt) const {
      const int lane = threadIdx.x & 63, chunk = lane % CPR;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = lane / CPR + i * STEP;
        *reinterpret_cast<u32x4*>(kt + off(row, chunk)) = k[i];
        *reinterpret_cast<u32x4*>(kt + VB + off(row_of(row), chunk)) = v[i];
      }
      if constexpr (CODES) {   // the powers of two of a key's scores and of its weights
#pragma unroll
        for (int y = 0; y < HP; ++y)
          reinterpret_cast<float*>(kt + 2 * VB)[64 * y + 2 * (lane & 31) + (lane >> 5)] = scale_of(scale[y]);
      }
    }
  };

  static __device__ __forceinline__ void run(const PrefixArgs& a, const Job& jb, const Row (&row)[NY], const Sights (&sg)[NR],
                                             int hk, uint8_t* smem) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
    const int wa = sg[0].wa, wb = sg[0].wb;
    const KeyTiles kt(jb.band, jb.len, wa, wb, 32);
    const int x0 = share(kt.count(), jb.split, jb.splits), x1 = share(kt.count(), jb.split + 1, jb.splits);
    const Heads<C> hd(a, hk);
    const float c = a.scale * kLog2e;
    uint8_t *ks = smem + wave * WAVE, *vt = ks + VB;
    auto place = [&](int x) __attribute__((always_inline)) {   // of key lane % 32
      Place p{};
      p.at = -1;
      if (x < x1) p = Place(a, jb.table, kt.tile(x) * 32 + (lane & 31), jb.len);
      return p;
    };
    int x = x0 + wave;
    const Place at0 = place(x);
    Place next = place(x + kWaves);
    bf16x8 q[QLDS ? 1 : NY][NQ][QLDS ? 1 : ST];
    u32x4* const qs = reinterpret_cast<u32x4*>(smem + kWaves * WAVE) + lane;
    static_assert(!QLDS || ST % kWaves == 0, "steps of the queries a wave");
#pragma unroll
    for (int y = 0; y < NY; ++y)
#pragma unroll
      for (int s0 = 0; s0 < (QLDS ? ST / kWaves : ST); ++s0) {
        const int s = QLDS ? s0 * kWaves + wave : s0, e = query_at(s);
        const T* at = reinterpret_cast<const T*>(a.q.p) + row[y].token * a.q.st + row[y].head * a.q.sh + e;
        const bool ok = row[y].ok && e < a.d;
        if constexpr (sizeof(T) == 2) {
          q[y][0][s0] = __builtin_bit_cast(bf16x8, load16(ok, at));
        } else {
          const f32x4 lo = __builtin_bit_cast(f32x4, load16(ok, at)), hi = __builtin_bit_cast(f32x4, load16(ok, at + 4));
          const float f[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          bf16x8 p[NQ];
          parts<NQ, false>(f, p);
#pragma unroll
          for (int k = 0; k < NQ; ++k) {
            if constexpr (QLDS) qs[((y * NQ + k) * ST + s) * 64] = __builtin_bit_cast(u32x4, p[k]);
            else q[y][k][s0] = p[k];
          }
        }
      }
    Slot<C> here(a, at0);
    Tile32 t;
    if (x < x1) t.load(a, hd, here);
    if constexpr (QLDS) __syncthreads();
    else arrived(q);
    Sums st;
#pragma unroll
    for (int y = 0; y < NY; ++y) {
#pragma unroll
      for (int b = 0; b < DB; ++b) st.o[y][b] = f32x4{};
      st.m[y] = neg_inf();
      st.l[y] = 0.0f;
    }
    for (; x < x1; x += kWaves) {
      const uint32_t there = (uint32_t)__ballot(here.at >= 0);
      const int k0 = kt.tile(x) * 32;
      const int what = there == 0xffffffffu ? sees(jb.band, jb.len, wa, wb, k0, 32) : 1;
      const bool scrubbed = what == 1 && __any(t.any_nonfinite());
      if (__builtin_expect(scrubbed, 0)) t.scrub();
      wave_fence();
      t.put(ks);
      wave_fence();
      // the next tile
      const Slot<C> old = here;
      here = Slot<C>(a, next);
      if (x + kWaves < x1) t.load(a, hd, here);
      next = place(x + 2 * kWaves);
      // scores
      f32x4 s[NY][2];
#pragma unroll
      for (int y = 0; y < NY; ++y) s[y][0] = s[y][1] = f32x4{};
      if constexpr (QLDS) {
#pragma unroll
        for (int i = 0; i < LK; ++i) {
          u32x4 chunk[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) chunk[u] = *reinterpret_cast<const u32x4*>(ks + off(16 * u + n, g + 4 * i));
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const bf16x8 kr[2] = {rows(chunk[0], h), rows(chunk[1], h)};
#pragma unroll
            for (int y = 0; y < NY; ++y)
#pragma unroll
              for (int p = NQ - 1; p >= 0; --p) {
                const bf16x8 part = __builtin_bit_cast(bf16x8, qs[((y * NQ + p) * ST + 2 * i + h) * 64]);
#pragma unroll
                for (int u = 0; u < 2; ++u) s[y][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr[u], part, s[y][u], 0, 0, 0);
              }
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < LK * HP; ++i)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int hp = i / LK, ih = i % LK;
            const u32x4 chunk = *reinterpret_cast<const u32x4*>(ks + off(16 * u + n, hp * CPH + g + 4 * ih));
#pragma unroll
            for (int h = 0; h < (CODES ? 2 : 1); ++h) {
              const bf16x8 kr = rows(chunk, h);
#pragma unroll
              for (int y = hp * NR; y < (hp + 1) * NR; ++y)
#pragma unroll
                for (int p = NQ - 1; p >= 0; --p)
                  s[y][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr, q[y][p][CODES ? 2 * ih + h : ih], s[y][u], 0, 0, 0);
            }
          }
      }
      float kf[HP][2][4], vf[HP][2][4];
#pragma unroll
      for (int hp = 0; hp < HP; ++hp)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if constexpr (CODES) {
            const f32x4* f = reinterpret_cast<const f32x4*>(ks + 2 * VB + 256 * hp + (16 * u + 4 * g) * 8);
            const f32x4 lo = f[0], hi = f[1];
            kf[hp][u][0] = lo[0], vf[hp][u][0] = lo[1], kf[hp][u][1] = lo[2], vf[hp][u][1] = lo[3];
            kf[hp][u][2] = hi[0], vf[hp][u][2] = hi[1], kf[hp][u][3] = hi[2], vf[hp][u][3] = hi[3];
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) kf[hp][u][i] = 1.0f, vf[hp][u][i] = 1.0f;
          }
        }
      if (what) {
        bf16x8 w[NY][NP];
#pragma unroll
        for (int y = 0; y < NY; ++y) {
          float z[2][4], mx = neg_inf();
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) z[u][i] = s[y][u][i] * kf[y / NR][u][i] * c;   // (the score first: 2^119 c may be past fp32)
          if (what == 1) {
            const int jlo = sg[y % NR].p - jb.band.win + 1, jhi = sg[y % NR].jhi, sink = min(jb.band.sinks, jhi + 1);
            const int lo = jhi < jlo ? 1 << 30 : jlo;
            const uint32_t span = (uint32_t)max(jhi - jlo, 0);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int r = 16 * u + 4 * g + i, j = k0 + r;
                if (!((((uint32_t)(j - lo) <= span) | (j < sink)) && (there >> r & 1))) z[u][i] = neg_inf();
              }
          }
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, z[u][i]);
          // the maximum follows late, as Softmax's
          if (__any(mx > st.m[y] + 8.0f)) {
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const bool up = mx > st.m[y] + 8.0f;
            const float f = up ? __builtin_amdgcn_exp2f(st.m[y] - mx) : 1.0f;
            st.m[y] = up ? mx : st.m[y];
            st.l[y] *= f;
#pragma unroll
            for (int b = 0; b < DB; ++b) st.o[y][b] *= f;
          }
          const float m = st.m[y] == neg_inf() ? 0.0f : st.m[y];
          float p[8];
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float e = __builtin_amdgcn_exp2f(z[u][i] - m);
              st.l[y] += e;
              p[4 * u + i] = CODES ? (what == 1 && e == 0.0f ? 0.0f : e * vf[y / NR][u][i]) : e;
            }
          parts<NP, true>(p, w[y]);
        }
#pragma unroll
        for (int b = 0; b < DB * HP; ++b) {
          const bf16x8 vc = columns(vt, b);
#pragma unroll
          for (int y = b / DB * NR; y < (b / DB + 1) * NR; ++y)
#pragma unroll
            for (int p = NP - 1; p >= 0; --p)
              st.o[y][b % DB] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vc, w[y][p], st.o[y][b % DB], 0, 0, 0);
        }
      }
      if (__builtin_expect(scrubbed, 0)) {
#pragma unroll 1
        for (int r = 0; r < 32; ++r) {
          const int64_t o = shfl64(old.at, r);
          if (o < 0) continue;
          restore(st, a, hd, jb, sg, o, k0 + r);
        }
      }
    }
#pragma unroll
    for (int y = 0; y < NY; ++y) {
      st.l[y] += __shfl_xor(st.l[y], 16, 64);
      st.l[y] += __shfl_xor(st.l[y], 32, 64);
    }
    // the waves' sums in a fixed order: (0 + 2) + (1 + 3)
    float* sums = reinterpret_cast<float*>(smem);
    __syncthreads();
    if (wave >= 2) st.put(sums + (wave - 2) * (SUMS / 4));
    __syncthreads();
    if (wave < 2) st.join(sums + wave * (SUMS / 4));
    __syncthreads();
    if (wave == 1) st.put(sums);
    __syncthreads();
    if (wave) return;
    st.join(sums);
#pragma unroll
    for (int y = 0; y < NY; ++y) {
      if (!row[y].ok) continue;
      const int64_t to = part_row(a, max(jb.part, 0), row[y]);
      const float inv = st.l[y] == 0.0f ? 0.0f : 1.0f / st.l[y];
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const int e = 16 * b + 4 * g;
        if (e >= a.d) continue;
        const f32x4 o = st.o[y][b];
        if (jb.part >= 0) {
          *reinterpret_cast<f32x4*>(a.part + to * a.d + e) = o;
        } else if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<u32x2*>(out_row<T>(a, row[y]) + e) = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
        } else {
          *reinterpret_cast<f32x4*>(out_row<T>(a, row[y]) + e) = o * inv;
        }
      }
      if (jb.part >= 0 && g == 0) *part_sums(a, to) = f32x2{st.m[y], st.l[y]};
    }
  }

  // (as add_nonfinite()) key j at offset o, whose values were scrubbed
  static __device__ __forceinline__ void restore(Sums& st, const PrefixArgs& a, const Heads<C>& hd, const Job& jb,
                                                 const Sights (&sg)[NR], int64_t o, int j) {
    int g = (threadIdx.x & 63) >> 4;
    asm volatile("" : "+v"(g));
#pragma unroll
    for (int y = 0; y < NY; ++y) {
      const int jlo = sg[y % NR].p - jb.band.win + 1, jhi = sg[y % NR].jhi;
      if (!((j >= jlo && j <= jhi) || j < min(jb.band.sinks, jhi + 1))) continue;
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = 16 * b + 4 * g + i;
          if (e >= a.d) continue;
          const int64_t at = o + y / NR * a.c.sh + e;
          float x;
          if constexpr (CODES) x = (hd.v[at] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.0f;
          else x = (float)hd.v[at];
          if (!(fabsf(x) < __builtin_inff())) st.o[y][b][i] += x;
        }
    }
  }
};

// The shapes of a role's workgroups: 16 or 32 rows whose waves take turns at
// the keys (16 of one key head or of two), or 128.
enum Shape { kNone, kRows16, kRows32, kRows128, kPairs16 };

template <typename T, class C, int DP, int SHAPE>
struct Role {
  static constexpr bool PAGED32 = sizeof(T) == 4 && !std::is_same<C, Code>::value;   // an fp32 cache
  static constexpr int R = SHAPE == kRows128 ? 128 : SHAPE == kRows16 || SHAPE == kPairs16 ? 16 : 32;
  static constexpr int NR = R / 16;
  static constexpr int HP = SHAPE == kPairs16 ? 2 : 1;   // key heads a workgroup
  static constexpr int smem() {
    if constexpr (SHAPE == kNone) return 0;
    else if constexpr (SHAPE == kRows128) return Shapes<T, DP>::WIDE;
    else if constexpr (PAGED32) return kWaves * Shapes<T, DP>::WAVE;
    else return Slim<T, C, DP, NR, HP>::SMEM;
  }
};

// Workgroups a CU that the registers are to allow.
template <typename T, class C, int DP, int PS, int OS>
constexpr int occupancy() {
  constexpr bool few = PS != kRows128 && OS != kRows128 && !Role<T, C, DP, OS>::PAGED32;   // rows
  return DP <= 128 && (sizeof(T) == 2 || few) ? 2 : 1;
}

// LDS that all shapes have: flags of the wide one, positions of the waves' rows, offsets.
struct Words {
  uint32_t mask[2];
  int found, sights[2 * kWaves], offsets[kOffsets + 1];
};

template <typename T, class C, int DP, int SHAPE, bool GROUP, bool WHOLE>
__device__ __forceinline__ void work(const PrefixArgs& a, const Offsets& off, const Job& jb, int p0, int hk, uint8_t* smem,
                                     Words& words) {
  using Ro = Role<T, C, DP, SHAPE>;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if constexpr (SHAPE == kRows128 || Ro::PAGED32) {
    const int wr = jb.r0 + (SHAPE == kRows128 ? 32 * wave : 0);
    const Row row(a, jb, hk, wr + (lane & 31));
    Sights sg;
    if constexpr (GROUP) {
      sg = group_sights<32>(a, off, jb, row);
      if (SHAPE == kRows128) join_sights(sg, words.sights);
    } else {
      sg = own_sights(a, jb, p0, row, wr, Ro::R);
    }
    if constexpr (SHAPE == kRows128) wide<T, C, DP, WHOLE>(a, jb, row, sg, hk, smem, words.mask, &words.found);
    else narrow<DP>(a, jb, row, sg, hk, smem);
  } else {
    constexpr int NR = Ro::NR, HP = Ro::HP;
    Row row[NR * HP];
    Sights sg[NR];
#pragma unroll
    for (int y = 0; y < NR * HP; ++y) {
      row[y] = Row(a, jb, hk + y / NR, jb.r0 + 16 * (y % NR) + (lane & 15));
      if (y >= NR) continue;
      if constexpr (GROUP) sg[y] = group_sights<16>(a, off, jb, row[y]);
      else sg[y] = own_sights(a, jb, p0, row[y], jb.r0, Ro::R);
    }
    if constexpr (GROUP)
      for (int y = 1; y < NR; ++y)
        if (sg[y].wa <= sg[y].wb) {
          sg[0].wa = min(sg[0].wa, sg[y].wa);
          sg[0].wb = max(sg[0].wb, sg[y].wb);
        }
    Slim<T, C, DP, NR, HP>::run(a, jb, row, sg, hk, smem);
  }
}

// Job j of a role whose workgroups have HP key heads: part u of the keys of a
// row tile, and the first head. Where a slot's heads share lines of memory (128
// bytes), those of one part are 8 jobs apart, so that one XCD works on them at about
// the same time and reads a line once: decoding of 64 sequences of up to 16384, 4 heads of
// 80 in 8 bits, 131 us for 189, of 96 181 for 212; 32 x 10 tokens over up to 6001, 8 heads of 64,
// 49 for 65. Heads of whole lines are neighbours: 64 sequences, heads of 128, 171 us for 175.
template <class C, int HP>
__device__ __forceinline__ void place_of_job(const PrefixArgs& a, int j, int& u, int& head) {
  const int n = a.Hkv / HP;
  constexpr uint32_t BYTES = HP * sizeof(typename std::conditional<std::is_same<C, Code>::value, uint8_t, C>::type);
  if ((uint32_t)a.c.sh * BYTES & 127) {
    const int i = j >> 3, q = i / n;
    u = q << 3 | (j & 7);
    head = (i - q * n) * HP;
  } else {
    u = j / n;
    head = (j - u * n) * HP;
  }
}

// PS, OS: the shapes of the rows over prefixes (or kNone) and over a sequence's own keys.
template <typename T, class C, int DP, int PS, int OS>
__global__ __launch_bounds__(64 * kWaves, (occupancy<T, C, DP, PS, OS>())) void k_prefix(const PrefixArgs a) {
  using P = Role<T, C, DP, PS>;
  using O = Role<T, C, DP, OS>;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[P::smem() > O::smem() ? P::smem() : O::smem()];
  __shared__ Words words;
  const Offsets off(a, words.offsets);
  Seq s;
  Job jb;
  jb.band = Band{a.win, 0, a.sinks};
  if constexpr (PS != kNone) {
    if ((int)blockIdx.x < a.pjobs) {
      int u, head;
      place_of_job<C, P::HP>(a, (int)blockIdx.x, u, head);
      const int t = u / a.psplits;
      if (!find_tile<true>(a, off, t, P::R, s, jb.r0)) return;
      jb.table = a.ptable + (int64_t)s.b * a.p_pages;
      jb.t0 = s.t0;
      jb.rows = s.rows;
      jb.len = s.len;
      jb.split = jb.part = u - t * a.psplits;
      jb.splits = a.psplits;
      work<T, C, DP, PS, true, OS != kRows128>(a, off, jb, 0, head, smem, words);
      return;
    }
  }
  int u, head;
  place_of_job<C, O::HP>(a, (int)blockIdx.x - (PS != kNone ? a.pjobs : 0), u, head);
  const int t = u / a.splits;
  if (!find_tile<false>(a, off, t, O::R, s, jb.r0)) return;
  jb.table = a.table + (int64_t)s.b * a.max_pages;
  jb.t0 = s.t0;
  jb.rows = s.rows;
  jb.len = s.len;
  jb.split = u - t * a.splits;
  jb.splits = a.splits;
  jb.part = PS != kNone || a.splits > 1 ? a.psplits + jb.split : -1;
  if constexpr (PS != kNone) {
    if (a.sinks) {   // those that its group's prefix leaves
      const int g = group_of(a, s.b);
      if (g >= 0) jb.band.sinks = max(0, a.sinks - clampi(a.plen[g], 0, a.p_pages * a.page));
    }
  }
  work<T, C, DP, OS, false, false>(a, off, jb, s.p0, head, smem, words);
}

// The parts of each (token, head), joined in a fixed order: those over its
// group's prefix, if it has one, and those over its own keys. Rows past the
// last sequence are left as they were. A row has G lanes of four elements,
// times W: the W-th parts from w on are added by lanes of their own, four
// loads in flight, and the W sums through LDS.
template <typename T>
__global__ __launch_bounds__(256) void k_prefix_join(const PrefixArgs a, int G, int W) {
  __shared__ f32x4 so[256];
  __shared__ f32x2 sm[256];
  const int lg = threadIdx.x & (G - 1), w = threadIdx.x / G & (W - 1);
  const int64_t rows = (int64_t)a.T * a.H, r = (int64_t)blockIdx.x * (256 / (G * W)) + threadIdx.x / (G * W);
  const bool there = r < rows;
  const int token = (int)((uint32_t)r / (uint32_t)a.H), head = (int)((uint32_t)r % (uint32_t)a.H), e = lg * 4;   // (rows < 2^29)
  const int all = a.psplits + a.splits;
  f32x2 x[4];
  f32x4 y[4];
  // (parts of a prefix that the row does not have are read, but not added: nothing waits to know)
  auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = s0 + i * W;
      const bool ok = there && s < all;
      x[i] = ok ? *part_sums(a, rows * s + r) : f32x2{neg_inf(), 0.0f};
      y[i] = ok && e < a.d ? *reinterpret_cast<const f32x4*>(a.part + (rows * s + r) * a.d + e) : f32x4{};
    }
  };
  load(w);
  const bool ok = there && token >= clampi(a.cu[0], 0, a.T) && token < clampi(a.cu[a.B], 0, a.T);
  int first = a.psplits;
  if (a.P) {
    auto at = [&](int g) { return clampi(a.cu[clampi(a.cu_seq[g], 0, a.B)], 0, a.T); };
    if (token >= at(0) && token < at(a.P)) first = 0;
  }
  float m = neg_inf(), sum = 0.0f;
  f32x4 o = {};
  auto add = [&](f32x2 x, f32x4 y) __attribute__((always_inline)) {
    const float up = fmaxf(m, x[0]), top = up == neg_inf() ? 0.0f : up;   // (scores of NaN alone leave a NaN of a sum, and no maximum)
    const float f = __builtin_amdgcn_exp2f(m - top), g = __builtin_amdgcn_exp2f(x[0] - top);
    sum = sum * f + x[1] * g;
    o = o * f + y * g;
    m = up;
  };
  for (int s0 = w;;) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (ok && s0 + i * W >= first && s0 + i * W < all) add(x[i], y[i]);
    s0 += 4 * W;
    if (s0 >= all) break;
    load(s0);
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

int shape_rows(int shape) { return shape == kRows128 ? 128 : shape == kRows16 || shape == kPairs16 ? 16 : 32; }
// Workgroups: row tiles of n sequences or groups, in parts, by eights, times (pairs of) key heads.
int64_t row_jobs(const PrefixArgs& a, int shape, int n, int splits) {
  const int64_t tiles = (int64_t)a.T * a.G / shape_rows(shape) + n;
  return (tiles * splits + 7) / 8 * 8 * (shape == kPairs16 ? a.Hkv / 2 : a.Hkv);
}

template <typename T, class C, int DP, int PS, int OS>
void start(const PrefixArgs& a, hipStream_t s) {
  const unsigned jobs = (unsigned)(a.pjobs + row_jobs(a, OS, a.B, a.splits));
  k_prefix<T, C, DP, PS, OS><<<jobs, 64 * kWaves, 0, s>>>(a);
}

template <typename T, class C, int DP>
hipError_t run(const PrefixArgs& a, hipStream_t s) {
  constexpr bool CODES = std::is_same<C, Code>::value, FP32 = sizeof(T) == 4 && !CODES;
  if constexpr (FP32 && DP == 256) {                // a wave's own tile would not fit
    start<T, C, DP, kRows128, kRows128>(a, s);
  } else {
    constexpr bool PAIRS = CODES && DP == 64, PARTS = CODES && sizeof(T) == 4;
    constexpr int k16 = FP32 ? kRows32 : kRows16;   // (an fp32 cache has one shape of few rows)
    constexpr int p16 = PAIRS ? kPairs16 : k16;
    // (fp32 queries over e4m3 numbers, whose bf16 products are those of the 32 rows: chunks of 200 tokens over 4096 to
    // 8192, 16 / 4 heads of 128, 186 us, and 128 rows with fp32 products 611; 12 of 160 behind 8192 keys 322 and 1094)
    constexpr int kMany = PARTS ? kRows32 : kRows128;
    if (!a.P) {
      if constexpr (CODES) {                        // (the other kinds have their own entry point)
        if (a.shape == kRows128) start<T, C, DP, kNone, kMany>(a, s);
        else if (a.shape == kRows32) start<T, C, DP, kNone, kRows32>(a, s);
        else if (a.shape == kRows16) start<T, C, DP, kNone, kRows16>(a, s);
        else start<T, C, DP, kNone, p16>(a, s);
      }
    } else if (a.shape == kRows128) {
      start<T, C, DP, kMany, kMany>(a, s);
    } else if (a.shape == kRows32 && !FP32) {
      start<T, C, DP, kMany, kRows32>(a, s);
    } else if (a.pshape == kRows128) {
      if (a.shape == kPairs16) start<T, C, DP, kMany, p16>(a, s);
      else start<T, C, DP, kMany, k16>(a, s);
    } else if (a.shape == kPairs16) {
      start<T, C, DP, kRows32, p16>(a, s);
    } else {
      start<T, C, DP, kRows32, k16>(a, s);
    }
  }
  if (a.P || a.splits > 1) {
    int G = 1, W = 1;
    while (G * 4 < a.d) G *= 2;
    const int64_t rows = (int64_t)a.T * a.H;
    while (G * W < 256 && 4 * W < a.psplits + a.splits && rows * G * W < 1024 * 256) W *= 2;
    const int per = 256 / (G * W);
    k_prefix_join<T><<<(unsigned)((rows + per - 1) / per), 256, 0, s>>>(a, G, W);
  }
  return hipGetLastError();
}

template <typename T, class C>
hipError_t run(const PrefixArgs& a, hipStream_t s) {
  return a.d <= 64 ? run<T, C, 64>(a, s) : a.d <= 128 ? run<T, C, 128>(a, s) : run<T, C, 256>(a, s);
}

}  // namespace
}  // namespace lact
