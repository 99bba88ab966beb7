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
#include <algorithm>
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
  __device__ __forceinline__ Row(const PrefixArgs& a, const Job& j, int hk, int r) {
    ok = r < j.rows;
    const int rc = ok ? r : j.rows - 1, t = rc / a.G;
    token = j.t0 + t;
    head = hk * a.G + rc - t * a.G;
  }
};

// The groups of a call, as find_rows() takes them.
struct Groups {
  const PrefixArgs& a;
  __device__ __forceinline__ int count() const { return a.P; }
  __device__ __forceinline__ int first(int g) const { return clampi(a.cu[clampi(a.cu_seq[g], 0, a.B)], 0, a.T); }
  __device__ __forceinline__ int len(int g) const { return clampi(a.plen[g], 0, a.p_pages * a.page); }
};

// The position of a token among its sequence's own keys (< 0 for one that its
// sequence does not hold). All 64 lanes take part. Up to 64 sequences stand a
// lane each.
__device__ __forceinline__ int own_position(const PrefixArgs& a, int token) {
  int b = 0, t1, len;
  if (a.B <= 64) {
    const int mine = min((int)(threadIdx.x & 63), a.B - 1), t0 = clampi(a.cu[mine], 0, a.T);
    b = -1;
    for (int j = 0; j < a.B; ++j) b += __builtin_amdgcn_readlane(t0, j) <= token;
    b = max(b, 0);
    t1 = __shfl(clampi(a.cu[mine + 1], 0, a.T), b, 64);
    len = __shfl(seq_len(a, mine), b, 64);
  } else {
    int hi = a.B - 1;
    while (b < hi) {
      const int mid = (b + hi + 1) >> 1;
      if (clampi(a.cu[mid], 0, a.T) <= token) b = mid;
      else hi = mid - 1;
    }
    t1 = clampi(a.cu[b + 1], 0, a.T);
    len = seq_len(a, b);
  }
  return len - (t1 - token);
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

// Where a key lies: offsets of its vectors and of its scales, `at` < 0 if there is none.
template <class C>
struct Slot {
  int64_t at;
  template <class Args>
  __device__ __forceinline__ void find(const Args& a, const int32_t* table, int key, int len) {
    at = slot_of(a, table, key, len);
  }
};
template <>
struct Slot<Code> {
  int64_t at, scale;
  template <class Args>
  __device__ __forceinline__ void find(const Args& a, const int32_t* table, int key, int len) {
    int pg, i;
    at = -1;
    if (!find_slot(a, table, key, len, pg, i)) return;
    at = pg * a.c.sb + i * a.c.st;
    scale = pg * a.cs.sb + i * a.cs.st;
  }
};

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

// A tile of KT keys and values on its way from memory to LDS through the
// registers of NT threads; what goes to LDS is T. Each wave's lanes know where
// the tile's keys lie (lane = key).
template <typename T, class C, int DP, int KT, int NT>
struct Stage : PagedStage<T, DP, NT> {
  using Base = PagedStage<T, DP, NT>;
  static_assert(KT == kKT, "tiles through registers");
  __device__ __forceinline__ void load(const Heads<T>& h, const Slot<T>& s, int d) { Base::load(h.k, h.v, s.at, d); }
  __device__ __forceinline__ void put(uint8_t* kt, uint8_t* vt, bool scrubbed) {
    if (__builtin_expect(scrubbed, 0)) Base::scrub();
    Base::store(kt, vt);
  }
};
template <typename T, int DP, int KT, int NT>
struct Stage<T, Code, DP, KT, NT> {
  using L = Tile<T, DP>;
  static constexpr int CPR = DP / 16;   // 16 numbers a load
  static constexpr int ALL = KT * CPR, N = ALL < NT ? 1 : ALL / NT, STEP = NT / CPR;
  static_assert(ALL < NT || ALL % NT == 0, "tile split");
  u32x4 k[N], v[N];
  int kb, vb;   // scales of the lane's key
  static __device__ __forceinline__ int row(int i) { return threadIdx.x % NT / CPR + i * STEP; }
  __device__ __forceinline__ void load(const Heads<Code>& h, const Slot<Code>& s, int d) {
    const int e = threadIdx.x % CPR * 16;
    kb = vb = 127;
    if (s.at >= 0) {
      kb = h.ks[s.scale];
      vb = h.vs[s.scale];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t o = shfl64(s.at, row(i) & 63);
      const bool ok = o >= 0 && e < d && (ALL >= NT || row(i) < KT);
      k[i] = ok ? *reinterpret_cast<const u32x4*>(h.k + o + e) : u32x4{};
      v[i] = ok ? *reinterpret_cast<const u32x4*>(h.v + o + e) : u32x4{};
    }
  }
  // a NaN among the values, or a scale that can make an infinity of one
  __device__ __forceinline__ bool any_nonfinite() const {
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) bad |= (v[i][x] & 0x7f7f7f7fu) + 0x01010101u;
    return (bad & 0x80808080u) || vb > kMaxExp + 127;
  }
  __device__ __forceinline__ void put(uint8_t* kt, uint8_t* vt, bool scrubbed) {
    constexpr int W = 4 * (int)sizeof(T);   // words of 16 elements
    const int c = threadIdx.x % CPR * (W / 4);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = row(i);
      const float ks = scale_of(__shfl(kb, r & 63, 64)), vs = scale_of(__shfl(vb, r & 63, 64));
      if (ALL < NT && r >= KT) continue;
      uint32_t w[W];
#pragma unroll
      for (int x = 0; x < 4; ++x) widen<T>(k[i][x], ks, w + x * W / 4);
#pragma unroll
      for (int x = 0; x < W; x += 4)
        *reinterpret_cast<u32x4*>(kt + L::off(r, c + x / 4)) = u32x4{w[x], w[x + 1], w[x + 2], w[x + 3]};
#pragma unroll
      for (int x = 0; x < 4; ++x) widen<T>(v[i][x], vs, w + x * W / 4);
      if (__builtin_expect(scrubbed, 0)) {
#pragma unroll
        for (int x = 0; x < W; ++x) w[x] = finite_or_zero<T>(w[x]);
      }
#pragma unroll
      for (int x = 0; x < W; x += 4)
        *reinterpret_cast<u32x4*>(vt + L::off(r, c + x / 4)) = u32x4{w[x], w[x + 1], w[x + 2], w[x + 3]};
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
        uint32_t w[sizeof(T)];
        widen<T>(row[e], scale, w);
        const float x = sizeof(T) == 2 ? __uint_as_float(w[0] << 16) : __uint_as_float(w[0]);
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
  const int rl = min(j.r0 + R, j.rows) - 1, wl = min(wr + 32, j.rows) - 1;
  s.pa = p0 + j.r0 / a.G;
  s.pb = p0 + rl / a.G;
  s.wa = p0 + wr / a.G;
  s.wb = wl >= wr ? p0 + wl / a.G : s.wa - 1;
  return s;
}

// Rows of a group over its prefix: the positions are those of their sequences,
// behind all keys. A row that its sequence does not hold stands before them.
__device__ __forceinline__ Sights group_sights(const PrefixArgs& a, const Job& j, const Row& row, int R) {
  Sights s;
  auto at = [&](int token) __attribute__((always_inline)) {
    const int p = own_position(a, token);
    return p < 0 ? -1 : j.len + p;
  };
  s.p = at(row.token);
  s.jhi = row.ok && s.p >= 0 ? j.len - 1 : -1;
  const int lane = threadIdx.x & 63;
  int lo = row.ok ? s.p : 1 << 30, hi = row.ok ? s.p : -1;
#pragma unroll
  for (int x = 1; x < 32; x *= 2) {
    lo = min(lo, __shfl_xor(lo, x, 64));
    hi = max(hi, __shfl_xor(hi, x, 64));
  }
  const bool some = __any(row.ok);
  s.wa = some ? __builtin_amdgcn_readfirstlane(lo) : 1;
  s.wb = some ? __builtin_amdgcn_readfirstlane(hi) : 0;
  s.pa = s.wa;
  s.pb = s.wb;
  if (R > 32) {   // the workgroup's rows, each wave by itself
    lo = 1 << 30;
    hi = -1;
    for (int r = j.r0 + lane; r - lane < min(j.r0 + R, j.rows); r += 64) {
      const int p = at(j.t0 + min(r, j.rows - 1) / a.G);
      if (r < j.rows) {
        lo = min(lo, p);
        hi = max(hi, p);
      }
    }
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
      lo = min(lo, __shfl_xor(lo, x, 64));
      hi = max(hi, __shfl_xor(hi, x, 64));
    }
    s.pa = __builtin_amdgcn_readfirstlane(lo);
    s.pb = __builtin_amdgcn_readfirstlane(hi);
  }
  return s;
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

template <typename T, class C, int DP>
struct Shapes {
  using L = Tile<T, DP>;
  static constexpr bool H = sizeof(T) == 2 && DP <= 128;
  static constexpr bool NARROW = !(sizeof(T) == 4 && DP == 256);   // a wave's own tile would not fit
  static constexpr int KT = H ? 64 : 32, BYTES = KT * L::PITCH, WIDE = 4 * BYTES;
  static constexpr int JOIN = 32 * (DP + 2) * 4;
  static constexpr int WAVE = ((2 * kKT * L::PITCH > JOIN ? 2 * kKT * L::PITCH : JOIN) + 1023) / 1024 * 1024;
};

// 128 rows, 32 a wave; the tiles pass through LDS for all waves. The elements
// of the call are copied there without registers between, e4m3 numbers are
// widened on the way.
template <typename T, class C, int DP>
__device__ __forceinline__ void wide(const PrefixArgs& a, const Job& jb, const Row& row, const Sights& sg, int hk,
                                     uint8_t* smem, uint32_t* mask, int* found) {
  using L = Tile<T, DP>;
  constexpr bool CODES = std::is_same<C, Code>::value;
  constexpr int KT = Shapes<T, C, DP>::KT, BYTES = KT * L::PITCH, NT = 64 * kWaves;
  using Cp = Copy<T, DP, KT, NT>;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const KeyTiles kt(jb.band, jb.len, sg.pa, sg.pb, KT);
  const int x0 = (int)((int64_t)kt.count() * jb.split / jb.splits), x1 = (int)((int64_t)kt.count() * (jb.split + 1) / jb.splits);
  const Heads<C> hd(a, hk);
  u32x4 q[L::KS];
  load_row<T, DP>(q, reinterpret_cast<const T*>(a.q.p) + row.token * a.q.st + row.head * a.q.sh, row.ok, a.d);
  Softmax<DP / 32> st;
  st.init();
  const float c = a.scale * kLog2e;
  // slots (a lane a key) run two tiles ahead of the products, the copies one
  auto slot = [&](int x) __attribute__((always_inline)) {
    Slot<C> s;
    s.at = -1;
    if (x < x1 && lane < KT) s.find(a, jb.table, kt.tile(x) * KT + lane, jb.len);
    return s;
  };
  auto tile_of = [&](int x) __attribute__((always_inline)) { return smem + ((x - x0) & 1) * 2 * BYTES; };
  Stage<T, Code, DP, KT, NT> stage;
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
    if constexpr (CODES) stage.put(tile_of(x), tile_of(x) + BYTES, false);
  };
  Slot<C> here = slot(x0), next = slot(x0 + 1);
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
    uint64_t bad = 0;   // keys whose values were scrubbed
    if ((!whole || sees(jb.band, jb.len, sg.pa, sg.pb, k0, KT) != 2) &&
        __builtin_expect(Cp::holds_nonfinite(ks + BYTES, x, found), 0))
      bad = Cp::scrub(ks + BYTES, mask);
    if (x + 1 < x1) copy(x + 1, next);
    const Slot<C> after = slot(x + 2);
    const Sight sight(jb.band, sg.p, sg.jhi, k0);
    const uint64_t mine = there >> (4 * (lane >> 5));
    auto see = [&](int r) __attribute__((always_inline)) { return sight.see(r) && (mine >> r & 1); };
    auto step = [&](auto rb) __attribute__((always_inline)) {
      constexpr int RB = decltype(rb)::value;
      const int what = sees(jb.band, jb.len, sg.wa, sg.wb, k0 + RB, 32);
      if (what) softmax_step<T, DP, RB>(st, q, ks, ks + BYTES, c, what == 1 || !whole, see);
    };
    step(std::integral_constant<int, 0>{});
    if constexpr (KT == 64) step(std::integral_constant<int, 32>{});
#pragma unroll 1
    for (; __builtin_expect(bad != 0, 0); bad &= bad - 1)
      restore_key<T, C, DP>(st, hd, here, __builtin_ctzll(bad), a.d, sight);
    if (x + 1 < x1) arrive(x + 1);
    here = next;
    next = after;
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

// 32 rows; the waves take turns at the tiles of keys, each through LDS of its
// own, and join their sums at the end.
template <typename T, class C, int DP>
__device__ __forceinline__ void narrow(const PrefixArgs& a, const Job& jb, const Row& row, const Sights& sg, int hk,
                                       uint8_t* smem) {
  using L = Tile<T, DP>;
  constexpr int BYTES = kKT * L::PITCH, WAVE = Shapes<T, C, DP>::WAVE;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const KeyTiles kt(jb.band, jb.len, sg.wa, sg.wb, kKT);
  const int x0 = (int)((int64_t)kt.count() * jb.split / jb.splits), x1 = (int)((int64_t)kt.count() * (jb.split + 1) / jb.splits);
  const Heads<C> hd(a, hk);
  u32x4 q[L::KS];
  load_row<T, DP>(q, reinterpret_cast<const T*>(a.q.p) + row.token * a.q.st + row.head * a.q.sh, row.ok, a.d);
  Softmax<DP / 32> st;
  st.init();
  const float c = a.scale * kLog2e;
  uint8_t* ks = smem + wave * WAVE;
  Stage<T, C, DP, kKT, 64> stage;
  auto slot = [&](int x) __attribute__((always_inline)) {
    Slot<C> s;
    s.at = -1;
    if (x < x1 && lane < kKT) s.find(a, jb.table, kt.tile(x) * kKT + lane, jb.len);
    return s;
  };
  int x = x0 + wave;
  Slot<C> at = slot(x);
  if (x < x1) stage.load(hd, at, a.d);
  for (; x < x1; x += kWaves) {
    const Slot<C> here = at;
    const uint32_t there = (uint32_t)__ballot(here.at >= 0);
    at = slot(x + kWaves);
    const int k0 = kt.tile(x) * kKT;
    const int what = there == 0xffffffffu ? sees(jb.band, jb.len, sg.wa, sg.wb, k0, kKT) : 1;
    const bool scrubbed = what == 1 && __any(stage.any_nonfinite());
    wave_fence();
    stage.put(ks, ks + BYTES, scrubbed);
    wave_fence();
    if (x + kWaves < x1) stage.load(hd, at, a.d);
    const Sight sight(jb.band, sg.p, sg.jhi, k0);
    const uint32_t mine = there >> (4 * (lane >> 5));
    auto see = [&](int r) __attribute__((always_inline)) { return sight.see(r) && (mine >> r & 1); };
    if (what) softmax_step<T, DP, 0, true>(st, q, ks, ks + BYTES, c, what == 1, see);
    if (__builtin_expect(scrubbed, 0)) {
#pragma unroll 1
      for (int j = 0; j < kKT; ++j) restore_key<T, C, DP>(st, hd, here, j, a.d, sight);
    }
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
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      T* dst = out_row<T>(a, out) + e;
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<u32x2*>(dst) = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
      else
        *reinterpret_cast<f32x4*>(dst) = o * inv;
    } else {
      const int64_t to = part_row(a, jb.part, out);
      *reinterpret_cast<f32x4*>(a.part + to * a.d + e) = o;
      if (e == 0) *part_sums(a, to) = f32x2{m, sum};
    }
  }
}

// PW, OW: whether the rows over prefixes, and over a sequence's own keys, are
// taken 128 or 32 a workgroup.
template <typename T, class C, int DP, bool PREFIX, bool PW, bool OW>
__global__ __launch_bounds__(64 * kWaves, (sizeof(T) == 2 && DP <= 128 ? 2 : 1)) void k_prefix(const PrefixArgs a) {
  using S = Shapes<T, C, DP>;
  constexpr bool ANYW = OW || (PREFIX && PW), ANYN = !OW || (PREFIX && !PW);
  constexpr int WB = ANYW ? S::WIDE : 0, NB = ANYN ? kWaves * S::WAVE : 0;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[WB > NB ? WB : NB];
  __shared__ uint32_t mask[2];
  __shared__ int found;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  Seq s;
  Job jb;
  if (PREFIX && (int)blockIdx.x < a.pjobs) {
    constexpr int R = PW ? 32 * kWaves : 32;
    const int heads = a.Hkv * a.psplits, t = (int)blockIdx.x / heads, y = (int)blockIdx.x - t * heads, hk = y % a.Hkv;
    if (!find_rows(a, Groups{a}, t, R, s, jb.r0)) return;
    jb.table = a.ptable + (int64_t)s.b * a.p_pages;
    jb.t0 = s.t0;
    jb.rows = s.rows;
    jb.len = s.len;
    jb.split = jb.part = y / a.Hkv;
    jb.splits = a.psplits;
    jb.band = Band{a.win, 0, a.sinks};
    const Row row(a, jb, hk, jb.r0 + (PW ? 32 * wave : 0) + (lane & 31));
    const Sights sg = group_sights(a, jb, row, R);
    if constexpr (PW) wide<T, C, DP>(a, jb, row, sg, hk, smem, mask, &found);
    else narrow<T, C, DP>(a, jb, row, sg, hk, smem);
    return;
  }
  constexpr int R = OW ? 32 * kWaves : 32;
  const int job = (int)blockIdx.x - (PREFIX ? a.pjobs : 0), heads = a.Hkv * a.splits;
  const int t = job / heads, y = job - t * heads, hk = y % a.Hkv;
  if (!find_rows(a, Sequences{a}, t, R, s, jb.r0)) return;
  jb.table = a.table + (int64_t)s.b * a.max_pages;
  jb.t0 = s.t0;
  jb.rows = s.rows;
  jb.len = s.len;
  jb.split = y / a.Hkv;
  jb.splits = a.splits;
  jb.part = PREFIX || a.splits > 1 ? a.psplits + jb.split : -1;
  jb.band = Band{a.win, 0, a.sinks};
  if (PREFIX) {
    const int g = group_of(a, s.b);
    if (g >= 0) jb.band.sinks = max(0, a.sinks - Groups{a}.len(g));
  }
  const int wr = jb.r0 + (OW ? 32 * wave : 0);
  const Row row(a, jb, hk, wr + (lane & 31));
  const Sights sg = own_sights(a, jb, s.p0, row, wr, R);
  if constexpr (OW) wide<T, C, DP>(a, jb, row, sg, hk, smem, mask, &found);
  else narrow<T, C, DP>(a, jb, row, sg, hk, smem);
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
  const int token = (int)(r / a.H), head = (int)(r % a.H), e = lg * 4, all = a.psplits + a.splits;
  const bool ok = r < rows && token >= clampi(a.cu[0], 0, a.T) && token < clampi(a.cu[a.B], 0, a.T);
  int s0 = a.psplits;
  if (a.P && token >= Groups{a}.first(0) && token < Groups{a}.first(a.P)) s0 = 0;
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
    for (s0 += w; s0 < all; s0 += 4 * W) {
      f32x2 x[4];
      f32x4 y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s = s0 + i * W;
        x[i] = s < all ? *part_sums(a, rows * s + r) : f32x2{neg_inf(), 0.0f};
        y[i] = s < all && e < a.d ? *reinterpret_cast<const f32x4*>(a.part + (rows * s + r) * a.d + e) : f32x4{};
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

int row_tiles(const PrefixArgs& a, bool wide, int n) { return (int)((int64_t)a.T * a.G / (wide ? 32 * kWaves : 32)) + n; }

template <typename T, class C, int DP, bool PREFIX, bool PW, bool OW>
void start(const PrefixArgs& a, hipStream_t s) {
  const unsigned jobs = (unsigned)(a.pjobs + row_tiles(a, OW, a.B) * a.Hkv * a.splits);
  k_prefix<T, C, DP, PREFIX, PW, OW><<<jobs, 64 * kWaves, 0, s>>>(a);
}

template <typename T, class C, int DP>
hipError_t run(const PrefixArgs& a, hipStream_t s) {
  constexpr bool N = Shapes<T, C, DP>::NARROW;   // else wide throughout
  if (!a.P) {
    if constexpr (std::is_same<C, Code>::value) {   // (the other kind has its own entry point)
      if (!N || a.wide) start<T, C, DP, false, true, true>(a, s);
      else start<T, C, DP, false, true, !N>(a, s);
    }
  } else if (!N || a.wide) {
    start<T, C, DP, true, true, true>(a, s);
  } else if (a.pwide) {
    start<T, C, DP, true, true, !N>(a, s);
  } else {
    start<T, C, DP, true, !N, !N>(a, s);
  }
  if (a.P || a.splits > 1) {
    int G = 1, W = 1;
    while (G * 4 < a.d) G *= 2;
    const int64_t rows = (int64_t)a.T * a.H;
    while (G * W < 256 && 4 * W < a.psplits + a.splits && rows * G * W < 256 * 256) W *= 2;
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

void prefix_plan(PrefixArgs& a, bool bf16) {
  const bool narrow = bf16 || a.d <= 128;
  a.wide = (int64_t)a.T * a.G > 32 * (int64_t)a.B || !narrow;
  const int64_t own_keys = (int64_t)a.max_pages * a.page;
  const int64_t groups = (int64_t)row_tiles(a, a.wide, a.B) * a.Hkv;
  const int64_t most = std::max<int64_t>(1, (own_keys + kKT - 1) / kKT / (2 * kWaves));
  a.psplits = a.pjobs = 0;
  if (a.P) {
    a.pwide = a.wide || (int64_t)a.T * a.G > 32 * (int64_t)a.P || !narrow;
    const int64_t pk = (int64_t)a.p_pages * a.page, pgroups = (int64_t)row_tiles(a, a.pwide, a.P) * a.Hkv;
    const int64_t pmost = std::max<int64_t>(1, pk / kKT / (2 * kWaves));
    // both roles' keys a workgroup about alike
    const double work = (double)pgroups * pk + (double)groups * own_keys, each = work / 512;
    a.psplits = (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)(pk / std::max(each, 1.0) + 0.5), pmost, 64}));
    a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)(own_keys / std::max(each, 1.0) + 0.5), most, 32}));
    a.pjobs = (int)(pgroups * a.psplits);
    return;
  }
  if (!a.wide) {
    a.splits = (int)std::max<int64_t>(1, std::min<int64_t>({(1024 + groups - 1) / groups, most, 32}));
    return;
  }
  double best = 0;
  for (int s = 1; s <= std::min<int64_t>(most, 16); ++s) {
    const double t = (double)((groups * s + 511) / 512) / s * (s > 1 ? 1.08 + 0.02 * s : 1.0);
    if (s == 1 || t < best) {
      best = t;
      a.splits = s;
    }
  }
}

hipError_t launch_prefix(const PrefixArgs& a, bool bf16, hipStream_t s) {
  if (a.codes) return bf16 ? run<__bf16, Code>(a, s) : run<float, Code>(a, s);
  return bf16 ? run<__bf16, __bf16>(a, s) : run<float, float>(a, s);
}

}  // namespace lact
