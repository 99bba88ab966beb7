// Tile primitives of the softmax-attention kernels (lact_window.hip,
// lact_paged.hip), 16-bit and fp32.
//
// All products are 32x32 MFMA tiles. A tile of keys (or queries) lies in LDS
// row by row, 16-byte chunks XOR-swizzled by the row, and is read two ways:
// by rows (a lane takes 16 bytes of row lane % 32: the operand whose
// contraction runs along d) and by columns (a lane takes one column d over
// several rows: the operand whose contraction runs over the rows).
//
// The accumulator of such a product holds, in lane l, column l % 32 and rows
// 8 (i / 4) + 4 (l / 32) + i % 4 (i = 0 .. 15). A second product that
// contracts over those rows takes them as its B operand in exactly the
// registers they are in: the order of a contraction is free, so the A operand
// is read with the same permutation of rows and nothing is exchanged between
// lanes. With scores held transposed (keys x queries) one lane owns one
// query: its running maximum and sum are scalars of the lane.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lact {
namespace attn {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kTiny = 1.17549435e-38f;       // least normal fp32 (and bf16)
constexpr uint32_t kBufOOB = 0x80000000u;      // a raw buffer offset past every range: loads zeros
constexpr int kBufFlags = 0x00020000;

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// Lane of the other half of the wave: max / sum of x over lanes l and l ^ 32.
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A tile of rows of DP elements of T (the head dimension padded to DP with
// zeros).
template <typename T, int DP>
struct Tile {
  static constexpr int E = 16 / (int)sizeof(T);   // elements per 16-byte chunk
  static constexpr int CPR = DP / E;              // chunks per row
  static constexpr int PITCH = DP * (int)sizeof(T);
  static constexpr int KS = CPR / 2;              // steps of a contraction over d (two chunks each)
  static constexpr int DB = DP / 32;              // 32-column blocks

  // Chunk swizzle: any 8 consecutive rows put one chunk into different banks
  // (16-byte reads by rows), and 4 consecutive rows from a multiple of 4 put
  // 32 aligned bytes into different quarters of the 64 banks (column reads).
  static __device__ __forceinline__ int swz(int row) {
    if constexpr (CPR >= 16) return ((row & 3) << 2) | ((row >> 1) & 2) | ((row >> 3) & 1);
    else return (((row >> 1) & 1) << 2) | ((row >> 1) & 2) | ((row >> 3) & 1);
  }
  static __device__ __forceinline__ int off(int row, int chunk) { return row * PITCH + ((chunk ^ swz(row)) << 4); }
  static __device__ __forceinline__ u32x4 row_chunk(const uint8_t* t, int row, int chunk) {
    return *reinterpret_cast<const u32x4*>(t + off(row, chunk));
  }
};

// acc += A B over the elements of one chunk pair (lanes 0-31 hold the first
// chunk, 32-63 the second): 16 contraction elements in bf16, 8 in fp32.
template <typename T>
__device__ __forceinline__ void mma_chunk(f32x16& acc, const u32x4& a, const u32x4& b) {
  if constexpr (sizeof(T) == 2) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0,
                                                  0, 0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], acc, 0, 0, 0);
  }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const f32x2 x = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// 32 rows of an accumulator as the B operand of a product that contracts over
// them. bf16: rounded to nearest, at most 2^-8 of each weight, which
// the sum over the rows averages; fp32: as they are.
template <typename T> struct RowsB;
template <> struct RowsB<__bf16> {
  u32x4 v[2];
  __device__ __forceinline__ explicit RowsB(const f32x16& s) {
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[g][i] = pack_bf16(s[8 * g + 2 * i], s[8 * g + 2 * i + 1]);
  }
};
template <> struct RowsB<float> {
  f32x16 v;
  __device__ __forceinline__ explicit RowsB(const f32x16& s) : v(s) {}
};

// The two 16-bit halves of a dword: whether they are infinite or NaN, +inf or
// NaN (`sign` 0), -inf or NaN (`sign` 0x8000), as 0 / 1.0 in bf16.
__device__ __forceinline__ uint32_t bf16_nonfinite(uint32_t x) {
  return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}
__device__ __forceinline__ uint32_t bf16_finite_or_zero(uint32_t x) {
  const uint32_t lo = (x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu;
  const uint32_t hi = (x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u;
  return lo | hi;
}
__device__ __forceinline__ uint32_t bf16_one_if(uint32_t x, uint32_t sign) {
  uint32_t r = 0;
#pragma unroll
  for (int s = 0; s < 32; s += 16) {
    const uint32_t h = (x >> s) & 0xffffu, mag = h & 0x7fffu;
    if (mag > 0x7f80u || (mag == 0x7f80u && (h & 0x8000u) == sign)) r |= 0x3f80u << s;
  }
  return r;
}
__device__ __forceinline__ uint32_t bf16_one_if_nonzero(uint32_t x) {
  return ((x & 0x7fffu) ? 0x3f80u : 0u) | ((x & 0x7fff0000u) ? 0x3f800000u : 0u);
}

// Infinities that the products of one block are known to hold.
__device__ __forceinline__ void add_infinities(f32x16& acc, const f32x16& plus, const f32x16& minus) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (plus[i] > 0.0f) acc[i] += __builtin_inff();
    if (minus[i] > 0.0f) acc[i] += neg_inf();
  }
}

// acc (32 columns d x 32 columns of b) += (rows rb .. rb + 31, columns
// 32 db ..  of the tile)^T x b.
//
// MASKED (b has weights that are zero because their pair is masked): a zero
// weight drops its product, so an infinity or NaN that stands in a masked
// place reaches no output; products with a non-zero weight are as in IEEE
// arithmetic (an infinity stays one, NaN stays NaN). Such values are rare:
// they are looked for, and only then the slower form runs, which multiplies
// them as zeros and then adds what they amount to (+inf, -inf, or both for
// NaN) wherever a non-zero weight meets them.
template <typename T, int DP, bool MASKED>
__device__ __forceinline__ void mma_rows(f32x16& acc, const RowsB<T>& b, const uint8_t* tile, int rb, int db) {
  using L = Tile<T, DP>;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  if constexpr (sizeof(T) == 2) {
    const int g = (lane >> 4) & 1, sl = lane & 15;
    const int chunk = 4 * db + 2 * g + ((sl >> 1) & 1);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int r0 = rb + 16 * s + 4 * half + (sl >> 2), r1 = r0 + 8;
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                     (lds_s16x4*)(tile + L::off(r0, chunk) + ((sl & 1) << 3))));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                     (lds_s16x4*)(tile + L::off(r1, chunk) + ((sl & 1) << 3))));
      u32x4 a = {lo[0], lo[1], hi[0], hi[1]};
      if constexpr (MASKED) {
        const uint32_t bad =
            bf16_nonfinite(a[0]) | bf16_nonfinite(a[1]) | bf16_nonfinite(a[2]) | bf16_nonfinite(a[3]);
        if (__builtin_expect(__any(bad != 0), 0)) {
          u32x4 w, ap, am;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = bf16_one_if_nonzero(b.v[s][i]);
            ap[i] = bf16_one_if(a[i], 0u);
            am[i] = bf16_one_if(a[i], 0x8000u);
            a[i] = bf16_finite_or_zero(a[i]);
          }
          f32x16 plus = {}, minus = {};
          mma_chunk<T>(plus, ap, w);
          mma_chunk<T>(minus, am, w);
          add_infinities(acc, plus, minus);
        }
      }
      mma_chunk<T>(acc, a, b.v[s]);
    }
  } else {
    const int col = 32 * db + (lane & 31);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int row = rb + 8 * (i >> 2) + 4 * half + (i & 3);
      float a = *reinterpret_cast<const float*>(tile + L::off(row, col >> 2) + ((col & 3) << 2));
      if constexpr (MASKED) {
        const bool bad = !(fabsf(a) < __builtin_inff());
        if (__builtin_expect(__any(bad), 0)) {
          const float w = b.v[i] != 0.0f ? 1.0f : 0.0f, inf = __builtin_inff();
          f32x16 plus = {}, minus = {};
          plus = __builtin_amdgcn_mfma_f32_32x32x2f32(bad && a != -inf ? 1.0f : 0.0f, w, plus, 0, 0, 0);
          minus = __builtin_amdgcn_mfma_f32_32x32x2f32(bad && a != inf ? 1.0f : 0.0f, w, minus, 0, 0, 0);
          add_infinities(acc, plus, minus);
          if (bad) a = 0.0f;
        }
      }
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a, b.v[i], acc, 0, 0, 0);
    }
  }
}

// acc (32 rows of the tile from rb x 32 columns of b) = rows . b over d; b
// holds a lane's column as Tile::KS chunks.
template <typename T, int DP>
__device__ __forceinline__ void mma_dot(f32x16& acc, const uint8_t* tile, int rb, const u32x4 (&b)[(Tile<T, DP>::KS)]) {
  using L = Tile<T, DP>;
  const int lane = threadIdx.x & 63;
  acc = f32x16{};
#pragma unroll
  for (int c = 0; c < L::KS; ++c)
    mma_chunk<T>(acc, L::row_chunk(tile, rb + (lane & 31), 2 * c + (lane >> 5)), b[c]);
}

// One lane's row (16-byte chunks 2c + lane / 32) of a matrix in memory, zeros
// where !ok and past d.
template <typename T, int DP>
__device__ __forceinline__ void load_row(u32x4 (&r)[(Tile<T, DP>::KS)], const T* row, bool ok, int d) {
  using L = Tile<T, DP>;
  const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int c = 0; c < L::KS; ++c) {
    const int e = (2 * c + half) * L::E;
    r[c] = ok && e < d ? *reinterpret_cast<const u32x4*>(row + e) : u32x4{};
  }
}

// A tile of R rows on its way from memory to LDS through the registers of NT
// threads, 16 bytes a time along the rows: the loads of the next tile are
// issued before the products of the present one and stored after them.
template <typename T, int DP, int R, int NT>
struct Stage {
  using L = Tile<T, DP>;
  static constexpr int N = R * L::CPR / NT;     // chunks per thread
  static constexpr int STEP = NT / L::CPR;      // rows between them
  static_assert(N >= 1 && R * L::CPR % NT == 0 && NT % L::CPR == 0, "tile split");
  u32x4 r[N];

  // rows of `ld` bytes from `base` (the same in all threads), `rows` of them
  // (<= 0: none); the rest, and columns past d, are zeros
  __device__ __forceinline__ void load(const T* base, int ld, int64_t rows, int d) {
    const int row = threadIdx.x % NT / L::CPR, c = threadIdx.x % L::CPR;
    const int n = (int)(rows < R ? rows : R);
    const int span = n > 0 ? (n - 1) * ld + d * (int)sizeof(T) : 0;
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, span, kBufFlags);
    const uint32_t o = c * L::E < d ? (uint32_t)(row * ld + c * 16) : kBufOOB;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, o + (uint32_t)(i * STEP * ld), 0, 0);
  }
  __device__ __forceinline__ void store(uint8_t* tile) const {
    const int row = threadIdx.x % NT / L::CPR, c = threadIdx.x % L::CPR;
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(tile + L::off(row + i * STEP, c)) = r[i];
  }
};

// acc (columns d in rows, this lane's row in its column) * f to the lane's
// row of d elements at `out`, 16 bytes a store.
template <typename T, int NB>
__device__ __forceinline__ void store_row(T* out, const f32x16 (&acc)[NB], float f, int d0, int d, bool ok, bool zero) {
  const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int db = 0; db < NB; ++db) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int g = 0; g < 4; g += 2) {
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = 4 * (g + (i >> 1)) + 2 * (i & 1);
          x[i] = zero ? 0u : pack_bf16(acc[db][k] * f, acc[db][k + 1] * f);
        }
        // lanes 0-31 take the eight elements of block g, lanes 32-63 those of g + 1
        const auto a = __builtin_amdgcn_permlane32_swap(x[0], x[2], false, false);
        const auto b = __builtin_amdgcn_permlane32_swap(x[1], x[3], false, false);
        const int e = d0 + 32 * db + 8 * (g + half);
        if (ok && e < d) *reinterpret_cast<u32x4*>(out + e) = u32x4{a[0], b[0], a[1], b[1]};
      }
    } else {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int e = d0 + 32 * db + 8 * g + 4 * half;
        f32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = zero ? 0.0f : acc[db][4 * g + i] * f;
        if (ok && e < d) *reinterpret_cast<f32x4*>(out + e) = x;
      }
    }
  }
}

// Running softmax of one lane's query (scores times the scale and log2 e).
// The maximum follows the scores only when some lane's has grown by more than
// 8 (a factor of 256 in the weights, far from fp32's limits): most tiles then
// leave the accumulators as they are. m is shared by the lane's two halves of
// the keys, l is this half's sum.
template <int NB>
struct Softmax {
  f32x16 o[NB];
  float m, l;
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int i = 0; i < NB; ++i) o[i] = f32x16{};
    m = neg_inf();
    l = 0.0f;
  }
  __device__ __forceinline__ void grow(float mx) {
    if (!__any(mx > m + 8.0f)) return;
    const float mn = fmaxf(m, mx);
    const float f = mn == m ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    l *= f;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int k = 0; k < 16; ++k) o[i][k] *= f;
  }
};

// One tile of KT keys: scores, weights, and their products with the values.
// see(j) says whether the lane's query sees key j of the tile (MASKED).
template <typename T, int DP, int KT, bool MASKED, class See>
__device__ __forceinline__ void softmax_tile(Softmax<DP / 32>& st, const u32x4 (&q)[(Tile<T, DP>::KS)], const uint8_t* kt,
                                             const uint8_t* vt, float c, See&& see) {
  constexpr int MB = KT / 32;
  const int half = (threadIdx.x >> 5) & 1;
  f32x16 s[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) mma_dot<T, DP>(s[b], kt, 32 * b, q);
  float mx = neg_inf();
#pragma unroll
  for (int b = 0; b < MB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (MASKED)
        if (!see(32 * b + 8 * (i >> 2) + 4 * half + (i & 3))) s[b][i] = neg_inf();
      mx = fmaxf(mx, s[b][i]);
    }
  st.grow(half_max(mx) * c);
  const float m = st.m == neg_inf() ? 0.0f : st.m;   // a query that has seen nothing: weights of 0, not NaN
  float sum = 0.0f;
#pragma unroll
  for (int b = 0; b < MB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], c, -m));
      // a visible weight stays above zero, which is what marks a masked one
      if constexpr (MASKED) p = p < kTiny && s[b][i] != neg_inf() ? kTiny : p;
      s[b][i] = p;
      sum += p;
    }
  st.l += sum;
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const RowsB<T> w(s[b]);
#pragma unroll
    for (int db = 0; db < DP / 32; ++db) mma_rows<T, DP, MASKED>(st.o[db], w, vt, 32 * b, db);
  }
}

// The band of an attention is args.win, .look and .sinks: position p sees key j
// when j <= p + look and (j > p - win or j < sinks).
//
// The tiles of KT keys that positions pa .. pb see: n1 of them from the first
// (they hold sinks), then n2 from t2 on.
struct KeyTiles {
  int n1, t2, n2;
  template <class Args>
  __device__ __forceinline__ KeyTiles(const Args& a, int len, int pa, int pb, int KT) {
    n1 = t2 = n2 = 0;
    const int hi = min(len - 1, pb + a.look), lo = max(0, pa - a.win + 1);
    if (pa > pb || hi < 0) return;
    const int sk = min(a.sinks, hi + 1);
    n1 = (sk + KT - 1) / KT;
    if (lo > hi) return;
    t2 = max(lo / KT, n1);
    n2 = max(0, hi / KT - t2 + 1);
  }
  __device__ __forceinline__ int count() const { return n1 + n2; }
  __device__ __forceinline__ int tile(int i) const { return i < n1 ? i : t2 + (i - n1); }
};

// What the 32 queries of a wave (positions wa .. wb, those of the sequence)
// see of the keys k0 .. k0 + KT - 1: nothing (0), something (1) or all (2).
template <class Args>
__device__ __forceinline__ int sees(const Args& a, int len, int wa, int wb, int k0, int KT) {
  const int k1 = k0 + KT - 1;
  if (wa > wb || k0 >= len || k0 > wb + a.look || (k1 <= wa - a.win && k0 >= a.sinks)) return 0;
  return k1 < len && k1 <= wa + a.look && (k0 > wb - a.win || k1 < a.sinks) ? 2 : 1;
}

}  // namespace attn
}  // namespace lact
