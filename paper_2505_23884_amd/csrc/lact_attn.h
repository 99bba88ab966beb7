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
constexpr uint32_t kBufOOB = 0x80000000u;      // a raw buffer offset past every range: loads zeros
constexpr int kBufFlags = 0x00020000;

// At most N of this wave's loads and copies still in flight (those that were
// issued last).
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// A barrier that waits for nothing else: reads of LDS before it are complete
// (their results are in use), copies behind it go on.
__device__ __forceinline__ void barrier_only() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

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
// the sum over the rows averages; fp32: as they are. Outputs then are off by
// 0.0023 of their norm where a form that rounds only them is off by 0.0017. A
// second product, of what is left, takes that away for a quarter to 38 % more
// time where products bound the kernel (window attention [1, 16, 16384, 128],
// window 2048: 409 us without and 519 with it; [2, 32 / 8, 8192, 64], causal: 720
// and 996; chunks over pages: 337 and 418), and for 0 to 5 % where memory does.
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

// What the rounding to bf16 leaves of 32 rows: their product added to that of
// the rounded ones is the product of the rows to 2^-16.
__device__ __forceinline__ f32x16 below_bf16(const f32x16& s) {
  f32x16 r;
#pragma unroll
  for (int e = 0; e < 16; ++e) r[e] = s[e] - (float)(__bf16)s[e];
  return r;
}

// The bf16 next below each weight (0 of 0): it and what it leaves, at most 2^-7
// of the weight, are both above zero, so that an infinity times the two parts
// stays one.
__device__ __forceinline__ f32x16 under_bf16(const f32x16& s) {
  f32x16 r;
#pragma unroll
  for (int e = 0; e < 16; ++e)
    r[e] = __uint_as_float(__builtin_elementwise_sub_sat(__float_as_uint(s[e]), 1u) & 0xffff0000u);
  return r;
}

// What stands at a masked place must not reach an output, but zero times an
// infinity or NaN is NaN, and a weight of zero is how a masked pair enters the
// second products. Such values are rare: tiles at the edge of some query's
// view are looked through once they are in LDS, and one that holds any is
// scrubbed there (infinities and NaN become zeros); what they amount to is
// then given to the pairs that are visible.

// A chunk of 16 bytes of T: whether it holds an infinity or NaN, and the
// chunk without them.
template <typename T>
__device__ __forceinline__ bool nonfinite(const u32x4& x) {
  uint32_t bad = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) bad |= (x[i] & 0x7f807f80u) + 0x00800080u;   // carries into the sign bits
    else bad |= (x[i] & 0x7f800000u) + 0x00800000u;
  }
  return bad & (sizeof(T) == 2 ? 0x80008000u : 0x80000000u);
}
template <typename T>
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t x) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t lo = (x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu;
    const uint32_t hi = (x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u;
    return lo | hi;
  } else {
    return (x & 0x7f800000u) == 0x7f800000u ? 0u : x;
  }
}

// LDS fragments are read in batches, each with its wait in the same asm
// statement: the compiler would drain the copies in flight to the
// other stage before every read that it can see, since it cannot tell the
// stages apart. The waves of a SIMD cover each other's waits.
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  typedef __attribute__((address_space(3))) const void lds_cvoid;
  return (uint32_t)(uintptr_t)(lds_cvoid*)p;
}
template <int OFF>
__device__ __forceinline__ void read_rows4(u32x4 (&r)[4], const uint32_t (&a)[4]) {
  asm volatile(
      "ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%8\n\t"
      "ds_read_b128 %2, %6 offset:%8\n\tds_read_b128 %3, %7 offset:%8\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
      : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(OFF)
      : "memory");
}
template <int OFF>
__device__ __forceinline__ void read_rows8(u32x4 (&r)[8], const uint32_t (&a)[8]) {
  asm volatile(
      "ds_read_b128 %0, %8 offset:%16\n\tds_read_b128 %1, %9 offset:%16\n\t"
      "ds_read_b128 %2, %10 offset:%16\n\tds_read_b128 %3, %11 offset:%16\n\t"
      "ds_read_b128 %4, %12 offset:%16\n\tds_read_b128 %5, %13 offset:%16\n\t"
      "ds_read_b128 %6, %14 offset:%16\n\tds_read_b128 %7, %15 offset:%16\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(a[4]), "v"(a[5]), "v"(a[6]), "v"(a[7]), "n"(OFF)
      : "memory");
}
// Column fragments of two 32-column blocks and both 16-row steps: r[4 b + 2 s]
// rows 16 s + 4 half + 0..3, r[4 b + 2 s + 1] the rows 8 further (lo, hi: the
// lane's addresses of the two in each block).
template <int OFF, int STEP>
__device__ __forceinline__ void read_cols2(u32x2 (&r)[8], const uint32_t (&lo)[2], const uint32_t (&hi)[2]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %9 offset:%12\n\t"
      "ds_read_b64_tr_b16 %2, %8 offset:%13\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
      "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %11 offset:%12\n\t"
      "ds_read_b64_tr_b16 %6, %10 offset:%13\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(lo[0]), "v"(hi[0]), "v"(lo[1]), "v"(hi[1]), "n"(OFF), "n"(OFF + STEP)
      : "memory");
}

// The same of four blocks in one batch.
template <int OFF, int STEP>
__device__ __forceinline__ void read_cols4(u32x2 (&r)[16], const uint32_t (&lo)[4], const uint32_t (&hi)[4]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %16 offset:%24\n\tds_read_b64_tr_b16 %1, %17 offset:%24\n\t"
      "ds_read_b64_tr_b16 %2, %16 offset:%25\n\tds_read_b64_tr_b16 %3, %17 offset:%25\n\t"
      "ds_read_b64_tr_b16 %4, %18 offset:%24\n\tds_read_b64_tr_b16 %5, %19 offset:%24\n\t"
      "ds_read_b64_tr_b16 %6, %18 offset:%25\n\tds_read_b64_tr_b16 %7, %19 offset:%25\n\t"
      "ds_read_b64_tr_b16 %8, %20 offset:%24\n\tds_read_b64_tr_b16 %9, %21 offset:%24\n\t"
      "ds_read_b64_tr_b16 %10, %20 offset:%25\n\tds_read_b64_tr_b16 %11, %21 offset:%25\n\t"
      "ds_read_b64_tr_b16 %12, %22 offset:%24\n\tds_read_b64_tr_b16 %13, %23 offset:%24\n\t"
      "ds_read_b64_tr_b16 %14, %22 offset:%25\n\tds_read_b64_tr_b16 %15, %23 offset:%25\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7]),
        "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]), "=&v"(r[14]), "=&v"(r[15])
      : "v"(lo[0]), "v"(hi[0]), "v"(lo[1]), "v"(hi[1]), "v"(lo[2]), "v"(hi[2]), "v"(lo[3]), "v"(hi[3]), "n"(OFF),
        "n"(OFF + STEP)
      : "memory");
}

// One fp32 column over 32 rows: r[i] of row 8 (i / 4) + i % 4 from the lane's
// first, whose addresses with the swizzles of rows 0 .. 3 and 8 .. 11 are a[0 .. 7].
template <int OFF, int PITCH>
__device__ __forceinline__ void read_col32(float (&r)[16], const uint32_t (&a)[8]) {
  asm volatile(
      "ds_read_b32 %0, %16 offset:%24\n\tds_read_b32 %1, %17 offset:%25\n\t"
      "ds_read_b32 %2, %18 offset:%26\n\tds_read_b32 %3, %19 offset:%27\n\t"
      "ds_read_b32 %4, %20 offset:%24\n\tds_read_b32 %5, %21 offset:%25\n\t"
      "ds_read_b32 %6, %22 offset:%26\n\tds_read_b32 %7, %23 offset:%27\n\t"
      "ds_read_b32 %8, %16 offset:%28\n\tds_read_b32 %9, %17 offset:%29\n\t"
      "ds_read_b32 %10, %18 offset:%30\n\tds_read_b32 %11, %19 offset:%31\n\t"
      "ds_read_b32 %12, %20 offset:%28\n\tds_read_b32 %13, %21 offset:%29\n\t"
      "ds_read_b32 %14, %22 offset:%30\n\tds_read_b32 %15, %23 offset:%31\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7]),
        "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]), "=&v"(r[14]), "=&v"(r[15])
      : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(a[4]), "v"(a[5]), "v"(a[6]), "v"(a[7]), "n"(OFF),
        "n"(OFF + PITCH), "n"(OFF + 2 * PITCH), "n"(OFF + 3 * PITCH), "n"(OFF + 16 * PITCH), "n"(OFF + 17 * PITCH),
        "n"(OFF + 18 * PITCH), "n"(OFF + 19 * PITCH)
      : "memory");
}

// acc (32 rows of the tile from RB x 32 columns of b) += rows . b over d; b
// holds a lane's column as Tile::KS chunks. N chunks a batch of reads.
template <typename T, int DP, int RB, int N = (Tile<T, DP>::KS < 8 ? 4 : 8)>
__device__ __forceinline__ void mma_dot_add(f32x16& acc, const uint8_t* tile, const u32x4 (&b)[(Tile<T, DP>::KS)]) {
  using L = Tile<T, DP>;
  const int lane = threadIdx.x & 63;
  // chunk 2c + half of the row: the lane's first address with bits 5 and up of c flipped in
  const uint32_t a0 = lds_addr(tile) + L::off(lane & 31, lane >> 5);
#pragma unroll
  for (int c = 0; c < L::KS; c += N) {
    uint32_t a[N];
    u32x4 r[N];
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = a0 ^ (uint32_t)((c + i) << 5);
    if constexpr (N == 4) read_rows4<RB * L::PITCH>(r, a);
    else read_rows8<RB * L::PITCH>(r, a);
#pragma unroll
    for (int i = 0; i < N; ++i) mma_chunk<T>(acc, r[i], b[c + i]);
  }
}
template <typename T, int DP, int RB>
__device__ __forceinline__ void mma_dot(f32x16& acc, const uint8_t* tile, const u32x4 (&b)[(Tile<T, DP>::KS)]) {
  acc = f32x16{};
  mma_dot_add<T, DP, RB>(acc, tile, b);
}
// The same with b's columns as rows of another tile in LDS (16-bit).
template <int DP>
__device__ __forceinline__ void mma_dot_lds(f32x16& acc, const uint8_t* tile, const uint8_t* bt) {
  using L = Tile<__bf16, DP>;
  const int lane = threadIdx.x & 63, o = L::off(lane & 31, lane >> 5);
  const uint32_t a0 = lds_addr(tile) + o, b0 = lds_addr(bt) + o;
#pragma unroll
  for (int c = 0; c < L::KS; c += 4) {
    uint32_t ad[8];
    u32x4 r[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      ad[i] = a0 ^ (uint32_t)((c + i) << 5);
      ad[4 + i] = b0 ^ (uint32_t)((c + i) << 5);
    }
    read_rows8<0>(r, ad);
#pragma unroll
    for (int i = 0; i < 4; ++i) mma_chunk<__bf16>(acc, r[i], r[4 + i]);
  }
}

// acc[0 .. NB) (32-column blocks db0 .. of d x 32 columns of b) += (rows RB ..
// RB + 31 of the tile)^T x b.
template <typename T, int DP, int NB, int RB>
__device__ __forceinline__ void mma_rows(f32x16 (&acc)[NB], const RowsB<T>& b, const uint8_t* tile, int db0) {
  using L = Tile<T, DP>;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  if constexpr (sizeof(T) == 2) {
    constexpr int M = NB % 4 ? 2 : 4;   // column blocks a batch
    static_assert(NB % M == 0, "column blocks are read in pairs");
    const int g = (lane >> 4) & 1, sl = lane & 15, row = 4 * half + (sl >> 2), chunk = 2 * g + ((sl >> 1) & 1);
    const uint32_t base = lds_addr(tile) + ((sl & 1) << 3);
    const uint32_t a0 = base + L::off(row, chunk), a1 = base + L::off(row + 8, chunk);
#pragma unroll
    for (int x = 0; x < NB; x += M) {
      uint32_t lo[M], hi[M];
#pragma unroll
      for (int y = 0; y < M; ++y) {
        lo[y] = a0 ^ (uint32_t)((db0 + x + y) << 6);
        hi[y] = a1 ^ (uint32_t)((db0 + x + y) << 6);
      }
      u32x2 r[4 * M];
      if constexpr (M == 4) read_cols4<RB * L::PITCH, 16 * L::PITCH>(r, lo, hi);
      else read_cols2<RB * L::PITCH, 16 * L::PITCH>(r, lo, hi);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int y = 0; y < M; ++y) {
          const u32x2 p = r[4 * y + 2 * s], q = r[4 * y + 2 * s + 1];
          mma_chunk<T>(acc[x + y], u32x4{p[0], p[1], q[0], q[1]}, b.v[s]);
        }
    }
  } else {
    // the lane's column of block db0 in rows 4 half + 0 .. 3 and 8 further
    uint32_t a[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = 8 * (i >> 2) + 4 * half;   // + i % 4: in the read's offset, but not in the swizzle
      const int c = (lane & 31) >> 2;
      a[i] = lds_addr(tile) + row * L::PITCH + ((c ^ L::swz(row + (i & 3))) << 4) + ((lane & 3) << 2);
    }
#pragma unroll
    for (int x = 0; x < NB; ++x) {
      uint32_t ax[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) ax[i] = a[i] ^ (uint32_t)((db0 + x) << 7);
      float r[16];
      read_col32<RB * L::PITCH, L::PITCH>(r, ax);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        acc[x] = __builtin_amdgcn_mfma_f32_32x32x2f32(r[i], b.v[i], acc[x], 0, 0, 0);
    }
  }
}

// The infinities and NaN of a scrubbed row (d elements in memory), added to
// the lane's column of acc where its query (or key) sees the row: the product
// with any weight above zero.
template <typename T, int NB>
__device__ __forceinline__ void add_nonfinite(f32x16 (&acc)[NB], const T* row, bool see, int d0, int d) {
  int half = (threadIdx.x >> 5) & 1;
  asm volatile("" : "+v"(half));   // nothing of this is worked out ahead of a loop, for it hardly ever runs
#pragma unroll
  for (int db = 0; db < NB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int e = d0 + 32 * db + 8 * (i >> 2) + 4 * half + (i & 3);
      if (!see || e >= d) continue;
      const float x = (float)row[e];
      if (!(fabsf(x) < __builtin_inff())) acc[db][i] += x;
    }
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

// A tile of R rows copied from memory to LDS by the NT threads of a
// workgroup, 16 bytes a lane and without registers between (each wave
// instruction fills 1 KiB in order; the swizzle is in the source addresses).
// The copies are done when vmcnt is 0 (a __syncthreads waits for it).
template <typename T, int DP, int R, int NT>
struct Copy {
  using L = Tile<T, DP>;
  static constexpr int N = R * L::CPR / NT;     // chunks per thread
  static constexpr int STEP = NT / L::CPR;      // rows between them
  static_assert(N >= 1 && R * L::CPR % NT == 0 && NT % L::CPR == 0, "tile split");
  typedef __attribute__((address_space(3))) void lds_void;

  // A wave of a workgroup may have tiles of its own (NT = 64): its barriers
  // are only waits.
  static __device__ __forceinline__ int thread() { return NT == 64 ? threadIdx.x & 63 : threadIdx.x; }
  static __device__ __forceinline__ void sync() {
    if constexpr (NT == 64) {
      wait_loads<0>();
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
      __builtin_amdgcn_wave_barrier();
    } else {
      __syncthreads();
    }
  }

  // rows of `ld` bytes from `base` (the same in all threads), `rows` of them
  // (<= 0: none); the rest, and columns past d, are zeros
  // FRESH: the offsets are worked out each time (about 10 instructions a
  // chunk) instead of staying in registers through a loop.
  template <bool FRESH = false>
  static __device__ __forceinline__ void rows(uint8_t* tile, const T* base, int ld, int64_t rows, int d) {
    int tid = thread();
    if constexpr (FRESH) asm volatile("" : "+v"(tid));
    const int n = (int)(rows < R ? rows : R);
    const int span = n > 0 ? (n - 1) * ld + d * (int)sizeof(T) : 0;
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, span, kBufFlags);
    const int wave = NT == 64 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = tid / L::CPR + i * STEP, c = (tid % L::CPR) ^ L::swz(row);
      const uint32_t o = c * L::E < d ? (uint32_t)(row * ld + c * 16) : kBufOOB;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(tile + (i * NT + wave * 64) * 16), 16, o, 0, 0, 0);
    }
  }
  // this thread's part of a tile in LDS: whether it holds an infinity or NaN, and without them
  static __device__ __forceinline__ bool any_nonfinite(const uint8_t* tile) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < N; ++i) bad |= nonfinite<T>(*reinterpret_cast<const u32x4*>(tile + (i * NT + thread()) * 16));
    return bad;
  }
  // whether tile x holds an infinity or NaN, by all NT threads with a
  // barrier; `found`: a word of LDS, -1 at first
  static __device__ __forceinline__ bool holds_nonfinite(const uint8_t* tile, int x, int* found) {
    if (any_nonfinite(tile)) *found = x;
    sync();
    return *found == x;
  }
  // scrubs the tile; the rows that held one, a bit each (`mask`: two words of
  // LDS). By all NT threads, with barriers before and after.
  static __device__ __forceinline__ uint64_t scrub(uint8_t* tile, uint32_t* mask) {
    if (thread() < 2) mask[thread()] = 0;
    sync();
#pragma unroll 1
    for (int i = 0; i < N; ++i) {
      const int at = i * NT + thread(), row = at / L::CPR;
      u32x4 x = *reinterpret_cast<const u32x4*>(tile + at * 16);
      if (!nonfinite<T>(x)) continue;
      atomicOr(&mask[row >> 5], 1u << (row & 31));
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = finite_or_zero<T>(x[k]);
      *reinterpret_cast<u32x4*>(tile + at * 16) = x;
    }
    sync();
    const uint32_t lo = __builtin_amdgcn_readfirstlane(mask[0]), hi = __builtin_amdgcn_readfirstlane(mask[1]);
    sync();
    return ((uint64_t)hi << 32) | lo;
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
    const bool up = mx > m + 8.0f;   // by lane: a row's result does not depend on its neighbours'
    if (!__any(up)) return;
    const float f = up ? __builtin_amdgcn_exp2f(m - mx) : 1.0f;
    m = up ? mx : m;
    l *= f;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int k = 0; k < 16; ++k) o[i][k] *= f;
  }
  // The lane's sums to LDS, a float every 64 (16 NB + 2 of them), and those of
  // other keys added.
  __device__ __forceinline__ void put(float* to) const {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int k = 0; k < 16; ++k) to[(i * 16 + k) * 64] = o[i][k];
    to[NB * 16 * 64] = m;
    to[(NB * 16 + 1) * 64] = l;
  }
  __device__ __forceinline__ void join(const float* from) {
    const float m2 = from[NB * 16 * 64], up = fmaxf(m, m2);
    const float f = m == up ? 1.0f : __builtin_amdgcn_exp2f(m - up), g = m2 == up ? 1.0f : __builtin_amdgcn_exp2f(m2 - up);
    m = up;
    l = l * f + from[(NB * 16 + 1) * 64] * g;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int k = 0; k < 16; ++k) o[i][k] = o[i][k] * f + from[(i * 16 + k) * 64] * g;
  }
};

// What a lane's query sees of a tile: rows r with r - lo <= span (unsigned) or
// r < sink, r counted from the tile's first key plus 4 (lane / 32).
struct Sight {
  int lo, sink;
  uint32_t span;
  template <class Args>
  __device__ __forceinline__ Sight(const Args& a, int p, int jhi, int k0) {
    const int at = k0 + 4 * (int)((threadIdx.x >> 5) & 1), jlo = p - a.win + 1;
    lo = jhi < jlo ? (1 << 30) : jlo - at;
    span = (uint32_t)max(jhi - jlo, 0);
    sink = k0 < a.sinks ? min(a.sinks, jhi + 1) - at : -(1 << 30);
  }
  __device__ __forceinline__ bool see(int r) const { return ((uint32_t)(r - lo) <= span) | (r < sink); }
};

// The 32 keys of a tile from row RB: scores, weights, and their products with
// the values. see(r) says whether the lane's query sees row r + 4 (lane / 32)
// (`masked`, the same in all lanes; else it sees all of them). Whole: the
// weights in two parts, so that their rounding to bf16 costs nothing.
template <typename T, int DP, int RB, bool Whole = false, class See>
__device__ __forceinline__ void softmax_step(Softmax<DP / 32>& st, const u32x4 (&q)[(Tile<T, DP>::KS)],
                                             const uint8_t* kt, const uint8_t* vt, float c, bool masked, See&& see) {
  f32x16 s;
  mma_dot<T, DP, RB>(s, kt, q);
  if (masked) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (!see(RB + 8 * (i >> 2) + (i & 3))) s[i] = neg_inf();
  }
  float mx = neg_inf();
#pragma unroll
  for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[i]);
  st.grow(half_max(mx) * c);
  const float m = st.m == neg_inf() ? 0.0f : st.m;   // a query that has seen nothing: weights of 0, not NaN
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -m));
    sum += s[i];
  }
  st.l += sum;
  if constexpr (Whole && sizeof(T) == 2) {
    const f32x16 most = under_bf16(s);
    mma_rows<T, DP, DP / 32, RB>(st.o, RowsB<T>(most), vt, 0);
    s -= most;
  }
  mma_rows<T, DP, DP / 32, RB>(st.o, RowsB<T>(s), vt, 0);
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
