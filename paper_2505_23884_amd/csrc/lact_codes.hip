// Keys and values into a cache of e4m3 numbers, and back out of it.
#include "lact_codes.h"
#include "lact_paged.h"

namespace lact {
namespace {

using namespace attn;

// The sequence of a token and its position there; false for a token of no
// sequence. All 64 lanes take part. Up to 64 sequences stand a lane each: the
// last one that starts at or before the token is their number that do, less
// one; more are searched.
__device__ __forceinline__ bool find_token(const CodeArgs& a, int token, int& b, int64_t& pos) {
  if (a.B <= 64) {
    const int lane = threadIdx.x & 63, c = lane < a.B ? a.cu[lane] : 0x7fffffff;
    b = -1;
    for (int j = 0; j < a.B; j += 8)
#pragma unroll
      for (int i = 0; i < 8; ++i) b += __builtin_amdgcn_readlane(c, j + i) <= token;
    // (offsets that fall again: a sequence that starts after the token is not its own)
    b = max(b, 0);
  } else {
    int hi = a.B - 1;
    b = 0;
    while (b < hi) {
      const int mid = (b + hi + 1) >> 1;
      if (a.cu[mid] <= token) b = mid;
      else hi = mid - 1;
    }
  }
  if (token >= a.T) return false;
  const int t0 = a.cu[b], t1 = min(a.cu[b + 1], a.T);
  if (token < t0 || token >= t1) return false;
  pos = seq_len(a, b) - ((int64_t)t1 - token);
  return true;
}

constexpr float kMaxCode = 448.0f;

// The slots of a workgroup's tokens, found by its first wave a lane each before
// anything is moved: where the vectors of head 0 lie, and their scales. < 0: a
// token of no sequence, or one that has no slot.
constexpr int kTokens = 64;
constexpr int64_t kNoRow = -1, kNoSlot = -2;
struct Slots {
  int64_t at[kTokens], scale[kTokens];
  __device__ __forceinline__ void find(const CodeArgs& a, int token0) {
    const int lane = threadIdx.x;
    if (lane < 64) {
      int b = 0, pg = 0, i = 0;
      int64_t pos = 0, x = kNoRow, y = 0;
      if (find_token(a, lane < a.per ? token0 + lane : a.T, b, pos)) {
        x = kNoSlot;
        if (pos >= 0 && find_slot(a, a.table + (int64_t)b * a.max_pages, (int)pos, a.max_pages * a.page, pg, i)) {
          x = pg * a.c.sb + i * a.c.st;
          y = pg * a.cs.sb + i * a.cs.st;
        }
      }
      at[lane] = x;
      scale[lane] = y;
    }
    __syncthreads();
  }
};

// Elements of T that a lane moves: 16 bytes of them.
template <typename T>
constexpr int kElems = 16 / (int)sizeof(T);

template <typename T>
__device__ __forceinline__ void spread(float (&x)[kElems<T>], const u32x4& r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      x[2 * i] = __uint_as_float(r[i] << 16);
      x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    } else {
      x[i] = __uint_as_float(r[i]);
    }
  }
}

__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < __builtin_inff(); }

// A vector of P lanes, N elements each: its scale's byte, and the numbers of
// this lane, four a word.
template <int N>
__device__ __forceinline__ void quantise(const float (&x)[N], int P, int& byte, uint32_t (&r)[N / 4]) {
  float a = 0.0f;
  bool fine = true;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    a = fmaxf(a, is_finite(x[i]) ? fabsf(x[i]) : 0.0f);
    fine &= is_finite(x[i]);
  }
  for (int s = 1; s < P; s *= 2) a = fmaxf(a, __shfl_xor(a, s, 64));
  byte = scale_byte(a);
  const float f = scale_of(254 - byte);   // 2^-e
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    float y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = fminf(fmaxf(x[4 * i + k] * f, -kMaxCode), kMaxCode);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    r[i] = (uint32_t)w;
  }
  if (__builtin_expect(!fine, 0)) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!is_finite(x[i])) r[i / 4] = (r[i / 4] & ~(0xffu << (i % 4 * 8))) | 0x7fu << (i % 4 * 8);
  }
}

// A vector of a key and one of a value by P lanes (a power of two), two of each
// a thread at a time: the largest element, by P lanes' exchanges, gives the scale. Bound by HBM:
// 8 chunks of up to 4000 tokens, 8 heads of 128, bf16, 152 MB in 40 us (3.8 TB/s; in fp32 253 MB in
// 79); four at a time the same; 64 tokens 5.8 us, the first rows loaded while their
// slots are found (7.7 us after).
template <typename T>
__global__ __launch_bounds__(256) void k_append_e4m3(const CodeArgs a, int P) {
  constexpr int N = kElems<T>, U = 2;
  __shared__ Slots slots;
  const int token0 = (int)blockIdx.x * a.per;
  const int vecs = min(a.per, a.T - token0) * a.Hkv, e = (int)(threadIdx.x & (unsigned)(P - 1)) * N, step = 256 / P;
  u32x4 k[U], v[U];
  int t[U], h[U];
  auto load = [&](int v0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int vec = v0 + u * step, x = min(vec, vecs - 1);
      t[u] = page_of(x, a.hmul, a.hshift);
      h[u] = x - t[u] * a.Hkv;
      const bool ok = vec < vecs && e < a.d;
      k[u] = load16(ok, reinterpret_cast<const T*>(a.k.p) + (token0 + t[u]) * a.k.st + h[u] * a.k.sh + e);
      v[u] = load16(ok, reinterpret_cast<const T*>(a.v.p) + (token0 + t[u]) * a.v.st + h[u] * a.v.sh + e);
    }
  };
  load(threadIdx.x / P);   // the first vectors come while their slots are found
  slots.find(a, token0);
  for (int v0 = threadIdx.x / P;;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[N], y[N];
      spread<T>(x, k[u]);
      spread<T>(y, v[u]);
      int kb, vb;
      uint32_t kn[N / 4], vn[N / 4];
      quantise<N>(x, P, kb, kn);
      quantise<N>(y, P, vb, vn);
      if (v0 + u * step >= vecs || e >= a.d || slots.at[t[u]] < 0) continue;
      const int64_t to = slots.at[t[u]] + h[u] * a.c.sh + e;
      if constexpr (N == 8) {
        *reinterpret_cast<u32x2*>(a.kc + to) = u32x2{kn[0], kn[1]};
        *reinterpret_cast<u32x2*>(a.vc + to) = u32x2{vn[0], vn[1]};
      } else {
        *reinterpret_cast<uint32_t*>(a.kc + to) = kn[0];
        *reinterpret_cast<uint32_t*>(a.vc + to) = vn[0];
      }
      if (e == 0) {
        const int64_t s = slots.scale[t[u]] + h[u] * a.cs.sh;
        a.ks[s] = (uint8_t)kb;
        a.vs[s] = (uint8_t)vb;
      }
    }
    v0 += U * step;
    if (v0 - (int)threadIdx.x / P >= vecs) break;
    load(v0);
  }
}

// 16 bytes of a key and of a value a thread, two of each at a time, so that a
// wave writes whole lines. Bound by HBM: 8 sequences of up to 16384 tokens, 4 heads of 128, to
// bf16, 294 MB in 50 us (5.9 TB/s, partly from the caches; 83 us with each thread finding
// its own slot); 64 tokens 4.1 us.
template <typename T>
__global__ __launch_bounds__(256) void k_read_e4m3(const CodeArgs a) {
  constexpr int N = kElems<T>, U = 2;
  __shared__ Slots slots;
  const int token0 = (int)blockIdx.x * a.per;
  slots.find(a, token0);
  const int items = a.Hkv * (a.d / N), all = min(a.per, a.T - token0) * items;
  for (int i0 = threadIdx.x; i0 < all; i0 += U * 256) {
    u32x2 k[U], v[U];
    int kb[U], vb[U], t[U], h[U], e[U];
    bool row[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * 256, x = min(i, all - 1);
      t[u] = page_of(x, a.mul2, a.shift2);
      const int y = x - t[u] * items;
      h[u] = page_of(y, a.hmul, a.hshift);
      e[u] = (y - h[u] * (a.d / N)) * N;
      const int64_t at = slots.at[t[u]];
      const bool ok = at >= 0;
      row[u] = i < all && at != kNoRow;
      const int64_t from = at + h[u] * a.c.sh + e[u], s = slots.scale[t[u]] + h[u] * a.cs.sh;
      kb[u] = load_byte(ok, a.ks + s);
      vb[u] = load_byte(ok, a.vs + s);
      if constexpr (N == 8) {
        k[u] = load8(ok, a.kc + from);
        v[u] = load8(ok, a.vc + from);
      } else {
        k[u][0] = load4(ok, a.kc + from);
        v[u][0] = load4(ok, a.vc + from);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!row[u]) continue;
      uint32_t kw[4], vw[4];
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        widen<T>(k[u][i], scale_of(kb[u]), kw + 2 * i);
        widen<T>(v[u][i], scale_of(vb[u]), vw + 2 * i);
      }
      *reinterpret_cast<u32x4*>(reinterpret_cast<T*>(a.k.p) + (token0 + t[u]) * a.k.st + h[u] * a.k.sh + e[u]) = u32x4{kw[0], kw[1], kw[2], kw[3]};
      *reinterpret_cast<u32x4*>(reinterpret_cast<T*>(a.v.p) + (token0 + t[u]) * a.v.st + h[u] * a.v.sh + e[u]) = u32x4{vw[0], vw[1], vw[2], vw[3]};
    }
  }
}

// Tokens a workgroup: enough of them to keep its loads in flight, where that
// leaves every CU some, and not more than an int counts the `items` of.
int tokens_each(int T, int64_t items) {
  int n = kTokens;
  while (n > 1 && ((n > 4 && (int64_t)T < 1024 * (int64_t)n) || n * items > 1 << 24)) n /= 2;
  return n;
}

}  // namespace

hipError_t launch_append_e4m3(const CodeArgs& args, bool bf16, hipStream_t s) {
  CodeArgs a = args;
  int P = 1;
  while (P * (bf16 ? 8 : 4) < a.d) P *= 2;
  a.per = tokens_each(a.T, (int64_t)a.Hkv * P);
  divider(a.Hkv, &a.hmul, &a.hshift);
  const unsigned blocks = (unsigned)((a.T + a.per - 1) / a.per);
  if (bf16) k_append_e4m3<__bf16><<<blocks, 256, 0, s>>>(a, P);
  else k_append_e4m3<float><<<blocks, 256, 0, s>>>(a, P);
  return hipGetLastError();
}

hipError_t launch_read_e4m3(const CodeArgs& args, bool bf16, hipStream_t s) {
  CodeArgs a = args;
  const int n = a.d / (bf16 ? 8 : 4);
  a.per = tokens_each(a.T, (int64_t)a.Hkv * n);
  divider(n, &a.hmul, &a.hshift);
  divider(a.Hkv * n, &a.mul2, &a.shift2);
  const unsigned blocks = (unsigned)((a.T + a.per - 1) / a.per);
  if (bf16) k_read_e4m3<__bf16><<<blocks, 256, 0, s>>>(a);
  else k_read_e4m3<float><<<blocks, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lact
