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
    const int lane = threadIdx.x & 63, c = a.cu[min(lane, a.B - 1)];
    b = -1;
    for (int j = 0; j < a.B; ++j) b += __builtin_amdgcn_readlane(c, j) <= token;
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

// Eight elements of T in memory as fp32.
template <typename T>
__device__ __forceinline__ void load8(float (&x)[8], const T* p) {
  if constexpr (sizeof(T) == 2) {
    const u32x4 r = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(r[i] << 16);
      x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x4 r = *reinterpret_cast<const f32x4*>(p + 4 * i);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[4 * i + k] = r[k];
    }
  }
}

__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < __builtin_inff(); }

// A vector of P lanes, eight elements each: its scale's byte, and the eight
// numbers of this lane.
__device__ __forceinline__ u32x2 quantise(const float (&x)[8], int P, int& byte) {
  float a = 0.0f;
  bool fine = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    a = fmaxf(a, is_finite(x[i]) ? fabsf(x[i]) : 0.0f);
    fine &= is_finite(x[i]);
  }
  for (int s = 1; s < P; s *= 2) a = fmaxf(a, __shfl_xor(a, s, 64));
  byte = scale_byte(a);
  const float f = scale_of(254 - byte);   // 2^-e
  uint32_t r[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = fminf(fmaxf(x[4 * i + k] * f, -kMaxCode), kMaxCode);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    r[i] = (uint32_t)w;
  }
  if (__builtin_expect(!fine, 0)) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!is_finite(x[i])) r[i / 4] = (r[i / 4] & ~(0xffu << (i % 4 * 8))) | 0x7fu << (i % 4 * 8);
  }
  return u32x2{r[0], r[1]};
}

// A vector of a key and one of a value by P lanes (a power of two, eight
// elements a lane).
template <typename T>
__global__ __launch_bounds__(256) void k_append_e4m3(const CodeArgs a, int P) {
  const uint32_t x = blockIdx.x * 256u + threadIdx.x, vec = x / (uint32_t)P;
  const int token = (int)min(vec / (uint32_t)a.Hkv, (uint32_t)a.T), h = (int)(vec % (uint32_t)a.Hkv);
  const int e = (int)(x & (uint32_t)(P - 1)) * 8;
  int b;
  int64_t pos;
  bool ok = find_token(a, token, b, pos) && pos >= 0;
  int pg = 0, at = 0;
  ok = ok && find_slot(a, a.table + (int64_t)b * a.max_pages, (int)pos, a.max_pages * a.page, pg, at);
  float k[8] = {}, v[8] = {};
  if (ok && e < a.d) {
    load8(k, reinterpret_cast<const T*>(a.k.p) + token * a.k.st + h * a.k.sh + e);
    load8(v, reinterpret_cast<const T*>(a.v.p) + token * a.v.st + h * a.v.sh + e);
  }
  int kbyte, vbyte;
  const u32x2 kn = quantise(k, P, kbyte), vn = quantise(v, P, vbyte);
  if (!ok || e >= a.d) return;
  const int64_t to = pg * a.c.sb + h * a.c.sh + at * a.c.st + e;
  *reinterpret_cast<u32x2*>(a.kc + to) = kn;
  *reinterpret_cast<u32x2*>(a.vc + to) = vn;
  if (e == 0) {
    const int64_t s = pg * a.cs.sb + h * a.cs.sh + at * a.cs.st;
    a.ks[s] = (uint8_t)kbyte;
    a.vs[s] = (uint8_t)vbyte;
  }
}

// Eight elements of a key and of a value a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_read_e4m3(const CodeArgs a) {
  const uint32_t cpt = (uint32_t)a.Hkv * (a.d / 8), x = blockIdx.x * 256u + threadIdx.x;
  const int token = (int)min(x / cpt, (uint32_t)a.T), y = (int)(x % cpt), h = y / (a.d / 8), e = (y - h * (a.d / 8)) * 8;
  int b;
  int64_t pos;
  if (!find_token(a, token, b, pos)) return;
  int pg = 0, at = 0;
  const bool ok = pos >= 0 && find_slot(a, a.table + (int64_t)b * a.max_pages, (int)pos, a.max_pages * a.page, pg, at);
  u32x2 k = {}, v = {};
  int kb = 127, vb = 127;
  if (ok) {
    const int64_t from = pg * a.c.sb + h * a.c.sh + at * a.c.st + e, s = pg * a.cs.sb + h * a.cs.sh + at * a.cs.st;
    kb = a.ks[s];
    vb = a.vs[s];
    k = *reinterpret_cast<const u32x2*>(a.kc + from);
    v = *reinterpret_cast<const u32x2*>(a.vc + from);
  }
  constexpr int W = (int)sizeof(T) / 2 * 4;   // words of eight elements
  uint32_t kw[W], vw[W];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    widen<T>(k[i], scale_of(kb), kw + i * W / 2);
    widen<T>(v[i], scale_of(vb), vw + i * W / 2);
  }
  T* ko = reinterpret_cast<T*>(a.k.p) + token * a.k.st + h * a.k.sh + e;
  T* vo = reinterpret_cast<T*>(a.v.p) + token * a.v.st + h * a.v.sh + e;
#pragma unroll
  for (int i = 0; i < W; i += 4) {
    *reinterpret_cast<u32x4*>(reinterpret_cast<uint32_t*>(ko) + i) = u32x4{kw[i], kw[i + 1], kw[i + 2], kw[i + 3]};
    *reinterpret_cast<u32x4*>(reinterpret_cast<uint32_t*>(vo) + i) = u32x4{vw[i], vw[i + 1], vw[i + 2], vw[i + 3]};
  }
}

}  // namespace

hipError_t launch_append_e4m3(const CodeArgs& a, bool bf16, hipStream_t s) {
  int P = 1;
  while (P * 8 < a.d) P *= 2;
  const int64_t n = (int64_t)a.T * a.Hkv * P;
  const unsigned blocks = (unsigned)((n + 255) / 256);
  if (bf16) k_append_e4m3<__bf16><<<blocks, 256, 0, s>>>(a, P);
  else k_append_e4m3<float><<<blocks, 256, 0, s>>>(a, P);
  return hipGetLastError();
}

hipError_t launch_read_e4m3(const CodeArgs& a, bool bf16, hipStream_t s) {
  const int64_t n = (int64_t)a.T * a.Hkv * (a.d / 8);
  const unsigned blocks = (unsigned)((n + 255) / 256);
  if (bf16) k_read_e4m3<__bf16><<<blocks, 256, 0, s>>>(a);
  else k_read_e4m3<float><<<blocks, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lact
