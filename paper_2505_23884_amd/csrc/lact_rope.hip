// Norm of queries and keys for each head with the position rotation, and its
// reverse: y = R(pos) (w o x r), r = 1 / sqrt(mean(x^2) + eps), with R a
// rotation of pairs of the first `rot` elements by pos freq_i.
//
//   g = R(-pos) dy,  n = w o g,  dx = r n - (r^3 / d) x <x, n>,  dw = sum g o x r
//
// Bound by HBM: x is read and y written once (the reverse reads x and dy and
// writes dx). A workgroup takes `tb` tokens of every head: their angles are
// computed once, in fp64 (a position of 10^5 times a frequency keeps 10^-11
// of a turn) reduced to a fraction of a turn, into LDS, and used by all heads.
// A group of lanes owns a vector; a lane holds two pieces of GE elements that
// rotate into each other, so nothing is exchanged but the sum of squares.
#include <algorithm>

#include "lact_attn.h"
#include "lact_internal.h"

namespace lact {
namespace {

using namespace attn;

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 16;     // most tokens a step
constexpr int kRopeMaxD = 512;

template <typename T, int GE>
__device__ __forceinline__ void load_piece(float (&x)[GE], const T* p) {
  if constexpr (sizeof(T) == 4) {
    static_assert(GE == 4, "fp32 pieces are 16 bytes");
    const f32x4 u = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = u[i];
  } else {
    uint32_t u[GE / 2];
    if constexpr (GE == 8) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = v[i];
    } else {
      const u32x2 v = *reinterpret_cast<const u32x2*>(p);
      u[0] = v[0];
      u[1] = v[1];
    }
#pragma unroll
    for (int i = 0; i < GE / 2; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
}

template <typename T, int GE>
__device__ __forceinline__ void store_piece(T* p, const float (&x)[GE]) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
  } else if constexpr (GE == 8) {
    *reinterpret_cast<u32x4*>(p) =
        u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
  } else {
    *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
  }
}

// The two pieces of lane l of a vector's group: elements e[0] .. e[0] + GE - 1
// and e[1] .. (ok: they exist). Half-split rotation: e[1] = e[0] + rot / 2;
// otherwise neighbours.
template <int GE>
struct Pieces {
  int e[2];
  bool ok[2], turned;
  __device__ __forceinline__ Pieces(const RopeArgs& a, int l) {
    const int h = a.interleaved ? 0 : a.rot / 2 / GE;   // lanes whose pieces rotate into each other
    turned = !a.interleaved && l < h;
    e[0] = turned ? l * GE : 2 * h * GE + 2 * (l - h) * GE;
    e[1] = turned ? e[0] + a.rot / 2 : e[0] + GE;
    ok[0] = e[0] < a.d;
    ok[1] = e[1] < a.d;
  }
};

// Rotation of a lane's pieces by the angles of its token (cs: cos, sin pairs
// of the token's rot / 2 frequencies), by -angle with s = -1.
template <int GE>
__device__ __forceinline__ void turn(const RopeArgs& a, const Pieces<GE>& pc, float (&x)[2][GE], const f32x2* cs, float s) {
  if (pc.turned) {
#pragma unroll
    for (int i = 0; i < GE; ++i) {
      const f32x2 t = cs[pc.e[0] + i];
      const float u = x[0][i], v = x[1][i], sn = s * t[1];
      x[0][i] = u * t[0] - v * sn;
      x[1][i] = v * t[0] + u * sn;
    }
  } else if (a.interleaved) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < GE; i += 2) {
        if (pc.e[k] + i >= a.rot) continue;
        const f32x2 t = cs[(pc.e[k] + i) >> 1];
        const float u = x[k][i], v = x[k][i + 1], sn = s * t[1];
        x[k][i] = u * t[0] - v * sn;
        x[k][i + 1] = v * t[0] + u * sn;
      }
  }
}

// cos and sin of tokens t0 .. of the step into cs[token][rot / 2]
__device__ __forceinline__ void angles(const RopeArgs& a, f32x2* cs, int64_t t0, int count) {
  const int half = a.rot / 2;
  for (int x = threadIdx.x; x < count * half; x += kRopeThreads) {
    const int64_t t = t0 + x / half;
    const double pos = a.pos ? (double)a.pos[t] : (double)(a.pos0 + t % a.n);
    const double turns = pos * (a.freq[x % half] * 0.15915494309189533577);   // 1 / (2 pi)
    const float part = 2.0f * (float)(turns - rint(turns));
    float s, c;
    sincospif(part, &s, &c);
    cs[x] = f32x2{c, s};
  }
}

__device__ __forceinline__ float group_add(float v, int G) {
  for (int o = G >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// One token of the step and one head (q's, then k's).
struct RopeAt {
  int which, h;
  int64_t b, l;
  __device__ __forceinline__ RopeAt(const RopeArgs& a, int64_t t, int head) {
    which = head >= a.H[0];
    h = which ? head - a.H[0] : head;
    if (a.B * a.n < ((int64_t)1 << 31)) {
      const uint32_t bi = (uint32_t)t / (uint32_t)a.n;
      b = bi;
      l = (uint32_t)t - bi * (uint32_t)a.n;
    } else {
      b = t / a.n;
      l = t - b * a.n;
    }
  }
  template <typename T>
  __device__ __forceinline__ T* row(const AttnView& v) const {
    return reinterpret_cast<T*>(v.p) + b * v.sb + h * v.sh + l * v.st;
  }
};

template <typename T, int GE>
__global__ __launch_bounds__(kRopeThreads) void k_rope(const RopeArgs a, int G) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  f32x2* cs = reinterpret_cast<f32x2*>(smem);
  const int64_t tokens = (int64_t)a.B * a.n, t0 = (int64_t)(blockIdx.x / a.hs) * a.tb;
  const int count = (int)(tokens - t0 < a.tb ? tokens - t0 : a.tb), heads = a.H[0] + a.H[1];
  const int part = blockIdx.x % a.hs, h0 = heads * part / a.hs, h1 = heads * (part + 1) / a.hs;
  angles(a, cs, t0, count);
  __syncthreads();
  const int lg = threadIdx.x & (G - 1), NG = kRopeThreads / G;
  const Pieces<GE> pc(a, lg);
  for (int v = threadIdx.x / G; v < count * (h1 - h0); v += NG) {
    const int ti = v % count, head = h0 + v / count;
    const RopeAt at(a, t0 + ti, head);
    const T* src = at.row<const T>(a.x[at.which]);
    float x[2][GE];
    float ss = 0.0f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (pc.ok[k]) load_piece<T, GE>(x[k], src + pc.e[k]);
#pragma unroll
      for (int i = 0; i < GE; ++i) {
        if (!pc.ok[k]) x[k][i] = 0.0f;
        ss += x[k][i] * x[k][i];
      }
    }
    const float r = 1.0f / sqrtf(group_add(ss, G) / (float)a.d + a.eps);
    const float* w = a.w[at.which];
    if (w && a.per_head) w += (int64_t)at.h * a.d;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < GE; ++i) x[k][i] *= w && pc.ok[k] ? r * w[pc.e[k] + i] : r;
    turn<GE>(a, pc, x, cs + ti * (a.rot / 2), 1.0f);
    T* dst = at.row<T>(a.y[at.which]);
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (pc.ok[k]) store_piece<T, GE>(dst + pc.e[k], x[k]);
  }
}

// The reverse. dw is summed per lane over the vectors of its group, over the
// groups of the workgroup through LDS, and over the workgroups by
// k_rope_dw_sum, all in a fixed order. With a weight per head the heads are
// the outer loop and each head's sum is written as it ends.
template <typename T, int GE, bool PER_HEAD>
__global__ __launch_bounds__(kRopeThreads) void k_rope_bwd(const RopeArgs a, int G) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  f32x2* cs = reinterpret_cast<f32x2*>(smem);
  float* red = reinterpret_cast<float*>(smem + (size_t)a.tb * (a.rot / 2) * 8);   // [NG][d]
  const int64_t tokens = (int64_t)a.B * a.n;
  const int heads = a.H[0] + a.H[1];
  const int lg = threadIdx.x & (G - 1), NG = kRopeThreads / G, gi = threadIdx.x / G;
  const Pieces<GE> pc(a, lg);
  float acc[PER_HEAD ? 1 : 2][2][GE] = {};
  const bool any_dw = a.dw[0] || a.dw[1];
  // the sums of `which` (q or k), head slot `at` of this workgroup's partials
  auto flush = [&](float (&s)[2][GE], int at) {
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < GE; ++i) {
        if (pc.ok[k]) red[gi * a.d + pc.e[k] + i] = s[k][i];
        s[k][i] = 0.0f;
      }
    __syncthreads();
    const int slots = PER_HEAD ? heads : 2;
    for (int e = threadIdx.x; e < a.d; e += kRopeThreads) {
      float sum = 0.0f;
      for (int g = 0; g < NG; ++g) sum += red[g * a.d + e];
      a.part[((int64_t)blockIdx.x * slots + at) * a.d + e] = sum;
    }
  };
  auto vector = [&](int64_t t, int ti, int head) {
    const RopeAt at(a, t, head);
    const T* src = at.row<const T>(a.x[at.which]);
    const T* gsrc = at.row<const T>(a.y[at.which]);
    float x[2][GE], g[2][GE];
    float ss = 0.0f, dot = 0.0f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (pc.ok[k]) {
        load_piece<T, GE>(x[k], src + pc.e[k]);
        load_piece<T, GE>(g[k], gsrc + pc.e[k]);
      } else {
#pragma unroll
        for (int i = 0; i < GE; ++i) x[k][i] = g[k][i] = 0.0f;
      }
    }
    turn<GE>(a, pc, g, cs + ti * (a.rot / 2), -1.0f);
    const float* w = a.w[at.which];
    if (w && a.per_head) w += (int64_t)at.h * a.d;
    float n[2][GE];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < GE; ++i) {
        n[k][i] = w && pc.ok[k] ? g[k][i] * w[pc.e[k] + i] : g[k][i];
        ss += x[k][i] * x[k][i];
        dot += x[k][i] * n[k][i];
      }
    const float r = 1.0f / sqrtf(group_add(ss, G) / (float)a.d + a.eps);
    const float c = r * r * r * (group_add(dot, G) / (float)a.d);
    T* dst = at.row<T>(a.dx[at.which]);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int i = 0; i < GE; ++i) {
        const float gxr = g[k][i] * x[k][i] * r;
        if (PER_HEAD || !at.which) acc[0][k][i] += gxr;
        else acc[PER_HEAD ? 0 : 1][k][i] += gxr;
        n[k][i] = r * n[k][i] - c * x[k][i];
      }
      if (pc.ok[k]) store_piece<T, GE>(dst + pc.e[k], n[k]);
    }
  };
  if constexpr (PER_HEAD) {
    for (int head = 0; head < heads; ++head) {
      for (int64_t t0 = (int64_t)blockIdx.x * a.tb; t0 < tokens; t0 += (int64_t)gridDim.x * a.tb) {
        const int count = (int)(tokens - t0 < a.tb ? tokens - t0 : a.tb);
        __syncthreads();
        angles(a, cs, t0, count);
        __syncthreads();
        for (int v = gi; v < count; v += NG) vector(t0 + v, v, head);
      }
      if (any_dw) flush(acc[0], head);
    }
  } else {
    for (int64_t t0 = (int64_t)blockIdx.x * a.tb; t0 < tokens; t0 += (int64_t)gridDim.x * a.tb) {
      const int count = (int)(tokens - t0 < a.tb ? tokens - t0 : a.tb);
      __syncthreads();
      angles(a, cs, t0, count);
      __syncthreads();
      for (int v = gi; v < count * heads; v += NG) vector(t0 + v % count, v % count, v / count);
    }
    if (any_dw) {
      flush(acc[0], 0);
      flush(acc[1], 1);
    }
  }
}

// dw[i] = sum over the workgroups' partials, 8 rows of them a time in a fixed
// order; columns [0, n0) go to dw0, the rest to dw1.
__global__ __launch_bounds__(256) void k_rope_dw_sum(const float* part, float* dw0, float* dw1, int nblk, int n0, int n) {
  __shared__ float red[8][32];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), r = threadIdx.x >> 5;
  float s = 0.0f;
  if (col < n)
    for (int x = r; x < nblk; x += 8) s += part[(int64_t)x * n + col];
  red[r][threadIdx.x & 31] = s;
  __syncthreads();
  if (r || col >= n) return;
#pragma unroll
  for (int x = 1; x < 8; ++x) s += red[x][threadIdx.x];
  float* out = col < n0 ? dw0 : dw1;
  if (out) out[col < n0 ? col : col - n0] = s;
}

// Elements of a piece: 16 bytes, or 4 elements where half the rotated ones
// are no multiple of 8.
int piece(const RopeArgs& a, bool bf16) { return bf16 && (a.interleaved || a.rot % 16 == 0) ? 8 : 4; }
int lanes(const RopeArgs& a, int ge) {
  int g = 1;
  while (g * 2 * ge < a.d) g *= 2;
  return g;
}

}  // namespace

void rope_plan(RopeArgs& a, bool bf16, bool bwd) {
  const int64_t tokens = (int64_t)a.B * a.n;
  const int heads = a.H[0] + a.H[1], groups = kRopeThreads / lanes(a, piece(a, bf16));
  a.tb = (int)std::max<int64_t>(1, std::min<int64_t>(kRopeTokens, tokens / 1024));
  const int64_t steps = (tokens + a.tb - 1) / a.tb;
  a.hs = 1;
  if (bwd) {
    a.nblk = (int)std::min<int64_t>(steps, 1024);
  } else {
    // few tokens: their heads over several workgroups, a vector a group at least
    if (steps < 512)
      a.hs = (int)std::max<int64_t>(1, std::min<int64_t>(heads * (int64_t)a.tb / groups, 512 / std::max<int64_t>(steps, 1)));
    a.nblk = (int)std::min<int64_t>(steps * a.hs, 0x7fffffff);
  }
}

size_t rope_part_floats(const RopeArgs& a) {
  return (size_t)a.nblk * (a.per_head ? a.H[0] + a.H[1] : 2) * a.d;
}

hipError_t launch_rope(const RopeArgs& a, bool bf16, hipStream_t s) {
  const size_t lds = (size_t)a.tb * (a.rot / 2) * 8;
  const int ge = piece(a, bf16), G = lanes(a, ge);
  if (!bf16) k_rope<float, 4><<<a.nblk, kRopeThreads, lds, s>>>(a, G);
  else if (ge == 8) k_rope<__bf16, 8><<<a.nblk, kRopeThreads, lds, s>>>(a, G);
  else k_rope<__bf16, 4><<<a.nblk, kRopeThreads, lds, s>>>(a, G);
  return hipGetLastError();
}

template <typename T, int GE>
static void bwd_one(const RopeArgs& a, int G, hipStream_t s) {
  const size_t lds = (size_t)a.tb * (a.rot / 2) * 8 + (size_t)(kRopeThreads / G) * a.d * 4;
  if (a.per_head) k_rope_bwd<T, GE, true><<<a.nblk, kRopeThreads, lds, s>>>(a, G);
  else k_rope_bwd<T, GE, false><<<a.nblk, kRopeThreads, lds, s>>>(a, G);
}

hipError_t launch_rope_bwd(const RopeArgs& a, bool bf16, hipStream_t s) {
  const int ge = piece(a, bf16), G = lanes(a, ge);
  if (a.nblk > 0) {
    if (!bf16) bwd_one<float, 4>(a, G, s);
    else if (ge == 8) bwd_one<__bf16, 8>(a, G, s);
    else bwd_one<__bf16, 4>(a, G, s);
  }
  if (a.dw[0] || a.dw[1]) {
    const int n0 = (a.per_head ? a.H[0] : 1) * a.d, n = n0 + (a.per_head ? a.H[1] : 1) * a.d;
    k_rope_dw_sum<<<(n + 31) / 32, 256, 0, s>>>(a.part, a.dw[0], a.dw[1], a.nblk, n0, n);
  }
  return hipGetLastError();
}

}  // namespace lact
