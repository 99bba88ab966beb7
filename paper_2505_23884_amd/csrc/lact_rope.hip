// Norm of queries and keys for each head with the position rotation, and its
// reverse: y = R(pos) (w o x r), r = 1 / sqrt(mean(x^2) + eps), with R a
// rotation of pairs of the first `rot` elements by pos freq_i.
//
//   u = r x,  g = R(-pos) dy,  n = w o g,  dx = r (n - u <u, n> / d),  dw = sum g o u
//
// Bound by HBM: x is read and y written once (the reverse reads x and dy and
// writes dx). A workgroup takes `tb` tokens of q's heads or of k's: their
// angles are computed once, in fp64 (a position of 10^5 times a frequency
// keeps 10^-11 of a turn) reduced to a fraction of a turn, into LDS, and used
// by all heads. A group of lanes owns a vector; a lane holds two pieces of GE
// elements that rotate into each other, so nothing is exchanged but the sum of
// squares. [4, 8191, 16 + 4, 128] bf16: 101 us for 336 MB (3.3 TB/s, its angles
// and its launch included), the reverse 122 us for 503 MB (4.1 TB/s); a token
// of 64 sequences 4.4 us.
#include <algorithm>

#include "lact_attn.h"
#include "lact_internal.h"

namespace lact {
namespace {

using namespace attn;

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 16;     // most tokens a step

// GE elements as they lie in memory, and as floats.
template <typename T, int GE>
struct Raw {
  static_assert(sizeof(T) == 2 || GE == 4, "fp32 pieces are 16 bytes");
  static constexpr int N = GE * (int)sizeof(T) / 4;
  uint32_t u[N];
  __device__ __forceinline__ void load(const T* p, bool ok) {
    if constexpr (N == 4) {
      const u32x4 v = ok ? *reinterpret_cast<const u32x4*>(p) : u32x4{};
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = v[i];
    } else {
      const u32x2 v = ok ? *reinterpret_cast<const u32x2*>(p) : u32x2{};
      u[0] = v[0];
      u[1] = v[1];
    }
  }
  __device__ __forceinline__ void get(float (&x)[GE]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 4) {
        x[i] = __uint_as_float(u[i]);
      } else {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
      }
    }
  }
};

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

// cos and sin of a lane's pairs, for the token whose rot / 2 (cos, sin) pairs
// are at cs, and the rotation of its pieces by them (by -angle with s = -1).
template <int GE>
struct Angles {
  float c[GE], s[GE];   // half-split: pair i; interleaved: pair i / 2 of piece i % 2 ...
  __device__ __forceinline__ void load(const RopeArgs& a, const Pieces<GE>& pc, const f32x2* cs) {
#pragma unroll
    for (int i = 0; i < GE; ++i) {
      // interleaved: pairs 0 .. GE / 2 - 1 are piece 0's, the rest piece 1's
      const int k = i / (GE / 2), e = pc.e[k] + 2 * (i % (GE / 2));
      const bool on = a.interleaved ? e < a.rot : pc.turned;
      const f32x2 t = on ? cs[a.interleaved ? e >> 1 : pc.e[0] + i] : f32x2{1.0f, 0.0f};
      c[i] = t[0];
      s[i] = t[1];
    }
  }
  __device__ __forceinline__ void turn(const RopeArgs& a, const Pieces<GE>& pc, float (&x)[2][GE], float sign) const {
    if (pc.turned) {
#pragma unroll
      for (int i = 0; i < GE; ++i) {
        const float u = x[0][i], v = x[1][i], sn = sign * s[i];
        x[0][i] = u * c[i] - v * sn;
        x[1][i] = v * c[i] + u * sn;
      }
    } else if (a.interleaved) {
#pragma unroll
      for (int i = 0; i < GE; ++i) {
        const int k = i / (GE / 2), e = 2 * (i % (GE / 2));
        if (pc.e[k] + e >= a.rot) continue;
        const float u = x[k][e], v = x[k][e + 1], sn = sign * s[i];
        x[k][e] = u * c[i] - v * sn;
        x[k][e + 1] = v * c[i] + u * sn;
      }
    }
  }
};

// cos and sin of tokens t0 .. of the step into cs[token][rot / 2]
__device__ __forceinline__ void angles(const RopeArgs& a, f32x2* cs, int64_t t0, int count) {
  const uint32_t half = (uint32_t)a.rot / 2;
  for (uint32_t x = threadIdx.x; x < count * half; x += kRopeThreads) {
    const uint32_t t = (uint32_t)t0 + x / half;   // B n <= 2^25
    const double pos = a.pos ? (double)a.pos[t] : (double)(a.pos0 + t % (uint32_t)a.n);
    const double turns = pos * (a.freq[x % half] * 0.15915494309189533577);   // 1 / (2 pi)
    const float part = 2.0f * (float)(turns - rint(turns));
    float s, c;
    sincospif(part, &s, &c);
    cs[x] = f32x2{c, s};
  }
}

// Sum over the G lanes of a group (a power of two): within 16 lanes by DPP,
// an instruction a step.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float group_add(float v, int G) {
  if (G >= 2) v = dpp_add<0xb1>(v);    // lanes 1 apart
  if (G >= 4) v = dpp_add<0x4e>(v);    // 2 apart
  if (G >= 8) v = dpp_add<0x141>(v);   // the other four of eight
  if (G >= 16) v = dpp_add<0x140>(v);  // the other eight of sixteen
  if (G >= 32) v += __shfl_xor(v, 16, 64);
  if (G >= 64) v += __shfl_xor(v, 32, 64);
  return v;
}

// Batch and token of token t.
struct RopeToken {
  int64_t b, l;
  __device__ __forceinline__ RopeToken(const RopeArgs& a, int64_t t) {
    const uint32_t bi = (uint32_t)t / (uint32_t)a.n;   // B n <= 2^25
    b = bi;
    l = (uint32_t)t - bi * (uint32_t)a.n;
  }
  template <typename T>
  __device__ __forceinline__ T* row(const AttnView& v, int h) const {
    return reinterpret_cast<T*>(v.p) + b * v.sb + h * v.sh + l * v.st;
  }
};

template <typename T, int GE>
__device__ __forceinline__ void load_pieces(Raw<T, GE> (&x)[2], const Pieces<GE>& pc, const T* row) {
#pragma unroll
  for (int k = 0; k < 2; ++k) x[k].load(row + pc.e[k], pc.ok[k]);
}

// A lane's weights, 1 without any.
template <int GE>
__device__ __forceinline__ void load_weights(float (&w)[2][GE], const Pieces<GE>& pc, const float* from) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < GE; ++i) w[k][i] = from && pc.ok[k] ? from[pc.e[k] + i] : 1.0f;
}

// A workgroup takes q's heads or k's (the first nblk[0] workgroups q's). Its
// groups stand for tokens gi % tb of the step and for every (groups / tb)-th
// head from gi / tb on: the token's angles stay in registers over the heads.
template <typename T, int GE>
__global__ __launch_bounds__(kRopeThreads) void k_rope(const RopeArgs a, int G) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  f32x2* cs = reinterpret_cast<f32x2*>(smem);
  const int which = (int)blockIdx.x >= a.nblk[0], blk = blockIdx.x - (which ? a.nblk[0] : 0);
  const int hs = a.hs[which], H = a.H[which];
  const int64_t tokens = (int64_t)a.B * a.n, t0 = (int64_t)(blk / hs) * a.tb;
  const int count = (int)(tokens - t0 < a.tb ? tokens - t0 : a.tb);
  const int part = blk % hs, h0 = H * part / hs, h1 = H * (part + 1) / hs;
  const int lg = threadIdx.x & (G - 1), NG = kRopeThreads / G, gi = threadIdx.x / G;
  const int ti = gi & (a.tb - 1), step = NG / a.tb;
  const Pieces<GE> pc(a, lg);
  const RopeToken at(a, t0 + min(ti, count - 1));
  const AttnView &xv = a.x[which], &yv = a.y[which];
  int h = h0 + gi / a.tb;
  Raw<T, GE> next[2];   // the loads run one vector ahead, the first beside the angles
  if (h < h1) load_pieces<T, GE>(next, pc, at.row<const T>(xv, h));
  float w[2][GE];
  if (!a.per_head) load_weights<GE>(w, pc, a.w[which]);
  angles(a, cs, t0, count);
  __syncthreads();
  if (ti >= count) return;
  Angles<GE> an;
  an.load(a, pc, cs + ti * (a.rot / 2));
  for (; h < h1; h += step) {
    float x[2][GE];
    next[0].get(x[0]);
    next[1].get(x[1]);
    if (h + step < h1) load_pieces<T, GE>(next, pc, at.row<const T>(xv, h + step));
    if (a.per_head) load_weights<GE>(w, pc, a.w[which] ? a.w[which] + (int64_t)h * a.d : nullptr);
    float ss = 0.0f;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < GE; ++i) ss += x[k][i] * x[k][i];
    const float r = 1.0f / sqrtf(group_add(ss, G) / (float)a.d + a.eps);
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < GE; ++i) x[k][i] *= r * w[k][i];
    an.turn(a, pc, x, 1.0f);
    T* dst = at.row<T>(yv, h);
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (pc.ok[k]) store_piece<T, GE>(dst + pc.e[k], x[k]);
  }
}

// One vector of the reverse: dx to its place, and its part of dw added to acc.
template <typename T, int GE>
__device__ __forceinline__ void rope_back(const RopeArgs& a, const Pieces<GE>& pc, const Angles<GE>& an,
                                          const RopeToken& at, int which, int h, int G, const float (&w)[2][GE],
                                          float (&acc)[2][GE], const Raw<T, GE> (&rx)[2], const Raw<T, GE> (&rg)[2]) {
  float x[2][GE], g[2][GE], n[2][GE];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    rx[k].get(x[k]);
    rg[k].get(g[k]);
  }
  an.turn(a, pc, g, -1.0f);
  float ss = 0.0f, dot = 0.0f;
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < GE; ++i) {
      n[k][i] = g[k][i] * w[k][i];
      ss += x[k][i] * x[k][i];
      dot += x[k][i] * n[k][i];
    }
  const float r = 1.0f / sqrtf(group_add(ss, G) / (float)a.d + a.eps);
  const float c = r * group_add(dot, G) / (float)a.d;   // of u, not of x: r^3 leaves fp32's range where x and r do not
  T* dst = at.row<T>(a.dx[which], h);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int i = 0; i < GE; ++i) {
      const float u = x[k][i] * r;
      acc[k][i] += g[k][i] * u;
      n[k][i] = r * (n[k][i] - c * u);
    }
    if (pc.ok[k]) store_piece<T, GE>(dst + pc.e[k], n[k]);
  }
}

// The reverse. dw is summed per lane over the vectors of its group, over the
// groups of the workgroup through LDS, and over the workgroups by
// k_rope_dw_sum, all in a fixed order. With a weight per head (PER_HEAD) the
// heads are the outer loop, each head's sum is written as it ends, and the
// angles are worked out again for each ([4, 8191, 16 + 4, 128] bf16: 236 us, with
// one weight for all heads 129).
template <typename T, int GE, bool PER_HEAD>
__global__ __launch_bounds__(kRopeThreads) void k_rope_bwd(const RopeArgs a, int G) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  f32x2* cs = reinterpret_cast<f32x2*>(smem);
  float* red = reinterpret_cast<float*>(smem + (size_t)a.tb * (a.rot / 2) * 8);   // [NG][d]
  const int which = (int)blockIdx.x >= a.nblk[0], blk = blockIdx.x - (which ? a.nblk[0] : 0);
  const int H = a.H[which];
  const int64_t tokens = (int64_t)a.B * a.n, stride = (int64_t)a.nblk[which] * a.tb;
  const int lg = threadIdx.x & (G - 1), NG = kRopeThreads / G, gi = threadIdx.x / G;
  const int ti = gi & (a.tb - 1), step = NG / a.tb;
  const Pieces<GE> pc(a, lg);
  float acc[2][GE] = {}, w[2][GE];
  // the workgroup's sums to `to`
  auto flush = [&](float* to) {
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < GE; ++i) {
        if (pc.ok[k]) red[gi * a.d + pc.e[k] + i] = acc[k][i];
        acc[k][i] = 0.0f;
      }
    __syncthreads();
    for (int e = threadIdx.x; e < a.d; e += kRopeThreads) {
      float sum = 0.0f;
      for (int g = 0; g < NG; ++g) sum += red[g * a.d + e];
      to[e] = sum;
    }
  };
  // partials: q's workgroups, then k's, PER_HEAD [head][d] each
  float* part = a.part + ((int64_t)(which ? a.nblk[0] : 0) * (PER_HEAD ? a.H[0] : 1) + (int64_t)blk * (PER_HEAD ? H : 1)) * a.d;
  auto tokens_of = [&](int64_t t0) { return (int)(tokens - t0 < a.tb ? tokens - t0 : a.tb); };
  if constexpr (PER_HEAD) {
    for (int h = 0; h < H; ++h) {
      load_weights<GE>(w, pc, a.w[which] ? a.w[which] + (int64_t)h * a.d : nullptr);
      for (int64_t t0 = (int64_t)blk * a.tb; t0 < tokens; t0 += stride) {
        const int count = tokens_of(t0);
        __syncthreads();
        angles(a, cs, t0, count);
        __syncthreads();
        if (gi >= count) continue;
        Angles<GE> an;
        an.load(a, pc, cs + gi * (a.rot / 2));
        const RopeToken at(a, t0 + gi);
        Raw<T, GE> x[2], g[2];
        load_pieces<T, GE>(x, pc, at.row<const T>(a.x[which], h));
        load_pieces<T, GE>(g, pc, at.row<const T>(a.y[which], h));
        rope_back<T, GE>(a, pc, an, at, which, h, G, w, acc, x, g);
      }
      if (a.dw[which]) flush(part + (int64_t)h * a.d);
    }
  } else {
    load_weights<GE>(w, pc, a.w[which]);
    for (int64_t t0 = (int64_t)blk * a.tb; t0 < tokens; t0 += stride) {
      const int count = tokens_of(t0);
      __syncthreads();
      angles(a, cs, t0, count);
      __syncthreads();
      if (ti >= count) continue;
      Angles<GE> an;
      an.load(a, pc, cs + ti * (a.rot / 2));
      const RopeToken at(a, t0 + ti);
      int h = gi / a.tb;
      Raw<T, GE> nx[2], ng[2];   // the loads run one vector ahead
      auto load = [&](int head) {
        load_pieces<T, GE>(nx, pc, at.row<const T>(a.x[which], head));
        load_pieces<T, GE>(ng, pc, at.row<const T>(a.y[which], head));
      };
      if (h < H) load(h);
      for (; h < H; h += step) {
        Raw<T, GE> x[2], g[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          x[k] = nx[k];
          g[k] = ng[k];
        }
        if (h + step < H) load(h + step);
        rope_back<T, GE>(a, pc, an, at, which, h, G, w, acc, x, g);
      }
    }
    if (a.dw[which]) flush(part);
  }
}

// dw[i] = the sum of the workgroups' partials in a fixed order: 16 columns a
// workgroup, 64 rows of partials a time; q's weights, then k's.
struct RopeSum {
  const float* part[2];
  float* dw[2];
  int nblk[2], n[2], groups;   // workgroups of q's weights
};
__global__ __launch_bounds__(1024) void k_rope_dw_sum(const RopeSum a) {
  __shared__ float red[64][16];
  const int which = (int)blockIdx.x >= a.groups, n = a.n[which], nblk = a.nblk[which];
  const int x = threadIdx.x & 15, r = threadIdx.x >> 4, col = (blockIdx.x - (which ? a.groups : 0)) * 16 + x;
  const float* part = a.part[which] + col;
  float s = 0.0f;
  if (col < n)
#pragma unroll 4
    for (int i = r; i < nblk; i += 64) s += part[(int64_t)i * n];
  red[r][x] = s;
  __syncthreads();
  for (int o = 32; o > 0; o >>= 1) {
    if (r < o) red[r][x] += red[r + o][x];
    __syncthreads();
  }
  if (r == 0 && col < n) a.dw[which][col] = red[0][x];
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
  const int groups = kRopeThreads / lanes(a, piece(a, bf16));
  a.tb = 1;
  // more tokens a step where there are enough of them for every CU's workgroups,
  // sooner where q's heads leave groups idle ([7, 521, 8 + 2, 64], both directions:
  // 36 us; by 2 tokens 50)
  while (a.tb * 2 <= std::min(kRopeTokens, groups) &&
         tokens >= (int64_t)a.tb * (a.tb * 2 * a.H[0] <= groups ? 512 : 2048))
    a.tb *= 2;
  const int64_t steps = (tokens + a.tb - 1) / a.tb;
  for (int w = 0; w < 2; ++w) {
    a.hs[w] = 1;
    if (bwd) {
      // three workgroups a CU, as many as its registers hold, q's and k's in proportion
      // to the heads ([4, 8191, 16 + 4, 128], both directions: 768 in all 233 us, 1024
      // 247, 2048 239); a partial sum of dw each
      const int share = std::max(1, (int)((int64_t)768 * a.H[w] / (a.H[0] + a.H[1])));
      a.nblk[w] = (int)std::min<int64_t>(steps, share);
    } else {
      // few tokens: their heads over several workgroups, a vector a group at least
      const int64_t most = std::max<int64_t>(1, (int64_t)a.H[w] * a.tb / groups);
      if (steps < 512) a.hs[w] = (int)std::min<int64_t>(most, 512 / std::max<int64_t>(steps, 1));
      a.nblk[w] = (int)(steps * a.hs[w]);   // tokens < 2^31, and hs is 1 beyond 512 steps
    }
  }
}

size_t rope_part_floats(const RopeArgs& a) {
  return ((size_t)a.nblk[0] * (a.per_head ? a.H[0] : 1) + (size_t)a.nblk[1] * (a.per_head ? a.H[1] : 1)) * a.d;
}

hipError_t launch_rope(const RopeArgs& a, bool bf16, hipStream_t s) {
  const size_t lds = (size_t)a.tb * (a.rot / 2) * 8;
  const int ge = piece(a, bf16), G = lanes(a, ge), grid = a.nblk[0] + a.nblk[1];
  if (!bf16) k_rope<float, 4><<<grid, kRopeThreads, lds, s>>>(a, G);
  else if (ge == 8) k_rope<__bf16, 8><<<grid, kRopeThreads, lds, s>>>(a, G);
  else k_rope<__bf16, 4><<<grid, kRopeThreads, lds, s>>>(a, G);
  return hipGetLastError();
}

template <typename T, int GE>
static void bwd_one(const RopeArgs& a, int G, hipStream_t s) {
  const size_t lds = (size_t)a.tb * (a.rot / 2) * 8 + (size_t)(kRopeThreads / G) * a.d * 4;
  const int grid = a.nblk[0] + a.nblk[1];
  if (a.per_head) k_rope_bwd<T, GE, true><<<grid, kRopeThreads, lds, s>>>(a, G);
  else k_rope_bwd<T, GE, false><<<grid, kRopeThreads, lds, s>>>(a, G);
}

hipError_t launch_rope_bwd(const RopeArgs& a, bool bf16, hipStream_t s) {
  const int ge = piece(a, bf16), G = lanes(a, ge);
  if (a.nblk[0] > 0) {
    if (!bf16) bwd_one<float, 4>(a, G, s);
    else if (ge == 8) bwd_one<__bf16, 8>(a, G, s);
    else bwd_one<__bf16, 4>(a, G, s);
  }
  RopeSum sum{};
  const float* part = a.part;
  int grid = 0;
  for (int w = 0; w < 2; ++w) {
    const int n = (a.per_head ? a.H[w] : 1) * a.d;
    sum.part[w] = part;
    sum.dw[w] = a.dw[w];
    sum.nblk[w] = a.nblk[w];
    sum.n[w] = n;
    part += (size_t)a.nblk[w] * n;
    if (a.dw[w]) grid += (n + 15) / 16;
    if (w == 0) sum.groups = grid;
  }
  if (grid) k_rope_dw_sum<<<grid, 1024, 0, s>>>(sum);
  return hipGetLastError();
}

}  // namespace lact
