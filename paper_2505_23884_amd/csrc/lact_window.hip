// Softmax attention with a sliding window and first tokens that stay visible
// (sinks), and its reverse.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(c q_i . k_j - lse_i) over the visible j
//   dv_j = sum_i p_ij do_i,  ds_ij = p_ij (do_i . v_j - delta_i),
//   delta_i = do_i . o_i,  dq_i = c sum_j ds_ij k_j,  dk_j = c sum_i ds_ij q_i
//
// Bound by the matrix cores: 4 d flops a visible pair forward, 10 d in the
// reverse; memory traffic is q, k, v and o once where the tiles of one head
// share an L2. Only tiles of keys that some query of the workgroup sees are
// visited, and only those at the edges of the window, at the diagonal and at
// the sequence's end are masked element by element.
#include <algorithm>
#include <type_traits>

#include "lact_attn.h"
#include "lact_internal.h"

namespace lact {
namespace {

using namespace attn;

// Consecutive work on one XCD: workgroups go round the 8 XCDs in turn, so
// workgroup b takes item (b % 8) * (n / 8) + ..., and the tiles of one head
// meet their keys in one L2.
__device__ __forceinline__ int xcd_order(int b, int n) {
  const int x = b & 7, per = n >> 3, extra = n & 7;
  return x * per + (x < extra ? x : extra) + (b >> 3);
}

template <typename T>
__device__ __forceinline__ T* row_of(const AttnView& v, int b, int h, int64_t t) {
  return reinterpret_cast<T*>(v.p) + b * v.sb + h * v.sh + t * v.st;
}

__device__ __forceinline__ int length_of(const WindowArgs& a, int b) {
  return a.len ? min(max(a.len[b], 0), a.n_kv) : a.n_kv;
}

template <typename T, int DP> constexpr int key_tile() { return sizeof(T) == 2 && DP <= 128 ? 64 : 32; }

// ------------------------------------------------------------------ forward
// A workgroup of NW waves owns 32 NW queries of one head, a wave 32 of them;
// keys and values pass through LDS in two stages. Scores are held transposed
// (lact_attn.h), so the softmax needs one exchange between lanes a tile.
template <typename T, int DP, int NW, int OCC>
__global__ __launch_bounds__(64 * NW, OCC) void k_window_fwd(const WindowArgs a) {
  constexpr int KT = key_tile<T, DP>(), QB = 32 * NW, NT = 64 * NW;
  using L = Tile<T, DP>;
  constexpr int BYTES = KT * L::PITCH;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * BYTES];
  const int ntile = (a.n_q + QB - 1) / QB;
  const int w = xcd_order(blockIdx.x, gridDim.x);
  const int bh = w / ntile, qt = ntile - 1 - w % ntile;   // the longest rows of a causal head first
  const int b = bh / a.H, h = bh % a.H, hk = h / a.G;
  const int len = length_of(a, b);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r0 = qt * QB, i = r0 + 32 * wave + (lane & 31);
  const int last = min(a.n_q, len - a.q_start) - 1;       // the last query of the sequence
  const int p = a.q_start + i;
  const bool live = i <= last;
  const KeyTiles kt(a, len, a.q_start + r0, a.q_start + min(r0 + QB - 1, last), KT);
  const int wa = a.q_start + r0 + 32 * wave, wb = a.q_start + min(r0 + 32 * wave + 31, last);
  const int jlo = p - a.win + 1, jhi = live ? min(p + a.look, len - 1) : -1;

  u32x4 q[L::KS];
  load_row<T, DP>(q, row_of<T>(a.q, b, h, min(i, a.n_q - 1)), live, a.d);
  Softmax<DP / 32> st;
  st.init();
  const float c = a.scale * kLog2e;
  const int n = kt.count();
  const int ldk = (int)(a.k.st * sizeof(T)), ldv = (int)(a.v.st * sizeof(T));
  Stage<T, DP, KT, NT> sk, sv;
  auto load = [&](int x) {
    const int k0 = kt.tile(x) * KT;
    sk.load(row_of<T>(a.k, b, hk, k0), ldk, len - k0, a.d);
    sv.load(row_of<T>(a.v, b, hk, k0), ldv, len - k0, a.d);
  };
  auto store = [&](int stage) {
    sk.store(smem + stage * 2 * BYTES);
    sv.store(smem + stage * 2 * BYTES + BYTES);
  };
  if (n > 0) {
    load(0);
    store(0);
  }
  __syncthreads();
  for (int x = 0; x < n; ++x) {
    const uint8_t* ks = smem + (x & 1) * 2 * BYTES;
    if (x + 1 < n) load(x + 1);
    const int k0 = kt.tile(x) * KT;
    const int what = sees(a, len, wa, wb, k0, KT);
    if (what == 2)
      softmax_tile<T, DP, KT, false>(st, q, ks, ks + BYTES, c, [](int) { return true; });
    else if (what == 1)
      softmax_tile<T, DP, KT, true>(st, q, ks, ks + BYTES, c, [&](int j) {
        const int key = k0 + j;
        return key <= jhi && (key >= jlo || key < a.sinks);
      });
    if (x + 1 < n) store((x + 1) & 1);
    __syncthreads();
  }
  const float l = half_sum(st.l);
  const bool none = !live || l == 0.0f;   // a row that sees nothing: 0, lse -inf
  if (i < a.n_q) {
    if (a.lse && lane < 32)
      a.lse[(int64_t)bh * a.n_q + i] = none ? neg_inf() : (st.m + __builtin_amdgcn_logf(l)) * kLn2;
  }
  store_row<T, DP / 32>(row_of<T>(a.o, b, h, min(i, a.n_q - 1)), st.o, 1.0f / l, 0, a.d, i < a.n_q, none);
}

// ------------------------------------------------------------------ reverse
// lse2 and delta, once per query: G lanes a row.
template <typename T>
__global__ __launch_bounds__(256) void k_window_delta(const WindowBwdArgs g, int G) {
  const WindowArgs& a = g.f;
  constexpr int E = 16 / (int)sizeof(T);
  const int lg = threadIdx.x & (G - 1);
  const int64_t rows = (int64_t)a.B * a.H * a.n_q, r = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
  if (r >= rows) return;   // whole groups
  const int64_t bh = r / a.n_q;
  const int b = (int)(bh / a.H), h = (int)(bh % a.H);
  const int64_t i = r - bh * a.n_q;
  float sum = 0.0f;
  for (int e = lg * E; e < a.d; e += G * E) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(row_of<T>(a.o, b, h, i) + e);
    const u32x4 y = *reinterpret_cast<const u32x4*>(row_of<T>(g.dout, b, h, i) + e);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 2)
        sum += __uint_as_float(x[k] << 16) * __uint_as_float(y[k] << 16) +
               __uint_as_float(x[k] & 0xffff0000u) * __uint_as_float(y[k] & 0xffff0000u);
      else
        sum += __uint_as_float(x[k]) * __uint_as_float(y[k]);
    }
  }
  for (int o = G >> 1; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if (lg == 0) {
    const float l = a.lse[r];
    g.lse2[r] = l == neg_inf() ? __builtin_inff() : l * kLog2e;   // weights of an empty row: exp2(-inf) = 0
    g.delta[r] = sum;
  }
}

// dq: queries stay in registers with their cotangents, keys and values pass
// through LDS as in the forward.
template <typename T, int DP, int NW, int OCC>
__global__ __launch_bounds__(64 * NW, OCC) void k_window_dq(const WindowBwdArgs g) {
  const WindowArgs& a = g.f;
  constexpr int KT = key_tile<T, DP>(), QB = 32 * NW, NT = 64 * NW;
  using L = Tile<T, DP>;
  constexpr int BYTES = KT * L::PITCH;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * BYTES];
  const int ntile = (a.n_q + QB - 1) / QB;
  const int w = xcd_order(blockIdx.x, gridDim.x);
  const int bh = w / ntile, qt = ntile - 1 - w % ntile;
  const int b = bh / a.H, h = bh % a.H, hk = h / a.G;
  const int len = length_of(a, b);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int r0 = qt * QB, i = r0 + 32 * wave + (lane & 31), ic = min(i, a.n_q - 1);
  const int last = min(a.n_q, len - a.q_start) - 1;
  const int p = a.q_start + i;
  const bool live = i <= last;
  const KeyTiles kt(a, len, a.q_start + r0, a.q_start + min(r0 + QB - 1, last), KT);
  const int wa = a.q_start + r0 + 32 * wave, wb = a.q_start + min(r0 + 32 * wave + 31, last);
  const int jlo = p - a.win + 1, jhi = live ? min(p + a.look, len - 1) : -1;

  u32x4 q[L::KS], go[L::KS];
  load_row<T, DP>(q, row_of<T>(a.q, b, h, ic), live, a.d);
  load_row<T, DP>(go, row_of<T>(g.dout, b, h, ic), live, a.d);
  const float lse2 = live ? g.lse2[(int64_t)bh * a.n_q + ic] : __builtin_inff();
  const float delta = live ? g.delta[(int64_t)bh * a.n_q + ic] : 0.0f;
  f32x16 dq[DP / 32];
#pragma unroll
  for (int x = 0; x < DP / 32; ++x) dq[x] = f32x16{};
  const float c = a.scale * kLog2e;
  const int n = kt.count();
  const int ldk = (int)(a.k.st * sizeof(T)), ldv = (int)(a.v.st * sizeof(T));
  Stage<T, DP, KT, NT> sk, sv;
  auto load = [&](int x) {
    const int k0 = kt.tile(x) * KT;
    sk.load(row_of<T>(a.k, b, hk, k0), ldk, len - k0, a.d);
    sv.load(row_of<T>(a.v, b, hk, k0), ldv, len - k0, a.d);
  };
  auto store = [&](int stage) {
    sk.store(smem + stage * 2 * BYTES);
    sv.store(smem + stage * 2 * BYTES + BYTES);
  };
  auto step = [&](const uint8_t* ks, int k0, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
#pragma unroll
    for (int mb = 0; mb < KT / 32; ++mb) {
      f32x16 s, dp;
      mma_dot<T, DP>(s, ks, 32 * mb, q);
      mma_dot<T, DP>(dp, ks + BYTES, 32 * mb, go);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float ds = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -lse2)) * (dp[e] - delta);
        if constexpr (MASKED) {
          const int key = k0 + 32 * mb + 8 * (e >> 2) + 4 * half + (e & 3);
          s[e] = key <= jhi && (key >= jlo || key < a.sinks) ? ds : 0.0f;
        } else {
          s[e] = ds;
        }
      }
      const RowsB<T> wb(s);
#pragma unroll
      for (int db = 0; db < DP / 32; ++db) mma_rows<T, DP, MASKED>(dq[db], wb, ks, 32 * mb, db);
    }
  };
  using Yes = std::true_type;
  using No = std::false_type;
  if (n > 0) {
    load(0);
    store(0);
  }
  __syncthreads();
  for (int x = 0; x < n; ++x) {
    const uint8_t* ks = smem + (x & 1) * 2 * BYTES;
    if (x + 1 < n) load(x + 1);
    const int k0 = kt.tile(x) * KT;
    const int what = sees(a, len, wa, wb, k0, KT);
    if (what == 2) step(ks, k0, No{});
    else if (what == 1) step(ks, k0, Yes{});
    if (x + 1 < n) store((x + 1) & 1);
    __syncthreads();
  }
  store_row<T, DP / 32>(row_of<T>(g.dq, b, h, ic), dq, a.scale, 0, a.d, i < a.n_q, !live);
}

// The job of a workgroup of k_window_dkv.
struct DkvJob {
  int tile, part, head_part, slot;   // slot < 0: the sums go to dk and dv
  int qa, qb;                        // queries [qa, qb)
  __device__ __forceinline__ DkvJob(const WindowArgs& a, const DkvPlan& pl, int len, int x) {
    head_part = x % pl.gs;
    x /= pl.gs;
    const bool sink = x < pl.st * pl.np_s;
    const int np = sink ? pl.np_s : pl.np_a, ch = sink ? pl.ch_s : pl.ch_a;
    if (!sink) x -= pl.st * pl.np_s;
    tile = x / np + (sink ? 0 : pl.st);
    part = x % np;
    const int before = sink || pl.np_s * pl.gs <= 1 ? 0 : pl.st * pl.np_s * pl.gs;
    slot = np * pl.gs > 1 ? before + (((sink ? tile : tile - pl.st) * np) + part) * pl.gs + head_part : -1;
    const int k0 = tile * pl.kb, k1 = min(k0 + pl.kb, len) - 1;   // keys k0 .. k1
    const int last = min(a.n_q, len - a.q_start);                  // queries of the sequence
    // j <= p + look and (p < j + win or j < sinks), p = q_start + i
    int ia = max(0, k0 - a.look - a.q_start);
    int ib = k0 < a.sinks ? last : min(last, k1 + a.win - a.q_start);
    if (k0 > k1) ib = ia;
    qa = ia + part * ch;
    qb = part == np - 1 ? ib : min(ib, qa + ch);
  }
};

// dk and dv: 32 keys and values a wave stay in registers, queries and
// cotangents pass through LDS, over every head that shares the keys. DO
// columns of dk and dv a workgroup (DP, or less where both would not fit the
// registers: the scores are then computed again for each part).
template <typename T, int DP, int DO, int QT, int NW>
__global__ __launch_bounds__(64 * NW) void k_window_dkv(const WindowBwdArgs g) {
  const WindowArgs& a = g.f;
  constexpr int KB = 32 * NW, NT = 64 * NW, NB = DO / 32;
  using L = Tile<T, DP>;
  constexpr int BYTES = QT * L::PITCH, STAGE = 2 * BYTES + 2 * QT * 4;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * STAGE];
  const int jobs = g.plan.jobs(), ND = DP / DO;
  const int w = xcd_order(blockIdx.x, gridDim.x);
  const int dsel = w % ND, bk = (w / ND) / jobs, b = bk / a.Hkv, hk = bk % a.Hkv;
  const int len = length_of(a, b);
  const DkvJob job(a, g.plan, len, (w / ND) % jobs);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int kw = job.tile * KB + 32 * wave, j = kw + (lane & 31), jc = min(j, a.n_kv - 1);
  const bool live = j < len;
  // positions that see key j
  const int plo = j - a.look, phi = !live ? -1 : (j < a.sinks ? len - 1 : min(len - 1, j + a.win - 1));
  const int iend = min(a.n_q, len - a.q_start);   // queries past it are padding

  u32x4 kf[L::KS], vf[L::KS];
  load_row<T, DP>(kf, row_of<T>(a.k, b, hk, jc), live, a.d);
  load_row<T, DP>(vf, row_of<T>(a.v, b, hk, jc), live, a.d);
  f32x16 dk[NB], dv[NB];
#pragma unroll
  for (int x = 0; x < NB; ++x) dk[x] = dv[x] = f32x16{};
  const float c = a.scale * kLog2e;
  const int steps = job.qb > job.qa ? (job.qb - job.qa + QT - 1) / QT : 0;
  const int gh = a.G / g.plan.gs, n = steps * gh;
  const int ldq = (int)(a.q.st * sizeof(T)), ldo = (int)(g.dout.st * sizeof(T));
  Stage<T, DP, QT, NT> sq, so;
  float s_lse = 0.0f, s_delta = 0.0f;
  auto load = [&](int x) {
    const int h = hk * a.G + job.head_part * gh + x / steps, i0 = job.qa + (x % steps) * QT;
    sq.load(row_of<T>(a.q, b, h, i0), ldq, job.qb - i0, a.d);
    so.load(row_of<T>(g.dout, b, h, i0), ldo, job.qb - i0, a.d);
    if ((int)threadIdx.x < QT) {
      const int i = i0 + threadIdx.x;
      const int64_t at = ((int64_t)b * a.H + h) * a.n_q + i;
      s_lse = i < job.qb ? g.lse2[at] : __builtin_inff();
      s_delta = i < job.qb ? g.delta[at] : 0.0f;
    }
  };
  auto store = [&](int stage) {
    uint8_t* s = smem + stage * STAGE;
    sq.store(s);
    so.store(s + BYTES);
    if ((int)threadIdx.x < QT) {
      reinterpret_cast<float*>(s + 2 * BYTES)[threadIdx.x] = s_lse;
      reinterpret_cast<float*>(s + 2 * BYTES)[QT + threadIdx.x] = s_delta;
    }
  };
  auto step = [&](const uint8_t* qs, int i0, int rb, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    const uint8_t* os = qs + BYTES;
    const float* rows = reinterpret_cast<const float*>(qs + 2 * BYTES) + rb;
    f32x16 s, dp;
    mma_dot<T, DP>(s, qs, rb, kf);
    mma_dot<T, DP>(dp, os, rb, vf);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4 ls = *reinterpret_cast<const f32x4*>(rows + 8 * e + 4 * half);
      const f32x4 dl = *reinterpret_cast<const f32x4*>(rows + QT + 8 * e + 4 * half);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int r = 4 * e + u;
        float pr = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -ls[u]));
        float ds = pr * (dp[r] - dl[u]);
        if constexpr (MASKED) {
          const int i = i0 + rb + 8 * e + 4 * half + u, p = a.q_start + i;
          const bool see = i < job.qb && p >= plo && p <= phi;
          pr = !see ? 0.0f : pr < kTiny ? kTiny : pr;   // a visible weight stays above zero (mma_rows)
          ds = see ? ds : 0.0f;
        }
        s[r] = pr;
        dp[r] = ds;
      }
    }
    const RowsB<T> wp(s), wd(dp);
#pragma unroll
    for (int x = 0; x < NB; ++x) {
      mma_rows<T, DP, MASKED>(dv[x], wp, os, rb, dsel * NB + x);
      mma_rows<T, DP, MASKED>(dk[x], wd, qs, rb, dsel * NB + x);
    }
  };
  using Yes = std::true_type;
  using No = std::false_type;
  const int kw1 = kw + 31;
  if (n > 0) {
    load(0);
    store(0);
  }
  __syncthreads();
  for (int x = 0; x < n; ++x) {
    const uint8_t* qs = smem + (x & 1) * STAGE;
    if (x + 1 < n) load(x + 1);
    const int i0 = job.qa + (x % steps) * QT;
#pragma unroll
    for (int rb = 0; rb < QT; rb += 32) {
      // the 32 queries against the wave's 32 keys: nothing, something or all
      const int pa = a.q_start + i0 + rb, pe = a.q_start + min(i0 + rb + 32, min(job.qb, iend)) - 1;
      const bool none = pa > pe || kw >= len || kw > pe + a.look || (kw >= a.sinks && kw1 <= pa - a.win);
      const bool all = pe - pa == 31 && kw1 < len && kw1 <= pa + a.look && (kw > pe - a.win || kw1 < a.sinks);
      if (none) continue;
      if (all) step(qs, i0, rb, No{});
      else step(qs, i0, rb, Yes{});
    }
    if (x + 1 < n) store((x + 1) & 1);
    __syncthreads();
  }
  if (job.slot < 0) {
    store_row<T, NB>(row_of<T>(g.dk, b, hk, jc), dk, a.scale, dsel * DO, a.d, j < a.n_kv, !live);
    store_row<T, NB>(row_of<T>(g.dv, b, hk, jc), dv, 1.0f, dsel * DO, a.d, j < a.n_kv, !live);
  } else {
    float* part = g.part + ((int64_t)bk * g.plan.slots() + job.slot) * 2 * KB * a.d + (int64_t)(32 * wave + (lane & 31)) * a.d;
    store_row<float, NB>(part, dk, a.scale, dsel * DO, a.d, true, !live);
    store_row<float, NB>(part + (int64_t)KB * a.d, dv, 1.0f, dsel * DO, a.d, true, !live);
  }
}

// dk and dv of the tiles whose sums came in parts, in the order of the parts:
// four elements a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_window_dkv_sum(const WindowBwdArgs g) {
  const WindowArgs& a = g.f;
  const DkvPlan& pl = g.plan;
  const bool ps = pl.np_s * pl.gs > 1, pa = pl.np_a * pl.gs > 1;
  const int t0 = ps ? 0 : pl.st, t1 = pa ? pl.ntile : pl.st;      // tiles in parts: [t0, t1)
  const int64_t per = (int64_t)(t1 - t0) * pl.kb * (a.d / 4);     // work per (batch, key head)
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (x >= per * a.B * a.Hkv) return;
  const int bk = (int)(x / per), b = bk / a.Hkv, hk = bk % a.Hkv;
  const int64_t y = x - bk * per;
  const int e = (int)(y % (a.d / 4)) * 4, row = (int)(y / (a.d / 4)) % pl.kb, t = t0 + (int)(y / (a.d / 4)) / pl.kb;
  const int64_t j = (int64_t)t * pl.kb + row;
  if (j >= a.n_kv) return;
  const bool sink = t < pl.st;
  const int np = (sink ? pl.np_s : pl.np_a) * pl.gs;
  const int slot = sink ? t * np : (ps ? pl.st * pl.np_s * pl.gs : 0) + (t - pl.st) * np;
  const float* part = g.part + ((int64_t)bk * pl.slots() + slot) * 2 * pl.kb * a.d + (int64_t)row * a.d + e;
  f32x4 k = {}, v = {};
  for (int s = 0; s < np; ++s) {
    k += *reinterpret_cast<const f32x4*>(part + (int64_t)s * 2 * pl.kb * a.d);
    v += *reinterpret_cast<const f32x4*>(part + (int64_t)(s * 2 + 1) * pl.kb * a.d);
  }
  T *ok = row_of<T>(g.dk, b, hk, j) + e, *ov = row_of<T>(g.dv, b, hk, j) + e;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<u32x2*>(ok) = u32x2{pack_bf16(k[0], k[1]), pack_bf16(k[2], k[3])};
    *reinterpret_cast<u32x2*>(ov) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  } else {
    *reinterpret_cast<f32x4*>(ok) = k;
    *reinterpret_cast<f32x4*>(ov) = v;
  }
}

int cdiv(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

template <typename T, int DP>
hipError_t fwd(const WindowArgs& a, hipStream_t s) {
  constexpr int OCC = sizeof(T) == 2 && DP <= 128 ? 2 : 1;
  const int64_t bh = (int64_t)a.B * a.H;
  k_window_fwd<T, DP, 4, OCC><<<(unsigned)(bh * cdiv(a.n_q, 128)), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T, int DP>
hipError_t bwd(const WindowBwdArgs& g, hipStream_t s) {
  const WindowArgs& a = g.f;
  constexpr bool H16 = sizeof(T) == 2;
  constexpr int DO = DP <= 128 ? DP : H16 ? 128 : 64, QT = H16 && DP <= 128 ? 64 : 32;
  const int64_t bh = (int64_t)a.B * a.H, bk = (int64_t)a.B * a.Hkv;
  if (a.n_q > 0) {
    int G = 1;
    while (G < 64 && G * (16 / (int)sizeof(T)) < a.d) G *= 2;
    k_window_delta<T><<<(unsigned)((bh * a.n_q + 256 / G - 1) / (256 / G)), 256, 0, s>>>(g, G);
    k_window_dq<T, DP, 4, 1><<<(unsigned)(bh * cdiv(a.n_q, 128)), 256, 0, s>>>(g);
  }
  if (a.n_kv > 0) {
    k_window_dkv<T, DP, DO, QT, 4><<<(unsigned)(bk * g.plan.jobs() * (DP / DO)), 256, 0, s>>>(g);
    const DkvPlan& pl = g.plan;
    const bool ps = pl.np_s * pl.gs > 1 && pl.st > 0, pa = pl.np_a * pl.gs > 1;
    const int t0 = pl.np_s * pl.gs > 1 ? 0 : pl.st, t1 = pa ? pl.ntile : pl.st;
    if (ps || pa) {
      const int64_t n = (int64_t)(t1 - t0) * pl.kb * (a.d / 4) * bk;
      if (n > 0) k_window_dkv_sum<T><<<(unsigned)((n + 255) / 256), 256, 0, s>>>(g);
    }
  }
  return hipGetLastError();
}

}  // namespace

DkvPlan window_dkv_plan(const WindowArgs& a, bool bf16) {
  DkvPlan p{};
  p.kb = 128;
  p.ntile = cdiv(a.n_kv, p.kb);
  p.st = 0;
  p.np_s = p.np_a = p.gs = 1;
  p.ch_s = p.ch_a = std::max(a.n_q, 1);
  (void)bf16;
  return p;
}

hipError_t launch_window_fwd(const WindowArgs& a, bool bf16, hipStream_t s) {
  if (a.n_q == 0) return hipSuccess;
  if (bf16) return a.d <= 64 ? fwd<__bf16, 64>(a, s) : a.d <= 128 ? fwd<__bf16, 128>(a, s) : fwd<__bf16, 256>(a, s);
  return a.d <= 64 ? fwd<float, 64>(a, s) : a.d <= 128 ? fwd<float, 128>(a, s) : fwd<float, 256>(a, s);
}

hipError_t launch_window_bwd(const WindowBwdArgs& g, bool bf16, hipStream_t s) {
  const int d = g.f.d;
  if (bf16) return d <= 64 ? bwd<__bf16, 64>(g, s) : d <= 128 ? bwd<__bf16, 128>(g, s) : bwd<__bf16, 256>(g, s);
  return d <= 64 ? bwd<float, 64>(g, s) : d <= 128 ? bwd<float, 128>(g, s) : bwd<float, 256>(g, s);
}

}  // namespace lact
