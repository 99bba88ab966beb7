// Host side of the attention entry points: validation (before any HIP call),
// workspaces and launches. All arithmetic runs in lact_window.hip,
// lact_paged.hip, lact_rope.hip, lact_codes.hip and lact_prefix.hip.
#include <algorithm>

#include "lact.h"
#include "lact_internal.h"

namespace lact {
namespace {

constexpr size_t kWsAlign = 256;
size_t ws_round(size_t x) { return (x + kWsAlign - 1) / kWsAlign * kWsAlign; }
constexpr int64_t kMaxTokenStride = (int64_t)1 << 22;   // 64 rows stay within a 31-bit buffer range
constexpr int64_t kMaxInt = (int64_t)0x7fffffff;
// A launch holds fewer than 2^32 threads in a direction.
// Tokens of a norm and rotation, of q and of k in one launch: four a workgroup
// of 256 at least (vectors of more than 256 elements by pieces of four).
constexpr int64_t kRopeRows = ((int64_t)1 << 25) - 4;
static_assert(2 * (kRopeRows / 4) * 256 < ((int64_t)1 << 32), "threads of a launch");
// Tiles of 128 queries, or keys, over the heads: workgroups of 512 at most
// (fp32 heads of more than 128 take twice that a tile of keys, but then 2^22
// tiles of dk and dv are more than the card holds).
constexpr int64_t kAttnTiles = (int64_t)1 << 23;
constexpr int64_t kPagedRows = (int64_t)1 << 28;      // new tokens times heads, 32 a workgroup of 256
constexpr int64_t kPagedElements = (int64_t)1 << 33;  // four a thread of the append

bool finite(float x) { return x - x == 0.0f; }

// A view of [batch][head][token] vectors of `es`-byte elements: LACT_OK or an
// error. `out`: its vectors must not overlap. `es` 0: bytes, without alignment.
int check_view(const lact_view* v, int64_t batch, int64_t head, int64_t token, int d, int es, bool out) {
  if (!v) return LACT_EINVAL;
  if (!batch || !head || !token) return LACT_OK;
  if (!v->data) return LACT_EINVAL;
  const int64_t ext[3] = {batch, head, token}, st[3] = {v->batch, v->head, v->token};
  for (int i = 0; i < 3; ++i) {
    if (ext[i] == 1) continue;
    if (st[i] < 0) return LACT_EINVAL;
  }
  if (out) {   // from the narrowest stride on, each steps over what lies within it
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int x, int y) { return st[x] < st[y]; });
    __int128 span = d;
    for (int i : order) {
      if (ext[i] == 1) continue;
      if (st[i] < span) return LACT_EINVAL;
      span += (__int128)(ext[i] - 1) * st[i];
    }
  }
  if (es && ((uintptr_t)v->data & 15)) return LACT_EALIGN;
  for (int i = 0; i < 3; ++i)
    if (ext[i] > 1 && st[i] * es % 16) return LACT_EALIGN;
  if (token > 1 && v->token > kMaxTokenStride) return LACT_EUNSUPPORTED;
  return LACT_OK;
}

// Strides of extents of 1 are not used: 0, so that no offset can overflow.
AttnView take(const lact_view* v, int64_t batch, int64_t head, int64_t token) {
  AttnView a{};
  if (!batch || !head || !token) return a;
  a.p = v->data;
  a.sb = batch > 1 ? v->batch : 0;
  a.sh = head > 1 ? v->head : 0;
  a.st = token > 1 ? v->token : 0;
  return a;
}

#define LACT_TRY(x)                 \
  do {                              \
    const int rc_ = (x);            \
    if (rc_ != LACT_OK) return rc_; \
  } while (0)

int check_heads(int32_t B, int32_t H, int32_t Hkv, int32_t d, int32_t io, int max_d) {
  if (B < 1 || H < 1 || Hkv < 1 || d < 1 || H % Hkv) return LACT_EINVAL;
  if (io != LACT_IO_BF16 && io != LACT_IO_FP32) return LACT_EINVAL;
  if (d % 8 || d > max_d || (int64_t)B * H > (1 << 20)) return LACT_EUNSUPPORTED;
  return LACT_OK;
}

int elem(int32_t io) { return io == LACT_IO_BF16 ? 2 : 4; }

// ---------------------------------------------------------------- norm and rotation
int check_rope(const lact_rope_desc* s) {
  if (!s) return LACT_EINVAL;
  LACT_TRY(check_heads(s->B, s->H, s->Hkv, s->d, s->io_dtype, 512));
  if (s->n < 0 || s->rot < 0 || s->rot > s->d || s->rot % 2 || s->reserved) return LACT_EINVAL;
  if ((s->interleaved | s->weight_per_head) & ~1) return LACT_EINVAL;
  if (!(s->eps >= 0.0f) || !finite(s->eps)) return LACT_EINVAL;
  if (!s->interleaved && s->rot % 8) return LACT_EUNSUPPORTED;
  const int64_t far = (int64_t)1 << 40;
  if (s->n > kRopeRows || s->B * s->n > kRopeRows || s->pos0 > far || s->pos0 < -far) return LACT_EUNSUPPORTED;
  return LACT_OK;
}

RopeArgs rope_args(const lact_rope_desc* s, bool bwd) {
  RopeArgs a{};
  a.pos0 = s->pos0;
  a.n = s->n;
  a.B = s->B;
  a.H[0] = s->H;
  a.H[1] = s->Hkv;
  a.d = s->d;
  a.rot = s->rot;
  a.interleaved = s->interleaved != 0;
  a.per_head = s->weight_per_head != 0;
  a.eps = s->eps;
  rope_plan(a, s->io_dtype == LACT_IO_BF16, bwd);
  return a;
}

int rope_common(const lact_rope_desc* s, const lact_view* q, const lact_view* k, const float* wq, const float* wk,
                const double* inv_freq, const int32_t* positions) {
  LACT_TRY(check_rope(s));
  if ((inv_freq != nullptr) != (s->rot > 0)) return LACT_EINVAL;
  const int es = elem(s->io_dtype);
  LACT_TRY(check_view(q, s->B, s->H, s->n, s->d, es, false));
  LACT_TRY(check_view(k, s->B, s->Hkv, s->n, s->d, es, false));
  if (((uintptr_t)wq & 3) || ((uintptr_t)wk & 3) || ((uintptr_t)inv_freq & 7) || ((uintptr_t)positions & 3))
    return LACT_EALIGN;
  return LACT_OK;
}

// ---------------------------------------------------------------- window attention
int check_attn(const lact_attn_desc* s) {
  if (!s) return LACT_EINVAL;
  LACT_TRY(check_heads(s->B, s->H, s->Hkv, s->d, s->io_dtype, 256));
  if (s->n_q < 0 || s->n_kv < 0 || s->window < -1 || s->lookahead < -1 || s->sinks < 0) return LACT_EINVAL;
  if (!(s->scale > 0.0f) || !finite(s->scale)) return LACT_EINVAL;
  if (s->scale < 1e-12f || s->scale > 1e12f) return LACT_EUNSUPPORTED;   // lse / scale stays far from overflow
  if (s->n_q > kAttnTokens || s->n_kv > kAttnTokens || s->q_start > kAttnTokens || s->q_start < -kAttnTokens ||
      s->q_start + s->n_q > kAttnTokens)
    return LACT_EUNSUPPORTED;
  if ((int64_t)s->B * s->H * ((std::max(s->n_q, s->n_kv) + 127) / 128) >= kAttnTiles) return LACT_EUNSUPPORTED;
  return LACT_OK;
}

WindowArgs window_args(const lact_attn_desc* s) {
  const int64_t far = (int64_t)1 << 30;   // beyond every distance of two positions
  WindowArgs a{};
  a.B = s->B;
  a.H = s->H;
  a.Hkv = s->Hkv;
  a.G = s->H / s->Hkv;
  a.d = s->d;
  a.n_q = (int)s->n_q;
  a.n_kv = (int)s->n_kv;
  a.q_start = (int)s->q_start;
  a.win = (int)(s->window < 0 ? far : std::min(s->window, far));
  a.look = (int)(s->lookahead < 0 ? far : std::min(s->lookahead, far));
  a.sinks = (int)std::min(s->sinks, kAttnTokens);
  a.scale = s->scale;
  return a;
}

struct WindowLayout {
  size_t nlse, ndelta, part, total;
};
WindowLayout window_layout(const WindowArgs& a, const DkvPlan& p) {
  WindowLayout l{};
  const size_t rows = ws_round((size_t)a.B * a.H * a.n_q * 4);
  l.ndelta = rows;
  l.part = 2 * rows;
  l.total = l.part + ws_round((size_t)a.B * a.Hkv * p.slots() * 2 * p.kb * a.d * 4);
  return l;
}

// ---------------------------------------------------------------- pages
int check_paged(const lact_paged_desc* s, bool attend) {
  if (!s) return LACT_EINVAL;
  LACT_TRY(check_heads(s->B, attend ? s->H : s->Hkv, s->Hkv, s->d, s->io_dtype, 256));
  if (s->n_new < 0 || s->pages < 0 || s->page < 1 || s->max_pages < 0) return LACT_EINVAL;
  if (attend && (s->window < -1 || s->sinks < 0 || !(s->scale > 0.0f) || !finite(s->scale))) return LACT_EINVAL;
  const int64_t rows = std::min(s->n_new, kAttnTokens) * (attend ? s->H : s->Hkv);
  if (s->pages > kMaxInt || (int64_t)s->max_pages * s->page > kAttnTokens || s->page > kAttnTokens ||
      s->n_new > kAttnTokens || rows > kPagedRows || rows * s->d > kPagedElements)
    return LACT_EUNSUPPORTED;
  return LACT_OK;
}

bool same_strides(const lact_paged_desc* s, const lact_view* x, const lact_view* y) {
  return s->pages == 0 || ((s->pages == 1 || x->batch == y->batch) && (s->Hkv == 1 || x->head == y->head) &&
                           (s->page == 1 || x->token == y->token));
}

int check_cache(const lact_paged_desc* s, int es, const lact_view* kc, const lact_view* vc, const int32_t* table,
                const int32_t* lens, const int32_t* cu, bool out) {
  LACT_TRY(check_view(kc, s->pages, s->Hkv, s->page, s->d, es, out));
  LACT_TRY(check_view(vc, s->pages, s->Hkv, s->page, s->d, es, out));
  if (!same_strides(s, kc, vc)) return LACT_EINVAL;
  if (!lens || !cu || (s->max_pages > 0 && !table)) return LACT_EINVAL;
  if (((uintptr_t)table & 3) || ((uintptr_t)lens & 3) || ((uintptr_t)cu & 3)) return LACT_EALIGN;
  return LACT_OK;
}

void fill_paged(PagedArgs& a, const lact_paged_desc* s) {
  const int64_t far = (int64_t)1 << 30;
  a.B = s->B;
  a.H = s->H;
  a.Hkv = s->Hkv;
  a.G = s->H / s->Hkv;
  a.d = s->d;
  a.T = (int)s->n_new;
  a.page = s->page;
  a.max_pages = s->pages > 0 ? s->max_pages : 0;
  a.pages = (int)s->pages;
  a.win = (int)(s->window < 0 ? far : std::min(s->window, far));
  a.look = 0;
  a.sinks = (int)std::min(s->sinks, kAttnTokens);
  a.scale = s->scale;
  divider(s->page, &a.mul, &a.shift);
}
PagedArgs paged_args(const lact_paged_desc* s) {
  PagedArgs a{};
  fill_paged(a, s);
  paged_plan(a, s->io_dtype == LACT_IO_BF16);
  return a;
}

size_t paged_bytes(const PagedArgs& a) {
  return a.splits > 1 ? ws_round((size_t)a.splits * a.T * a.H * (a.d + 2) * 4) : 0;
}

// ---------------------------------------------------------------- pages of e4m3 numbers, prefixes
// A cache of e4m3 numbers: vectors of d bytes, which the kernels move 16 at a
// time, and a byte for each.
int check_chunks(const lact_paged_desc* s) { return s->d % 16 ? LACT_EUNSUPPORTED : LACT_OK; }

int check_codes(const lact_paged_desc* s, const lact_view* kc, const lact_view* vc, const lact_view* ks,
                const lact_view* vs, const int32_t* table, const int32_t* lens, const int32_t* cu, bool out) {
  LACT_TRY(check_chunks(s));
  LACT_TRY(check_cache(s, 1, kc, vc, table, lens, cu, out));
  LACT_TRY(check_view(ks, s->pages, s->Hkv, s->page, 1, 0, out));
  LACT_TRY(check_view(vs, s->pages, s->Hkv, s->page, 1, 0, out));
  return same_strides(s, ks, vs) ? LACT_OK : LACT_EINVAL;
}

int check_prefix(const lact_paged_desc* s, const lact_prefix* p) {
  LACT_TRY(check_paged(s, true));
  if (!p || p->groups < 1 || p->max_pages < 0) return LACT_EINVAL;
  // (positions behind a prefix count its keys)
  if ((int64_t)p->groups * s->Hkv > (1 << 20) || ((int64_t)p->max_pages + s->max_pages) * s->page > kAttnTokens)
    return LACT_EUNSUPPORTED;
  return LACT_OK;
}

PrefixArgs prefix_args(const lact_paged_desc* s, const lact_prefix* p, bool codes) {
  PrefixArgs a{};
  fill_paged(a, s);
  if (p) {
    a.P = p->groups;
    a.p_pages = s->pages > 0 ? p->max_pages : 0;
    a.ptable = p->table;
    a.plen = p->lens;
    a.cu_seq = p->cu_seq;
  }
  a.codes = codes;
  prefix_plan(a, s->io_dtype == LACT_IO_BF16, codes);
  return a;
}

// (both roles are in one direction of one launch)
int check_jobs(const PrefixArgs& a) { return prefix_jobs(a) * 256 < ((int64_t)1 << 32) ? LACT_OK : LACT_EUNSUPPORTED; }

size_t prefix_bytes(const PrefixArgs& a) {
  const int parts = a.psplits + a.splits;
  return parts > 1 ? ws_round((size_t)parts * a.T * a.H * (a.d + 2) * 4) : 0;
}

// The workspace of a call whose descriptor was found to be `rc`.
size_t checked_bytes(const lact_paged_desc* s, const lact_prefix* p, bool codes, int rc, int* err) {
  PrefixArgs a{};
  if (!rc && codes) rc = check_chunks(s);
  if (!rc) {
    a = prefix_args(s, p, codes);
    rc = check_jobs(a);
  }
  if (err) *err = rc;
  return rc ? 0 : prefix_bytes(a);
}

CodeArgs code_args(const lact_paged_desc* s, const lact_view* k, const lact_view* v, const lact_view* kc,
                   const lact_view* vc, const lact_view* ks, const lact_view* vs, const int32_t* table,
                   const int32_t* lens, const int32_t* cu) {
  CodeArgs a{};
  a.k = take(k, 1, s->Hkv, s->n_new);
  a.v = take(v, 1, s->Hkv, s->n_new);
  a.c = take(kc, s->pages, s->Hkv, s->page);
  a.cs = take(ks, s->pages, s->Hkv, s->page);
  a.kc = static_cast<uint8_t*>(kc->data);
  a.vc = static_cast<uint8_t*>(vc->data);
  a.ks = static_cast<uint8_t*>(ks->data);
  a.vs = static_cast<uint8_t*>(vs->data);
  a.table = table;
  a.len = lens;
  a.cu = cu;
  a.B = s->B;
  a.Hkv = s->Hkv;
  a.d = s->d;
  a.T = (int)s->n_new;
  a.page = s->page;
  a.max_pages = s->pages > 0 ? s->max_pages : 0;
  a.pages = (int)s->pages;
  divider(s->page, &a.mul, &a.shift);
  return a;
}

int check_workspace(size_t need, const void* workspace, size_t bytes) {
  if (need && (!workspace || bytes < need)) return LACT_EWORKSPACE;
  if (need && ((uintptr_t)workspace & (kWsAlign - 1))) return LACT_EALIGN;
  return LACT_OK;
}

template <class A, hipError_t (*F)(const A&, bool, hipStream_t)>
int go(int kclass, const A& a, bool bf16, void* stream) {
  struct Ctx {
    const A& a;
    bool bf16;
    hipStream_t s;
  } c{a, bf16, (hipStream_t)stream};
  return timed_launch(
      kclass, 0.0, c.s,
      [](void* p) {
        Ctx* x = static_cast<Ctx*>(p);
        return F(x->a, x->bf16, x->s);
      },
      &c);
}

int check_rows(const lact_paged_desc* s, const lact_view* q, const lact_view* o) {
  const int es = elem(s->io_dtype);
  LACT_TRY(check_view(q, 1, s->H, s->n_new, s->d, es, false));
  return check_view(o, 1, s->H, s->n_new, s->d, es, true);
}

// The launch of a checked call; `a` has its plan, its prefixes and its scales.
int attend(const lact_paged_desc* s, PrefixArgs& a, const lact_view* q, const lact_view* kc, const lact_view* vc,
           const int32_t* table, const int32_t* lens, const int32_t* cu, const lact_view* o, void* workspace,
           size_t bytes, void* stream) {
  LACT_TRY(check_jobs(a));
  LACT_TRY(check_workspace(prefix_bytes(a), workspace, bytes));
  if (s->n_new == 0) return LACT_OK;
  a.q = take(q, 1, s->H, s->n_new);
  a.o = take(o, 1, s->H, s->n_new);
  a.c = take(kc, s->pages, s->Hkv, s->page);
  a.kc = kc->data;
  a.vc = vc->data;
  a.table = table;
  a.len = lens;
  a.cu = cu;
  a.part = static_cast<float*>(workspace);
  return go<PrefixArgs, launch_prefix>(LACT_KCLASS_ATTN, a, s->io_dtype == LACT_IO_BF16, stream);
}

}  // namespace
}  // namespace lact

using namespace lact;

extern "C" {

int lact_qk_norm_rope(const lact_rope_desc* desc, const lact_view* q, const lact_view* k, const float* wq,
                      const float* wk, const double* inv_freq, const int32_t* positions, const lact_view* qn,
                      const lact_view* kn, void* stream) {
  LACT_TRY(rope_common(desc, q, k, wq, wk, inv_freq, positions));
  const lact_rope_desc& s = *desc;
  const int es = elem(s.io_dtype);
  LACT_TRY(check_view(qn, s.B, s.H, s.n, s.d, es, true));
  LACT_TRY(check_view(kn, s.B, s.Hkv, s.n, s.d, es, true));
  if (s.n == 0) return LACT_OK;
  RopeArgs a = rope_args(desc, false);
  a.x[0] = take(q, s.B, s.H, s.n);
  a.x[1] = take(k, s.B, s.Hkv, s.n);
  a.y[0] = take(qn, s.B, s.H, s.n);
  a.y[1] = take(kn, s.B, s.Hkv, s.n);
  a.w[0] = wq;
  a.w[1] = wk;
  a.freq = inv_freq;
  a.pos = positions;
  return go<RopeArgs, launch_rope>(LACT_KCLASS_IO, a, s.io_dtype == LACT_IO_BF16, stream);
}

size_t lact_qk_norm_rope_backward_workspace_bytes(const lact_rope_desc* desc, int* err) {
  const int rc = check_rope(desc);
  if (err) *err = rc;
  return rc ? 0 : ws_round(rope_part_floats(rope_args(desc, true)) * 4);
}

int lact_qk_norm_rope_backward(const lact_rope_desc* desc, const lact_view* q, const lact_view* k, const float* wq,
                               const float* wk, const double* inv_freq, const int32_t* positions,
                               const lact_view* dqn, const lact_view* dkn, const lact_view* dq, const lact_view* dk,
                               float* dwq, float* dwk, void* workspace, size_t workspace_bytes, void* stream) {
  LACT_TRY(rope_common(desc, q, k, wq, wk, inv_freq, positions));
  const lact_rope_desc& s = *desc;
  const int es = elem(s.io_dtype);
  LACT_TRY(check_view(dqn, s.B, s.H, s.n, s.d, es, false));
  LACT_TRY(check_view(dkn, s.B, s.Hkv, s.n, s.d, es, false));
  LACT_TRY(check_view(dq, s.B, s.H, s.n, s.d, es, true));
  LACT_TRY(check_view(dk, s.B, s.Hkv, s.n, s.d, es, true));
  if ((dwq && !wq) || (dwk && !wk)) return LACT_EINVAL;
  if (((uintptr_t)dwq & 3) || ((uintptr_t)dwk & 3)) return LACT_EALIGN;
  RopeArgs a = rope_args(desc, true);
  const bool any = dwq || dwk;
  LACT_TRY(check_workspace(any ? ws_round(rope_part_floats(a) * 4) : 0, workspace, workspace_bytes));
  if (s.n == 0 && !any) return LACT_OK;
  a.x[0] = take(q, s.B, s.H, s.n);
  a.x[1] = take(k, s.B, s.Hkv, s.n);
  a.y[0] = take(dqn, s.B, s.H, s.n);
  a.y[1] = take(dkn, s.B, s.Hkv, s.n);
  a.dx[0] = take(dq, s.B, s.H, s.n);
  a.dx[1] = take(dk, s.B, s.Hkv, s.n);
  a.w[0] = wq;
  a.w[1] = wk;
  a.freq = inv_freq;
  a.pos = positions;
  a.dw[0] = dwq;
  a.dw[1] = dwk;
  a.part = static_cast<float*>(workspace);
  return go<RopeArgs, launch_rope_bwd>(LACT_KCLASS_IO, a, s.io_dtype == LACT_IO_BF16, stream);
}

int lact_window_attention(const lact_attn_desc* desc, const lact_view* q, const lact_view* k, const lact_view* v,
                          const int32_t* lengths, const lact_view* o, float* lse, void* stream) {
  LACT_TRY(check_attn(desc));
  const lact_attn_desc& s = *desc;
  const int es = elem(s.io_dtype);
  LACT_TRY(check_view(q, s.B, s.H, s.n_q, s.d, es, false));
  LACT_TRY(check_view(k, s.B, s.Hkv, s.n_kv, s.d, es, false));
  LACT_TRY(check_view(v, s.B, s.Hkv, s.n_kv, s.d, es, false));
  LACT_TRY(check_view(o, s.B, s.H, s.n_q, s.d, es, true));
  if (((uintptr_t)lengths & 3) || ((uintptr_t)lse & 3)) return LACT_EALIGN;
  if (s.n_q == 0) return LACT_OK;
  WindowArgs a = window_args(desc);
  a.q = take(q, s.B, s.H, s.n_q);
  a.k = take(k, s.B, s.Hkv, s.n_kv);
  a.v = take(v, s.B, s.Hkv, s.n_kv);
  a.o = take(o, s.B, s.H, s.n_q);
  a.lse = lse;
  a.len = lengths;
  return go<WindowArgs, launch_window_fwd>(LACT_KCLASS_ATTN, a, s.io_dtype == LACT_IO_BF16, stream);
}

size_t lact_window_attention_backward_workspace_bytes(const lact_attn_desc* desc, int* err) {
  const int rc = check_attn(desc);
  if (err) *err = rc;
  if (rc) return 0;
  const WindowArgs a = window_args(desc);
  return window_layout(a, window_dkv_plan(a, desc->io_dtype == LACT_IO_BF16)).total;
}

int lact_window_attention_backward(const lact_attn_desc* desc, const lact_view* q, const lact_view* k,
                                   const lact_view* v, const lact_view* o, const float* lse, const lact_view* dout,
                                   const int32_t* lengths, const lact_view* dq, const lact_view* dk,
                                   const lact_view* dv, void* workspace, size_t workspace_bytes, void* stream) {
  LACT_TRY(check_attn(desc));
  const lact_attn_desc& s = *desc;
  const int es = elem(s.io_dtype);
  LACT_TRY(check_view(q, s.B, s.H, s.n_q, s.d, es, false));
  LACT_TRY(check_view(k, s.B, s.Hkv, s.n_kv, s.d, es, false));
  LACT_TRY(check_view(v, s.B, s.Hkv, s.n_kv, s.d, es, false));
  LACT_TRY(check_view(o, s.B, s.H, s.n_q, s.d, es, false));
  LACT_TRY(check_view(dout, s.B, s.H, s.n_q, s.d, es, false));
  LACT_TRY(check_view(dq, s.B, s.H, s.n_q, s.d, es, true));
  LACT_TRY(check_view(dk, s.B, s.Hkv, s.n_kv, s.d, es, true));
  LACT_TRY(check_view(dv, s.B, s.Hkv, s.n_kv, s.d, es, true));
  if (s.n_q > 0 && !lse) return LACT_EINVAL;
  if (((uintptr_t)lengths & 3) || ((uintptr_t)lse & 3)) return LACT_EALIGN;
  const bool bf16 = s.io_dtype == LACT_IO_BF16;
  WindowBwdArgs g{};
  WindowArgs& a = g.f;
  a = window_args(desc);
  g.plan = window_dkv_plan(a, bf16);
  const WindowLayout l = window_layout(a, g.plan);
  LACT_TRY(check_workspace(l.total, workspace, workspace_bytes));
  if (s.n_q == 0 && s.n_kv == 0) return LACT_OK;
  a.q = take(q, s.B, s.H, s.n_q);
  a.k = take(k, s.B, s.Hkv, s.n_kv);
  a.v = take(v, s.B, s.Hkv, s.n_kv);
  a.o = take(o, s.B, s.H, s.n_q);
  a.lse = const_cast<float*>(lse);
  a.len = lengths;
  g.dout = take(dout, s.B, s.H, s.n_q);
  g.dq = take(dq, s.B, s.H, s.n_q);
  g.dk = take(dk, s.B, s.Hkv, s.n_kv);
  g.dv = take(dv, s.B, s.Hkv, s.n_kv);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  g.nlse = reinterpret_cast<float*>(ws + l.nlse);
  g.ndelta = reinterpret_cast<float*>(ws + l.ndelta);
  g.part = reinterpret_cast<float*>(ws + l.part);
  return go<WindowBwdArgs, launch_window_bwd>(LACT_KCLASS_ATTN, g, bf16, stream);
}

int lact_paged_append(const lact_paged_desc* desc, const lact_view* k, const lact_view* v, const lact_view* k_cache,
                      const lact_view* v_cache, const int32_t* table, const int32_t* lens, const int32_t* cu_new,
                      void* stream) {
  LACT_TRY(check_paged(desc, false));
  const lact_paged_desc& s = *desc;
  const int es = elem(s.io_dtype);
  LACT_TRY(check_view(k, 1, s.Hkv, s.n_new, s.d, es, false));
  LACT_TRY(check_view(v, 1, s.Hkv, s.n_new, s.d, es, false));
  LACT_TRY(check_cache(desc, es, k_cache, v_cache, table, lens, cu_new, true));
  if (s.n_new == 0 || s.pages == 0 || s.max_pages == 0) return LACT_OK;
  AppendArgs a{};
  a.k = take(k, 1, s.Hkv, s.n_new);
  a.v = take(v, 1, s.Hkv, s.n_new);
  a.c = take(k_cache, s.pages, s.Hkv, s.page);
  a.kc = k_cache->data;
  a.vc = v_cache->data;
  a.table = table;
  a.len = lens;
  a.cu = cu_new;
  a.B = s.B;
  a.Hkv = s.Hkv;
  a.d = s.d;
  a.T = (int)s.n_new;
  a.page = s.page;
  a.max_pages = s.max_pages;
  a.pages = (int)s.pages;
  divider(s.page, &a.mul, &a.shift);
  return go<AppendArgs, launch_append>(LACT_KCLASS_IO, a, s.io_dtype == LACT_IO_BF16, stream);
}

size_t lact_paged_attention_workspace_bytes(const lact_paged_desc* desc, int* err) {
  const int rc = check_paged(desc, true);
  if (err) *err = rc;
  return rc ? 0 : paged_bytes(paged_args(desc));
}

int lact_paged_attention(const lact_paged_desc* desc, const lact_view* q, const lact_view* k_cache,
                         const lact_view* v_cache, const int32_t* table, const int32_t* lens, const int32_t* cu_new,
                         const lact_view* o, void* workspace, size_t workspace_bytes, void* stream) {
  LACT_TRY(check_paged(desc, true));
  const lact_paged_desc& s = *desc;
  const int es = elem(s.io_dtype);
  LACT_TRY(check_view(q, 1, s.H, s.n_new, s.d, es, false));
  LACT_TRY(check_view(o, 1, s.H, s.n_new, s.d, es, true));
  LACT_TRY(check_cache(desc, es, k_cache, v_cache, table, lens, cu_new, false));
  PagedArgs a = paged_args(desc);
  LACT_TRY(check_workspace(paged_bytes(a), workspace, workspace_bytes));
  if (s.n_new == 0) return LACT_OK;
  a.q = take(q, 1, s.H, s.n_new);
  a.o = take(o, 1, s.H, s.n_new);
  a.c = take(k_cache, s.pages, s.Hkv, s.page);
  a.kc = k_cache->data;
  a.vc = v_cache->data;
  a.table = table;
  a.len = lens;
  a.cu = cu_new;
  a.part = static_cast<float*>(workspace);
  return go<PagedArgs, launch_paged>(LACT_KCLASS_ATTN, a, s.io_dtype == LACT_IO_BF16, stream);
}

int lact_paged_append_e4m3(const lact_paged_desc* desc, const lact_view* k, const lact_view* v,
                           const lact_view* k_cache, const lact_view* v_cache, const lact_view* k_scale,
                           const lact_view* v_scale, const int32_t* table, const int32_t* lens, const int32_t* cu_new,
                           void* stream) {
  LACT_TRY(check_paged(desc, false));
  const lact_paged_desc& s = *desc;
  const int es = elem(s.io_dtype);
  LACT_TRY(check_view(k, 1, s.Hkv, s.n_new, s.d, es, false));
  LACT_TRY(check_view(v, 1, s.Hkv, s.n_new, s.d, es, false));
  LACT_TRY(check_codes(desc, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new, true));
  if (s.n_new == 0 || s.pages == 0 || s.max_pages == 0) return LACT_OK;
  const CodeArgs a = code_args(desc, k, v, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new);
  return go<CodeArgs, launch_append_e4m3>(LACT_KCLASS_IO, a, s.io_dtype == LACT_IO_BF16, stream);
}

int lact_paged_read_e4m3(const lact_paged_desc* desc, const lact_view* k_cache, const lact_view* v_cache,
                         const lact_view* k_scale, const lact_view* v_scale, const int32_t* table, const int32_t* lens,
                         const int32_t* cu_new, const lact_view* k, const lact_view* v, void* stream) {
  LACT_TRY(check_paged(desc, false));
  const lact_paged_desc& s = *desc;
  const int es = elem(s.io_dtype);
  LACT_TRY(check_codes(desc, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new, false));
  LACT_TRY(check_view(k, 1, s.Hkv, s.n_new, s.d, es, true));
  LACT_TRY(check_view(v, 1, s.Hkv, s.n_new, s.d, es, true));
  if (s.n_new == 0) return LACT_OK;
  const CodeArgs a = code_args(desc, k, v, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new);
  return go<CodeArgs, launch_read_e4m3>(LACT_KCLASS_IO, a, s.io_dtype == LACT_IO_BF16, stream);
}

size_t lact_paged_attention_e4m3_workspace_bytes(const lact_paged_desc* desc, int* err) {
  return checked_bytes(desc, nullptr, true, check_paged(desc, true), err);
}

int lact_paged_attention_e4m3(const lact_paged_desc* desc, const lact_view* q, const lact_view* k_cache,
                              const lact_view* v_cache, const lact_view* k_scale, const lact_view* v_scale,
                              const int32_t* table, const int32_t* lens, const int32_t* cu_new, const lact_view* o,
                              void* workspace, size_t workspace_bytes, void* stream) {
  LACT_TRY(check_paged(desc, true));
  LACT_TRY(check_rows(desc, q, o));
  LACT_TRY(check_codes(desc, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new, false));
  PrefixArgs a = prefix_args(desc, nullptr, true);
  a.ks = static_cast<const uint8_t*>(k_scale->data);
  a.vs = static_cast<const uint8_t*>(v_scale->data);
  a.cs = take(k_scale, desc->pages, desc->Hkv, desc->page);
  return attend(desc, a, q, k_cache, v_cache, table, lens, cu_new, o, workspace, workspace_bytes, stream);
}

size_t lact_paged_prefix_attention_workspace_bytes(const lact_paged_desc* desc, const lact_prefix* prefix, int e4m3,
                                                   int* err) {
  return checked_bytes(desc, prefix, e4m3 != 0, check_prefix(desc, prefix), err);
}

int lact_paged_prefix_attention(const lact_paged_desc* desc, const lact_prefix* prefix, const lact_view* q,
                                const lact_view* k_cache, const lact_view* v_cache, const lact_view* k_scale,
                                const lact_view* v_scale, const int32_t* table, const int32_t* lens,
                                const int32_t* cu_new, const lact_view* o, void* workspace, size_t workspace_bytes,
                                void* stream) {
  LACT_TRY(check_prefix(desc, prefix));
  LACT_TRY(check_rows(desc, q, o));
  const bool codes = k_scale || v_scale;
  LACT_TRY(codes ? check_codes(desc, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new, false)
                 : check_cache(desc, elem(desc->io_dtype), k_cache, v_cache, table, lens, cu_new, false));
  if (!prefix->lens || !prefix->cu_seq || (prefix->max_pages > 0 && !prefix->table)) return LACT_EINVAL;
  if (((uintptr_t)prefix->table & 3) || ((uintptr_t)prefix->lens & 3) || ((uintptr_t)prefix->cu_seq & 3))
    return LACT_EALIGN;
  PrefixArgs a = prefix_args(desc, prefix, codes);
  if (codes) {
    a.ks = static_cast<const uint8_t*>(k_scale->data);
    a.vs = static_cast<const uint8_t*>(v_scale->data);
    a.cs = take(k_scale, desc->pages, desc->Hkv, desc->page);
  }
  return attend(desc, a, q, k_cache, v_cache, table, lens, cu_new, o, workspace, workspace_bytes, stream);
}

}  // extern "C"
