"""Cases of the attention half of the hybrid layer, through the package's public entry points.

``op`` of a case:

* "norm_rope": per-head RMS norm of queries and keys with the position rotation (``qk_norm_rope``);
* "norm_rope_train": the same and its reverse (``qk_norm_rope_backward``);
* "attention": softmax attention with a sliding window and first tokens that stay visible (``window_attention``);
* "attention_train": the same and its reverse (``window_attention_backward``);
* "paged": new tokens of many sequences over a cache of pages (``paged_attention``);
* "append": their keys and values written into those pages (``paged_append``).

With ``own`` false ``run`` computes the same from elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
BASE = 10000.0


def _rope(name, op, b, n, heads, kv_heads, d, rot, interleaved=False, fp32=False, far=0):
    return _named(name, {"op": op, "B": b, "n": n, "H": heads, "Hkv": kv_heads, "d": d, "rot": rot,
                         "interleaved": interleaved, "fp32": fp32, "far": far})


def _attn(name, op, b, n, heads, kv_heads, d, window, sinks=0, lookahead=0, ragged=False, fp32=False):
    return _named(name, {"op": op, "B": b, "n": n, "H": heads, "Hkv": kv_heads, "d": d, "window": window,
                         "sinks": sinks, "lookahead": lookahead, "ragged": ragged, "fp32": fp32})


def _paged(name, op, b, new, max_len, heads, kv_heads, d, page, window=-1, sinks=0, fp32=False):
    return _named(name, {"op": op, "B": b, "new": new, "max_len": max_len, "H": heads, "Hkv": kv_heads, "d": d,
                         "page": page, "window": window, "sinks": sinks, "fp32": fp32})


def _named(name, c):
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one decoding step of a batch: a token each, far into their sequences
        _rope("rope_token", "norm_rope", 16, 1, 16, 4, 128, 128, far=30000),
        # a training batch of odd length, half of each head rotated
        _rope("rope_train", "norm_rope_train", 4, 8191, 16, 4, 128, 64),
        # the smallest training call: a small fp32 layer (launches and latency)
        _attn("attn_tiny_fp32", "attention_train", 1, 256, 2, 2, 64, 64, fp32=True),
        # prefill of a language model's window attention, window of one chunk
        _attn("attn_lm", "attention", 1, 16384, 16, 16, 128, 2048),
        # video: every token of a chunk of frames sees the whole chunk
        _attn("attn_video", "attention", 2, 3120, 40, 40, 128, -1, lookahead=-1),
        # training with shared key heads and a few first tokens that stay visible
        _attn("attn_lm_train", "attention_train", 1, 8192, 16, 4, 128, 2048, sinks=4),
        # a padded training batch of odd lengths, narrow heads, a short window
        _attn("attn_ragged_train", "attention_train", 3, 2003, 32, 8, 64, 500, sinks=1, ragged=True),
        # decoding of a served batch over long caches
        _paged("paged_decode", "paged", 64, 1, 16384, 16, 4, 128, 16),
        # decoding of one sequence, window and sinks (latency)
        _paged("paged_one", "paged", 1, 1, 5003, 16, 4, 128, 64, window=2048, sinks=4),
        # chunks of prompts beside each other, pages that end inside a tile
        _paged("paged_chunk", "paged", 6, 700, 8192, 16, 4, 128, 24),
        # the keys and values of one decoding step
        _paged("append_token", "append", 64, 1, 4096, 16, 4, 128, 16),
        # the keys and values of long prompt chunks
        _paged("append_prefill", "append", 8, 4000, 8192, 16, 8, 128, 32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = _draw(rng)
    while work(c)["flops"] * (8 if c["fp32"] else 1) > 4e11 or work(c)["bytes"] > 1.5e9:   # no dearer than the listed
        if c["B"] > 1:
            c["B"] = (c["B"] + 1) // 2
        elif "n" in c:
            c["n"] = c["n"] * 4 // 5
        elif c["new"] > 1:
            c["new"] = c["new"] * 4 // 5
        else:
            c["max_len"] = c["max_len"] * 4 // 5
    return c


def _draw(rng):
    op = rng.choice(["norm_rope", "norm_rope_train", "attention", "attention", "attention_train", "attention_train",
                     "paged", "paged", "append"])
    d = rng.choice([64, 64, 80, 96, 128, 128, 128])
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 2, 4, 5, 8])
    heads = min(heads, 16 * kv, 40)
    heads -= heads % kv
    fp32 = rng.random() < 0.2
    if op.startswith("norm_rope"):
        n = _log(rng, 1, 8000)
        b = rng.randint(1, max(1, min(64, 16000 // n)))
        return _rope(None, op, b, n, heads, kv, d, rng.choice([d, d, d // 2]), rng.random() < 0.3, fp32,
                     rng.choice([0, 0, 100000]))
    if op.startswith("attention"):
        n = _log(rng, 1, 8000 if not fp32 else 2000)
        b = rng.randint(1, max(1, min(4, 8000 // n)))
        kind = rng.random()
        window = -1 if kind < 0.2 else min(_log(rng, 16, 4000), n)
        look = (-1 if window < 0 else rng.choice([0, window])) if rng.random() < 0.25 else 0
        return _attn(None, op, b, n, heads, kv, d, window, rng.choice([0, 0, 1, 4, 70]), look, rng.random() < 0.5, fp32)
    max_len = _log(rng, 16, 16000)
    b = _log(rng, 1, max(1, min(64, 400000 // max_len)))
    new = 1 if rng.random() < 0.5 else _log(rng, 1, min(max_len, 1000))
    if op == "append":
        return _paged(None, op, b, new, max_len, heads, kv, d, rng.choice([1, 8, 16, 24, 64, 128]), fp32=fp32)
    window = -1 if rng.random() < 0.5 else _log(rng, 16, 4000)
    return _paged(None, op, b, new, max_len, heads, kv, d, rng.choice([1, 8, 16, 24, 64, 128]), window,
                  rng.choice([0, 0, 1, 4, 70]), fp32)


def _lengths(case, seed):
    """Host integers of a case: lengths of a padded batch, or (lengths, new tokens) of sequences in pages."""
    g = torch.Generator().manual_seed(seed * 7919 + 13)
    b = case["B"]
    if "page" not in case:
        n = case["n"]
        lens = torch.randint((n + 1) // 2, n + 1, (b,), generator=g) if case["ragged"] else torch.full((b,), n)
        lens[0] = n
        return lens
    at = torch.Generator().manual_seed(b * 1009 + case["new"])       # the shapes of a case go by its sizes alone
    new = torch.randint((case["new"] + 1) // 2, case["new"] + 1, (b,), generator=at)
    new[0] = case["new"]
    lens = torch.randint((case["max_len"] + 1) // 2, case["max_len"] + 1, (b,), generator=g)
    lens[0] = case["max_len"]
    return torch.maximum(lens, new), new


def prepare(case, seed):
    dt = torch.float32 if case["fp32"] else torch.bfloat16
    gen = torch.Generator("cuda").manual_seed(seed)
    draw_ = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=dt)
    op, b, heads, kv, d = case["op"], case["B"], case["H"], case["Hkv"], case["d"]
    st = {"case": case}
    if op.startswith("norm_rope"):
        n, rot = case["n"], case["rot"]
        qkv = draw_(b, n, heads + 2 * kv, d)          # the fused projection: q and k are strided parts of it
        st["q"], st["k"] = qkv[:, :, :heads], qkv[:, :, heads:heads + kv]
        f32 = lambda *s: torch.rand(*s, generator=gen, device="cuda", dtype=torch.float32) + 0.5
        st["wq"], st["wk"] = f32(d), f32(d)
        st["inv_freq"] = BASE ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
        start = torch.randint(case["far"] // 2, case["far"] + 1, (b, 1), generator=gen, device="cuda") if case["far"] \
            else torch.zeros(b, 1, dtype=torch.int64, device="cuda")
        st["positions"] = (start + torch.arange(n, device="cuda")).to(torch.int32)
        if op == "norm_rope_train":
            st["dq"], st["dk"] = draw_(b, heads, n, d), draw_(b, kv, n, d)
        return st
    if op.startswith("attention"):
        n = case["n"]
        st["q"], st["k"], st["v"] = draw_(b, heads, n, d), draw_(b, kv, n, d), draw_(b, kv, n, d)
        st["lengths"] = _lengths(case, seed).to("cuda", torch.int32) if case["ragged"] else None
        if op == "attention_train":
            st["dout"] = draw_(b, heads, n, d)
        return st
    lens, new = _lengths(case, seed)
    page, width = case["page"], -(-case["max_len"] // case["page"])
    total = int(new.sum())
    pages = b * width
    st["k_cache"], st["v_cache"] = draw_(pages, page, kv, d), draw_(pages, page, kv, d)
    st["table"] = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).view(b, width).to("cuda", torch.int32)
    st["lens"] = lens.to("cuda", torch.int32)
    st["cu_new"] = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)]).to("cuda", torch.int32)
    if op == "append":
        st["k"], st["v"] = draw_(total, kv, d), draw_(total, kv, d)
    else:
        st["q"] = draw_(total, heads, d)
    return st


# ---------------------------------------------------------------- plain forms

def _angles(st, wide=torch.float32):
    a = st["positions"].double()[..., None] * st["inv_freq"]
    return torch.cos(a).to(wide)[:, :, None], torch.sin(a).to(wide)[:, :, None]


def _turn(x, c, s, rot, interleaved):
    """The rotation of the first `rot` elements of the last axis."""
    r, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([r, rest], -1)


def _norm_rope(st, x, w):
    c = st["case"]
    cs, sn = _angles(st)
    xf = x.float()
    y = xf * torch.rsqrt(xf.square().mean(-1, keepdim=True) + EPS) * w
    return _turn(y, cs, sn, c["rot"], c["interleaved"]).transpose(1, 2).to(x.dtype).contiguous()


def _norm_rope_back(st, x, w, dy):
    c = st["case"]
    cs, sn = _angles(st)
    xf = x.float()
    g = _turn(dy.float().transpose(1, 2), cs, -sn, c["rot"], c["interleaved"])
    r = torch.rsqrt(xf.square().mean(-1, keepdim=True) + EPS)
    dn = g * w
    dx = r * dn - xf * (r ** 3 * (xf * dn).mean(-1, keepdim=True))
    return dx.to(x.dtype), (g * xf * r).double().sum((0, 1, 2)).float()


def _visible(case, lens, n, device):
    """[B or 1, n, n]: which keys (last axis) a query sees."""
    p = torch.arange(n, device=device)[:, None]
    j = torch.arange(n, device=device)[None, :]
    see = torch.ones(n, n, dtype=torch.bool, device=device)
    if case["lookahead"] >= 0:
        see = see & (j <= p + case["lookahead"])
    if case["window"] >= 0:
        see = see & ((j > p - case["window"]) | (j < case["sinks"]))
    see = see[None]
    if lens is not None:
        ln = lens[:, None, None]
        see = see & (j < ln) & (p < ln)
    return see


def _weights(q, k, see, scale):
    """softmax over the visible keys, rows that see none are zero; q [B, Hkv, G, n, d], k [B, Hkv, 1, m, d]."""
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale
    s = s.masked_fill(~see[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
    del s
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, torch.ones_like(total), total)


def _grouped(x, kv):
    b, h, n, d = x.shape
    return x.float().view(b, kv, h // kv, n, d)


def _attention(st, train):
    c = st["case"]
    kv, scale = c["Hkv"], 1.0 / math.sqrt(c["d"])
    q, k, v = _grouped(st["q"], kv), _grouped(st["k"], kv), _grouped(st["v"], kv)
    p = _weights(q, k, _visible(c, st["lengths"], c["n"], q.device), scale)
    o = torch.matmul(p, v)
    out = o.flatten(1, 2).to(st["q"].dtype)
    if not train:
        return out
    do = _grouped(st["dout"], kv)
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), do).sum(2)
    delta = (do * o).sum(-1, keepdim=True)
    ds = torch.matmul(do, v.transpose(-1, -2).contiguous()).sub_(delta).mul_(p)
    del p
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q).sum(2) * scale
    dt = st["q"].dtype
    return out, dq.flatten(1, 2).to(dt), dk.to(dt), dv.to(dt)


def _places(st):
    """Of every new token: its sequence and its position there."""
    cu = st["cu_new"].long()
    counts = cu[1:] - cu[:-1]
    t = torch.arange(st["total"], device=cu.device)
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    return seq, t - cu[seq] + st["lens"].long()[seq] - counts[seq]


def _append(st):
    seq, pos = _places(dict(st, total=st["k"].shape[0]))
    page = st["case"]["page"]
    slot = st["table"].long()[seq, pos // page] * page + pos % page
    st["k_cache"].flatten(0, 1)[slot] = st["k"]
    st["v_cache"].flatten(0, 1)[slot] = st["v"]
    return st["k_cache"], st["v_cache"]


def _paged_attention(st):
    c = st["case"]
    b, kv, heads, d, new = c["B"], c["Hkv"], c["H"], c["d"], c["new"]
    total = st["q"].shape[0]
    seq, pos = _places(dict(st, total=total))
    at = torch.arange(total, device=seq.device) - st["cu_new"].long()[seq]
    q = torch.zeros(b, new, heads, d, device=seq.device)
    q[seq, at] = st["q"].float()
    p = torch.full((b, new), -1, device=seq.device)
    p[seq, at] = pos
    q = q.view(b, new, kv, heads // kv, d).permute(0, 2, 3, 1, 4)
    k = st["k_cache"][st["table"].long()].flatten(1, 2).float().transpose(1, 2)[:, :, None]
    v = st["v_cache"][st["table"].long()].flatten(1, 2).float().transpose(1, 2)[:, :, None]
    j = torch.arange(k.shape[3], device=seq.device)
    see = j <= p[..., None]
    if c["window"] >= 0:
        see = see & ((j > p[..., None] - c["window"]) | (j < c["sinks"]))
    o = torch.matmul(_weights(q, k, see, 1.0 / math.sqrt(d)), v)      # [B, Hkv, G, new, d]
    return o.permute(0, 3, 1, 2, 4).reshape(b, new, heads, d)[seq, at].to(st["q"].dtype)


def run(state):
    st, c = state, state["case"]
    op = c["op"]
    if own:
        return _run_own(st, c, op)
    if op == "norm_rope":
        return _norm_rope(st, st["q"], st["wq"]), _norm_rope(st, st["k"], st["wk"])
    if op == "norm_rope_train":
        return (_norm_rope(st, st["q"], st["wq"]), _norm_rope(st, st["k"], st["wk"]),
                *_norm_rope_back(st, st["q"], st["wq"], st["dq"]), *_norm_rope_back(st, st["k"], st["wk"], st["dk"]))
    if op in ("attention", "attention_train"):
        return _attention(st, op == "attention_train")
    return _append(st) if op == "append" else _paged_attention(st)


def _run_own(st, c, op):
    import paper_2505_23884_amd as P
    limit = lambda x: None if x < 0 else x
    if op.startswith("norm_rope"):
        kw = dict(positions=st["positions"], eps=EPS, interleaved=c["interleaved"])
        qn, kn = P.qk_norm_rope(st["q"], st["k"], st["wq"], st["wk"], st["inv_freq"], **kw)
        if op == "norm_rope":
            return qn, kn
        dq, dk, dwq, dwk = P.qk_norm_rope_backward(st["q"], st["k"], st["dq"], st["dk"], st["wq"], st["wk"],
                                                   st["inv_freq"], **kw)
        return qn, kn, dq, dwq, dk, dwk
    if op.startswith("attention"):
        kw = dict(window=limit(c["window"]), sinks=c["sinks"], lookahead=limit(c["lookahead"]), lengths=st["lengths"])
        if op == "attention":
            return P.window_attention(st["q"], st["k"], st["v"], **kw)
        o, lse = P.window_attention(st["q"], st["k"], st["v"], with_lse=True, **kw)
        return (o, *P.window_attention_backward(st["q"], st["k"], st["v"], o, lse, st["dout"], **kw))
    if op == "append":
        P.paged_append(st["k"], st["v"], st["k_cache"], st["v_cache"], st["table"], st["lens"], st["cu_new"])
        return st["k_cache"], st["v_cache"]
    return P.paged_attention(st["q"], st["k_cache"], st["v_cache"], st["table"], st["lens"], st["cu_new"],
                             window=limit(c["window"]), sinks=c["sinks"])


# ---------------------------------------------------------------- what a pass cannot do without

def _pairs(case, lens):
    """Visible (query, key) pairs of one head over the batch, as a float."""
    total = 0.0
    for n in lens:
        p = torch.arange(int(n), dtype=torch.float64)
        hi = torch.full_like(p, n) if case["lookahead"] < 0 else (p + 1 + case["lookahead"]).clamp(max=n)
        if case["window"] < 0:
            total += float(hi.sum())
            continue
        lo = (p - case["window"] + 1).clamp(min=0)
        total += float((hi - lo).clamp(min=0).sum() + torch.minimum(lo, hi).clamp(max=case["sinks"]).sum())
    return total


def work(case):
    es = 4 if case["fp32"] else 2
    op, b, heads, kv, d = case["op"], case["B"], case["H"], case["Hkv"], case["d"]
    if op.startswith("norm_rope"):
        vec = b * case["n"] * (heads + kv) * d
        passes = 2 if op == "norm_rope" else 5       # x in, y out; with the reverse x and dy in, dx out
        return {"bytes": vec * es * passes + b * case["n"] * 4, "flops": vec * (7 if op == "norm_rope" else 20)}
    if op.startswith("attention"):
        lens = _lengths(case, 1).tolist()
        pairs = _pairs(case, lens) * heads
        rows = b * case["n"] * d * es
        if op == "attention":
            return {"bytes": rows * (2 * heads + 2 * kv), "flops": 4 * d * pairs}
        return {"bytes": rows * (5 * heads + 6 * kv), "flops": 14 * d * pairs}
    lens, new = (x.tolist() for x in _lengths(case, 1))
    if op == "append":
        return {"bytes": 4 * sum(new) * kv * d * es, "flops": 0}
    pairs, keys = 0.0, 0.0
    for n, m in zip(lens, new):
        p = torch.arange(n - m, n, dtype=torch.float64)
        lo = torch.zeros_like(p) if case["window"] < 0 else (p - case["window"] + 1).clamp(min=0)
        pairs += float((p + 1 - lo).sum() + lo.clamp(max=case["sinks"]).sum())
        keys += n - float(lo[0]) + min(float(lo[0]), case["sinks"])
    return {"bytes": 2 * keys * kv * d * es + 2 * sum(new) * heads * d * es, "flops": 4 * d * heads * pairs}


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_turn(x, pos, inv_freq, rot, interleaved, sign):
    """Each pair as a complex number times e^(i sign pos f)."""
    y = x.clone()
    i = torch.arange(rot // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    z = torch.complex(x[..., a], x[..., b])
    ang = sign * pos.double()[:, :, None, None] * inv_freq
    z = z * torch.polar(torch.ones_like(ang), ang)
    y[..., a], y[..., b] = z.real, z.imag
    return y


def _exact_norm_rope(case, st, x, w, dy):
    x64, w64 = x.double(), w.double()
    d = x.shape[-1]
    norm = ((x64 * x64).sum(-1, keepdim=True) / d + EPS) ** 0.5
    args = (st["positions"], st["inv_freq"], case["rot"], case["interleaved"])
    y = _exact_turn(x64 / norm * w64, *args, 1.0).permute(0, 2, 1, 3)
    if dy is None:
        return (y,)
    g = _exact_turn(dy.double().permute(0, 2, 1, 3), *args, -1.0)
    u = x64 / norm
    gw = g * w64
    dx = (gw - u * (u * gw).sum(-1, keepdim=True) / d) / norm
    return y, dx, (g * u).sum(dim=(0, 1, 2))


def _exact_head(q, k, v, see, scale, do=None):
    """One head: q [n, d], k and v [m, d], see [n, m], in 64 bits."""
    z = torch.where(see, q @ k.t() * scale, torch.full((), -torch.inf, dtype=torch.float64, device=q.device))
    some = see.any(1)
    a = torch.zeros_like(z)
    a[some] = torch.softmax(z[some], dim=1)
    o = a @ v
    if do is None:
        return (o,)
    da = do @ v.t()
    dz = a * (da - (a * da).sum(1, keepdim=True))
    return o, dz @ k * scale, dz.t() @ q * scale, a.t() @ do


def exact(case, seed):
    st = prepare(case, seed)
    op, b, heads, kv, d = case["op"], case["B"], case["H"], case["Hkv"], case["d"]
    if op.startswith("norm_rope"):
        train = op == "norm_rope_train"
        q = _exact_norm_rope(case, st, st["q"], st["wq"], st["dq"] if train else None)
        k = _exact_norm_rope(case, st, st["k"], st["wk"], st["dk"] if train else None)
        return (q[0], k[0], q[1], q[2], k[1], k[2]) if train else (q[0], k[0])
    scale = d ** -0.5
    group = heads // kv
    if op.startswith("attention"):
        n, train = case["n"], op == "attention_train"
        lens = _lengths(case, seed).tolist()
        zeros = lambda h: torch.zeros(b, h, n, d, dtype=torch.float64, device="cuda")
        o, dq, dk, dv = zeros(heads), zeros(heads), zeros(kv), zeros(kv)
        for i in range(b):
            m = int(lens[i])
            gap = torch.arange(m, device="cuda")[None, :] - torch.arange(m, device="cuda")[:, None]
            see = torch.ones(m, m, dtype=torch.bool, device="cuda")
            if case["window"] >= 0:
                see = gap > -case["window"]
                see[:, :case["sinks"]] = True
            if case["lookahead"] >= 0:
                see = see & (gap <= case["lookahead"])
            for h in range(heads):
                q, k, v = st["q"][i, h, :m].double(), st["k"][i, h // group, :m].double(), st["v"][i, h // group, :m].double()
                r = _exact_head(q, k, v, see, scale, st["dout"][i, h, :m].double() if train else None)
                o[i, h, :m] = r[0]
                if train:
                    dq[i, h, :m] = r[1]
                    dk[i, h // group, :m] += r[2]
                    dv[i, h // group, :m] += r[3]
        return (o, dq, dk, dv) if train else o
    lens, new = (x.tolist() for x in _lengths(case, seed))
    page = case["page"]
    table = st["table"].tolist()
    if op == "append":
        kc, vc = st["k_cache"].double(), st["v_cache"].double()
        t = 0
        for i in range(b):
            pos = torch.arange(lens[i] - new[i], lens[i], device="cuda")
            where = torch.tensor(table[i], device="cuda")[pos // page]
            kc[where, pos % page] = st["k"][t:t + new[i]].double()
            vc[where, pos % page] = st["v"][t:t + new[i]].double()
            t += new[i]
        return kc, vc
    out = torch.zeros(sum(new), heads, d, dtype=torch.float64, device="cuda")
    t = 0
    for i in range(b):
        n, m = int(lens[i]), int(new[i])
        rows = torch.tensor(table[i], device="cuda")
        k = st["k_cache"][rows].double().reshape(-1, kv, d)[:n]
        v = st["v_cache"][rows].double().reshape(-1, kv, d)[:n]
        gap = torch.arange(n, device="cuda")[None, :] - torch.arange(n - m, n, device="cuda")[:, None]
        see = gap <= 0
        if case["window"] >= 0:
            see = see & ((gap > -case["window"]) | (torch.arange(n, device="cuda") < case["sinks"])[None, :])
        for h in range(heads):
            out[t:t + m, h] = _exact_head(st["q"][t:t + m, h].double(), k[:, h // group], v[:, h // group], see, scale)[0]
        t += m
    return out
