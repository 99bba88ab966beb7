"""Plain 64-bit forms of the attention entry points, on the CPU, with the
magnitudes that their error bounds are made of."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a rounding step, relative


def visible(n_q, n_kv, length, q_start, window, sinks, lookahead):
    p = q_start + torch.arange(n_q)[:, None]
    j = torch.arange(n_kv)[None, :]
    see = (j < length) & (p < length)
    if lookahead is not None:
        see &= j <= p + lookahead
    if window is not None:
        see &= (j > p - window) | (j < sinks)
    return see


def head(q, k, v, see, scale, do=None):
    """One head in 64 bits. Returns a dict of the outputs and of what bounds
    their errors: `e` is the relative error of a weight in fp32 arithmetic (its
    score, a sum of d products, is off by (d + 4) 2^-24 of the products'
    magnitudes; the sum over the keys by a step each), per query."""
    q, k, v = q.double(), k.double(), v.double()
    n, d = see.shape[1], q.shape[1]
    s = q @ k.t() * scale
    s = torch.where(see, s, torch.full_like(s, -math.inf))
    some = see.any(1)
    p = torch.zeros_like(s)
    p[some] = torch.softmax(s[some], 1)
    lse = torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    lse[some] = torch.logsumexp(s[some], 1)
    mag = (q.abs() @ k.abs().t() * scale * see).amax(1, keepdim=True) if n else torch.zeros(q.shape[0], 1)
    u = 2.0 ** -24
    err_s = (d + 8) * u * mag + 4 * u * torch.where(some, lse.abs(), torch.zeros_like(lse))[:, None]
    e = 2 * err_s + (n + 16) * u
    r = {"o": p @ v, "lse": lse, "p": p, "e": e, "some": some, "lse_err": err_s[:, 0] + (n + 8) * u,
         "o_mag": p @ v.abs()}
    if do is not None:
        do = do.double()
        dp = do @ v.t()
        delta = (p * dp).sum(1, keepdim=True)
        ds = p * (dp - delta)
        r.update(dv=p.t() @ do, dq=ds @ k * scale, dk=ds.t() @ q * scale)
        # |ds| is off by e p (|dp| + |delta|), by the sums behind dp and delta, and
        # by the rounding of o (half a step of its type) in delta
        mdp = do.abs() @ v.abs().t()
        mdelta = (do.abs() * r["o_mag"]).sum(1, keepdim=True)
        r["do"], r["ds"], r["mdp"], r["mdelta"] = do, ds, mdp, mdelta
    return r


def bounds(r, q, k, do_, scale, dtype):
    """Largest error of each output: fp32 arithmetic, the rounding of weights
    (and their cotangents) to bf16 before the second products, and the
    rounding of the output."""
    h = HALF[dtype]
    w = h if dtype == torch.bfloat16 else 0.0
    u = 2.0 ** -24
    n_q, n_kv = r["p"].shape
    t = {"o": r["o_mag"] * (r["e"] + w + n_kv * u) * 1.01 + r["o"].abs() * h, "lse": r["lse_err"] * 1.01 + 1e-7}
    if do_ is None:
        return t
    q, k = q.double().abs(), k.double().abs()
    d = q.shape[1]
    o_err = (r["do"].abs() * (t["o"] + r["o"].abs() * h)).sum(1, keepdim=True)     # delta from the rounded o
    e_ds = r["p"] * (r["e"] * (r["mdp"] + r["mdelta"]) + (d + 8) * u * (r["mdp"] + r["mdelta"]) + o_err) + \
        r["ds"].abs() * (w + r["e"])
    t["dv"] = (r["p"] * (r["e"] + w + n_q * u)).t() @ r["do"].abs() * 1.01 + r["dv"].abs() * h
    t["dq"] = (e_ds + r["ds"].abs() * n_kv * u) @ k * scale * 1.01 + r["dq"].abs() * h
    t["dk"] = (e_ds + r["ds"].abs() * n_q * u).t() @ q * scale * 1.01 + r["dk"].abs() * h
    return t


def attention(q, k, v, lengths=None, q_start=None, window=None, sinks=0, lookahead=0, scale=None, do=None):
    """All heads: (outputs, bounds) as dicts of [B, heads, n, ..] fp64 tensors."""
    B, H, n_q, d = q.shape
    Hkv, n_kv = k.shape[1], k.shape[2]
    G = H // Hkv
    scale = d ** -0.5 if scale is None else scale
    q_start = n_kv - n_q if q_start is None else q_start
    dtype = q.dtype
    q, k, v = (x.detach().cpu() for x in (q, k, v))
    do = None if do is None else do.detach().cpu()
    shapes = {"o": (B, H, n_q, d), "lse": (B, H, n_q), "dq": (B, H, n_q, d), "dk": (B, Hkv, n_kv, d), "dv": (B, Hkv, n_kv, d)}
    names = ["o", "lse"] + (["dq", "dk", "dv"] if do is not None else [])
    out = {x: torch.zeros(shapes[x], dtype=torch.float64) for x in names}
    tol = {x: torch.zeros(shapes[x], dtype=torch.float64) for x in names}
    for b in range(B):
        L = n_kv if lengths is None else max(0, min(int(lengths[b]), n_kv))
        see = visible(n_q, n_kv, L, q_start, window, sinks, lookahead)
        for h in range(H):
            kv = h // G
            r = head(q[b, h], k[b, kv], v[b, kv], see, scale, None if do is None else do[b, h])
            t = bounds(r, q[b, h], k[b, kv], do, scale, dtype)
            for x in names:
                i = kv if x in ("dk", "dv") else h
                out[x][b, i] += r[x]
                tol[x][b, i] += t[x]
    return out, tol


def check(name, got, want, tol):
    got = got.detach().double().cpu()
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), finite), f"{name}: infinities or NaN in other places"
    assert torch.equal(got[~finite], want[~finite]), name
    over = (got - want).abs() - tol - 1e-30
    over[~finite] = -1
    if over.numel():
        i = int(over.argmax())
        assert over.flatten()[i] <= 0, (f"{name}: {got.flatten()[i]:.8g} for {want.flatten()[i]:.8g}, allowed "
                                        f"{tol.flatten()[i]:.3g} at {i} of {tuple(got.shape)}")


def norm_rope(x, w, inv_freq, pos, eps, interleaved, dy=None):
    """x [B, n, H, d], pos [B, n]: y [B, H, n, d] in 64 bits and, with dy,
    (dx, dw per head) and the magnitudes behind dw."""
    x = x.detach().double().cpu()
    d = x.shape[-1]
    w = torch.ones(d, dtype=torch.float64) if w is None else w.detach().double().cpu()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    half = 0 if inv_freq is None else inv_freq.numel()
    ang = pos.double().cpu()[:, :, None, None] * inv_freq.cpu() if half else torch.zeros(*x.shape[:2], 1, 0).double()
    c, s = torch.cos(ang), torch.sin(ang)
    ia = torch.arange(half) * (2 if interleaved else 1)
    ib = ia + (1 if interleaved else half)

    def turn(z, sign):
        z = z.clone()
        a, b = z[..., ia], z[..., ib]
        z[..., ia], z[..., ib] = a * c - sign * b * s, b * c + sign * a * s
        return z

    y = turn(x * r * w, 1.0).transpose(1, 2)
    if dy is None:
        return y
    g = turn(dy.detach().double().cpu().transpose(1, 2), -1.0)
    n = g * w
    dx = r * n - r ** 3 / d * x * (x * n).sum(-1, keepdim=True)
    mag = r * n.abs() + r ** 3 / d * x.abs() * (x * n).abs().sum(-1, keepdim=True)
    return y, dx, (g * x * r).sum((0, 1)), mag, (g * x * r).abs().sum((0, 1))
