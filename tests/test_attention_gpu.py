"""The attention entry points on the GPU against plain 64-bit forms, with
bounds derived from the arithmetic (attention_reference.py)."""
import math

import pytest
import torch

import paper_2505_23884_amd as P
from attention_reference import HALF, attention, bounds, check, head, norm_rope, visible

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rnd(seed, *shape, dtype=torch.bfloat16, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=F32) * scale).to(dtype)


def strided(x):
    """The same [B, H, n, d] values with heads behind tokens and a gap after each token."""
    B, H, n, d = x.shape
    big = torch.full((B, n, H + 1, d), float("nan"), dtype=x.dtype, device=x.device)
    big[:, :, :H] = x.transpose(1, 2)
    return big[:, :, :H].transpose(1, 2)


BF, F32 = torch.bfloat16, torch.float32
# B, H, Hkv, n_q, n_kv, d, options
WINDOW = [
    (1, 1, 1, 1, 1, 64, {}),
    (2, 2, 1, 33, 33, 64, {}),
    (1, 4, 2, 130, 130, 128, {}),
    (1, 2, 2, 300, 300, 128, dict(window=1)),
    (1, 2, 1, 257, 257, 128, dict(window=64, sinks=4)),
    (1, 6, 2, 200, 200, 80, dict(window=50, sinks=70)),
    (2, 5, 1, 190, 190, 96, dict(window=17, lookahead=9)),
    (1, 2, 2, 140, 140, 64, dict(window=None, lookahead=None)),
    (1, 2, 1, 150, 150, 256, dict(window=40, sinks=2)),
    (1, 1, 1, 70, 70, 200, dict(lookahead=None)),
    (2, 2, 2, 7, 150, 64, dict(window=100)),              # queries at the end of longer keys
    (1, 2, 1, 150, 20, 64, {}),                           # more queries than keys: the first see nothing
    (1, 2, 2, 100, 100, 64, dict(window=0)),              # empty windows
    (1, 2, 2, 100, 100, 64, dict(window=0, sinks=3)),
    (1, 2, 1, 100, 300, 8, dict(q_start=50, window=60, lookahead=20)),
    (1, 1, 1, 90, 64, 64, dict(q_start=-30, window=10, lookahead=4)),
    (3, 2, 1, 210, 210, 64, dict(window=64, sinks=1, lengths=[0, 1, 131])),
    (4, 2, 2, 140, 140, 128, dict(window=None, lookahead=None, lengths=[140, 64, 128, -5])),
    (2, 8, 1, 65, 65, 24, dict(scale=0.5)),
    (1, 2, 1, 1000, 1000, 64, dict(window=100, sinks=130)),
    (1, 2, 1, 5, 0, 64, {}),                              # no keys
    (1, 2, 1, 0, 5, 64, {}),                              # no queries
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("i", range(len(WINDOW)))
def test_window_attention_matches_the_formula(i, dtype):
    B, H, Hkv, n_q, n_kv, d, opt = WINDOW[i]
    opt = dict(opt)
    q, k, v, do = (rnd(10 * i + x, B, h, n, d, dtype=dtype) for x, h, n in
                   ((0, H, n_q), (1, Hkv, n_kv), (2, Hkv, n_kv), (3, H, n_q)))
    want, tol = attention(q, k, v, do=do, **opt)
    if "lengths" in opt:
        opt["lengths"] = torch.tensor(opt["lengths"], dtype=torch.int32, device=DEV)
    q, k, v, do = (x.to(DEV) for x in (q, k, v, do))
    if i % 2:
        q, k, v, do = (strided(x) for x in (q, k, v, do))
    print(f"[gpu] window {WINDOW[i]} {dtype}", flush=True)
    o, lse = P.window_attention(q, k, v, with_lse=True, **opt)
    torch.cuda.synchronize()
    check("o", o, want["o"], tol["o"])
    check("lse", lse, want["lse"], tol["lse"])
    dq, dk, dv = P.window_attention_backward(q, k, v, o, lse, do, **opt)
    torch.cuda.synchronize()
    for name, got in (("dq", dq), ("dk", dk), ("dv", dv)):
        check(name, got, want[name], tol[name])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("n,d,opt", [(150, 64, dict(window=20, sinks=2)), (200, 128, dict(window=70)), (90, 256, {}),
                                     (130, 64, dict(window=10, lookahead=10)),
                                     (140, 128, dict(lookahead=None, lengths=[100]))])
def test_infinities_and_nan_reach_only_what_sees_them(n, d, opt, value, dtype):
    opt = dict(opt)
    H, Hkv, at = 2, 1, 75
    L = opt["lengths"][0] if "lengths" in opt else n
    q, k, v, do = (rnd(x, 1, h, n, d, dtype=dtype).to(DEV) for x, h in ((0, H), (1, Hkv), (2, Hkv), (3, H)))
    if "lengths" in opt:
        opt["lengths"] = torch.tensor(opt["lengths"], dtype=torch.int32, device=DEV)
    see = visible(n, n, L, 0, opt.get("window"), opt.get("sinks", 0), opt.get("lookahead", 0))
    o0, lse0 = P.window_attention(q, k, v, with_lse=True, **opt)
    g0 = P.window_attention_backward(q, k, v, o0, lse0, do, **opt)

    def spoil(x, rows):
        x = x.clone()
        x[:, :, rows, 5] = value
        return x

    def same(name, got, want, rows):      # rows that cannot be reached: bitwise as before
        assert torch.equal(got[:, :, rows.to(DEV)], want[:, :, rows.to(DEV)]), name

    for rows in ([at], [n - 1] if L < n else [at, 3]):
        hit_q = see[:, rows].any(1)                 # queries that see such a key
        hit_k = see[rows].any(0)                    # keys that such a query sees
        print(f"[gpu] nonfinite n={n} d={d} {opt} {value} rows {rows} {dtype}", flush=True)
        o, lse = P.window_attention(q, k, spoil(v, rows), with_lse=True, **opt)
        same("o", o, o0, ~hit_q)
        assert torch.equal(lse, lse0)
        assert bool((~torch.isfinite(o[:, :, hit_q.to(DEV), 5].float())).all())
        if math.isinf(value):
            assert bool((o[:, :, hit_q.to(DEV), 5] == value).all())
        o, lse = P.window_attention(q, spoil(k, rows), v, with_lse=True, **opt)
        same("o of k", o, o0, ~hit_q)
        dq, dk, dv = P.window_attention_backward(q, spoil(k, rows), v, o, lse, do, **opt)
        same("dq of k", dq, g0[0], ~hit_q)
        far = ~see[hit_q].any(0)                    # keys that no such query sees
        same("dk of k", dk, g0[1], far)
        same("dv of k", dv, g0[2], far)
        do2 = spoil(do, rows)
        dq, dk, dv = P.window_attention_backward(q, k, v, o0, lse0, do2, **opt)
        rest = torch.ones(n, dtype=torch.bool)
        rest[rows] = False
        same("dq of do", dq, g0[0], rest)
        same("dk of do", dk, g0[1], ~hit_k)
        same("dv of do", dv, g0[2], ~hit_k)
        assert bool((~torch.isfinite(dv[:, :, hit_k.to(DEV), 5].float())).all())
        q2 = spoil(q, rows)
        o, lse = P.window_attention(q2, k, v, with_lse=True, **opt)
        same("o of q", o, o0, rest)
        dq, dk, dv = P.window_attention_backward(q2, k, v, o, lse, do, **opt)
        same("dq of q", dq, g0[0], rest)
        same("dk of q", dk, g0[1], ~hit_k)
        same("dv of q", dv, g0[2], ~hit_k)


ROPE = [
    # B, n, H, Hkv, d, rot, interleaved, per_head, far
    (1, 1, 1, 1, 8, 8, False, False, 0),
    (2, 5, 3, 1, 64, 64, False, False, 0),
    (1, 40, 4, 2, 128, 128, False, False, 100000),
    (3, 17, 2, 2, 128, 64, False, True, 0),
    (1, 33, 5, 1, 80, 40, False, False, 7),
    (2, 9, 2, 1, 96, 96, True, False, 1000000),
    (1, 21, 2, 1, 64, 6, True, True, 3),
    (2, 3, 2, 2, 256, 0, False, False, 0),
    (1, 70, 1, 1, 512, 512, False, False, 0),
    (1, 2100, 2, 1, 72, 16, False, False, 0),
    (3, 6001, 2, 1, 64, 32, False, False, 50000),
    (1, 20000, 1, 1, 64, 64, True, True, 0),
    (2, 9001, 4, 2, 128, 128, False, True, 5),
    (1, 17000, 5, 1, 256, 256, False, False, 9),
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("i", range(len(ROPE)))
def test_qk_norm_rope_matches_the_formula(i, dtype):
    B, n, H, Hkv, d, rot, inter, per_head, far = ROPE[i]
    fused = rnd(i, B, n, H + 2 * Hkv, d, dtype=dtype).to(DEV)
    q, k = fused[:, :, :H], fused[:, :, H:H + Hkv]
    wq, wk = ((torch.rand(*((h, d) if per_head else (d,)), generator=torch.Generator().manual_seed(i + 50), dtype=F32) + 0.5).to(DEV)
              for h in (H, Hkv))
    if i == 0:
        wk = None
    inv = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).to(DEV) if rot else None
    pos = torch.arange(n, dtype=torch.int32).repeat(B, 1) * (1 if i % 3 else -1) + far
    kw = dict(eps=1e-5, interleaved=inter)
    if i % 2:
        kw["positions"] = pos.to(DEV)
    else:
        kw["pos0"] = far
        pos = torch.arange(n, dtype=torch.int32).repeat(B, 1) + far
    dqn, dkn = rnd(i + 7, B, H, n, d, dtype=dtype).to(DEV), rnd(i + 8, B, Hkv, n, d, dtype=dtype).to(DEV)
    print(f"[gpu] rope {ROPE[i]} {dtype}", flush=True)
    qn, kn = P.qk_norm_rope(q, k, wq, wk, inv, **kw)
    dq, dk, dwq, dwk = P.qk_norm_rope_backward(q, k, dqn, dkn, wq, wk, inv, **kw)
    torch.cuda.synchronize()
    h, u = HALF[dtype], 2.0 ** -24
    for x, w, y, dy, dx, dw, name in ((q, wq, qn, dqn, dq, dwq, "q"), (k, wk, kn, dkn, dk, dwk, "k")):
        ry, rdx, rdw, mag, wmag = norm_rope(x, w, inv, pos, 1e-5, inter, dy)
        # norm and products: d + 16 roundings; the angle's sine and cosine: a step each of 2 pi 2^-24
        e = (d + 32) * u
        amp = (x.double().abs().cpu() * (1.0 if w is None else w.double().cpu().abs())).amax(-1).transpose(1, 2)[..., None]
        r = (1.0 / torch.sqrt(x.double().cpu().square().mean(-1) + 1e-5)).transpose(1, 2)[..., None]
        check(name + "n", y, ry, ry.abs() * h + amp * r * e)
        check("d" + name, dx, rdx, rdx.abs() * h + mag.amax(-1, keepdim=True) * e * 2)
        if w is None:
            assert dw is None
        else:
            if not per_head:
                rdw, wmag = rdw.sum(0), wmag.sum(0)
            check("dw" + name, dw, rdw, wmag.max() * (e + B * n * H * u) + rdw.abs() * u)


def paged_setup(lens, new, H, Hkv, d, page, dtype, seed=0, extra=2):
    B = len(lens)
    width = max(1, max(-(-x // page) for x in lens)) + 1
    pages = B * width + extra
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:B * width].view(B, width)
    cu = [0]
    for x in new:
        cu.append(cu[-1] + x)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    kc, vc = (torch.full((pages, page, Hkv, d), float("nan"), dtype=dtype) for _ in range(2))
    K = [rnd(seed + 3 * b + 1, 1, Hkv, lens[b], d, dtype=dtype) for b in range(B)]
    V = [rnd(seed + 3 * b + 2, 1, Hkv, lens[b], d, dtype=dtype) for b in range(B)]
    for b in range(B):
        for p in range(lens[b]):
            kc[perm[b, p // page], p % page] = K[b][0, :, p]
            vc[perm[b, p // page], p % page] = V[b][0, :, p]
    q = rnd(seed + 99, cu[-1] + extra, H, d, dtype=dtype)
    return q.to(DEV), kc.to(DEV), vc.to(DEV), i32(perm.tolist()), i32(lens), i32(cu), K, V, cu


PAGED = [
    # lens, new, H, Hkv, d, page, options
    ([1], [1], 1, 1, 64, 16, {}),
    ([40, 1, 300], [1, 1, 1], 4, 1, 128, 16, {}),
    ([130, 7, 65, 257], [1, 1, 1, 1], 8, 2, 64, 24, dict(window=50, sinks=3)),
    ([600], [1], 16, 2, 128, 1, dict(window=64, sinks=1)),
    ([70, 200, 5], [70, 33, 5], 4, 2, 128, 7, {}),
    ([300, 90], [200, 1], 6, 2, 80, 16, dict(window=40, sinks=70)),
    ([64, 0, 128], [3, 0, 128], 5, 1, 96, 32, {}),
    ([100, 31], [4, 31], 2, 2, 256, 64, dict(window=20)),
    ([3, 10], [5, 2], 2, 1, 64, 4, {}),                  # more new tokens than the sequence holds
    ([1500], [1], 4, 4, 64, 128, dict(scale=0.2)),
    ([50, 60], [1, 1], 2, 1, 64, 16, dict(window=0)),
    ([900, 2000], [130, 257], 8, 4, 64, 128, dict(window=300, sinks=5)),
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("i", range(len(PAGED)))
def test_paged_attention_matches_the_formula(i, dtype):
    lens, new, H, Hkv, d, page, opt = PAGED[i]
    q, kc, vc, table, ln, cu_new, K, V, cu = paged_setup(lens, new, H, Hkv, d, page, dtype, seed=100 * i)
    out = torch.full_like(q, 7.0)
    print(f"[gpu] paged {PAGED[i]} {dtype}", flush=True)
    P.paged_attention(q, kc, vc, table, ln, cu_new, out=out, **opt)
    torch.cuda.synchronize()
    for b in range(len(lens)):
        if not new[b]:
            continue
        qb = q[cu[b]:cu[b + 1]].transpose(0, 1)[None].cpu()
        want, tol = attention(qb, K[b], V[b], q_start=lens[b] - new[b], **opt)
        check(f"sequence {b}", out[cu[b]:cu[b + 1]].transpose(0, 1)[None], want["o"], tol["o"])
    assert bool((out[cu[-1]:] == 7.0).all())               # rows of no sequence


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("lens,new,Hkv,d,page", [([1], [1], 1, 8, 1), ([40, 17, 64], [1, 17, 30], 2, 128, 16),
                                                 ([5, 9], [0, 9], 3, 80, 7), ([3], [6], 1, 64, 4)])
def test_paged_append_writes_the_slots_and_nothing_else(lens, new, Hkv, d, page, dtype):
    q, kc, vc, table, ln, cu_new, _, _, cu = paged_setup(lens, new, Hkv, Hkv, d, page, dtype, seed=5)
    k, v = rnd(1, cu[-1] + 2, Hkv, d, dtype=dtype).to(DEV), rnd(2, cu[-1] + 2, Hkv, d, dtype=dtype).to(DEV)
    kw, vw = torch.nan_to_num(kc, nan=3.0), torch.nan_to_num(vc, nan=3.0)
    kc, vc = kw.clone(), vw.clone()
    for b in range(len(lens)):
        for x in range(new[b]):
            p = lens[b] - new[b] + x
            if p >= 0:
                kw[table[b, p // page].item(), p % page] = k[cu[b] + x]
                vw[table[b, p // page].item(), p % page] = v[cu[b] + x]
    P.paged_append(k, v, kc, vc, table, ln, cu_new)
    torch.cuda.synchronize()
    assert torch.equal(kc, kw) and torch.equal(vc, vw)


def test_pages_outside_the_cache_hold_nothing():
    lens, new, H, Hkv, d, page = [100, 70], [3, 1], 4, 2, 64, 16
    q, kc, vc, table, ln, cu_new, K, V, cu = paged_setup(lens, new, H, Hkv, d, page, BF, seed=3)
    table[0, 2], table[1, 0], table[1, 4] = -1, kc.shape[0], 2 ** 31 - 1
    gone = {0: [(32, 48)], 1: [(0, 16), (64, 80)]}
    o = P.paged_attention(q, kc, vc, table, ln, cu_new)
    torch.cuda.synchronize()
    for b in range(2):
        keep = torch.ones(lens[b], dtype=torch.bool)
        for x, y in gone[b]:
            keep[x:y] = False
        for i in range(new[b]):           # each token over the keys that are there, all of them before it
            p = lens[b] - new[b] + i
            rows = keep.clone()
            rows[p + 1:] = False
            if not rows.any():
                continue
            qb = q[cu[b] + i][None, :, None].cpu()
            want, tol = attention(qb, K[b][:, :, rows], V[b][:, :, rows], lookahead=None)
            check(f"{b} {i}", o[cu[b] + i][None, :, None], want["o"], tol["o"])
    k = rnd(9, 4, Hkv, d).to(DEV)
    before = kc.clone()
    P.paged_append(k, k, kc, vc, table, ln, cu_new)
    torch.cuda.synchronize()
    changed = (kc.view(torch.int16) != before.view(torch.int16)).flatten(2).any(-1)
    want = torch.zeros_like(changed)
    for i, p in enumerate((97, 98, 99)):
        want[table[0, p // page].item(), p % page] = True
    assert torch.equal(changed, want)      # the second sequence's slot lies on a page that is none


def test_lengths_and_offsets_out_of_range_are_clamped():
    q, kc, vc, table, ln, cu_new, K, V, cu = paged_setup([40, 50], [2, 3], 2, 1, 64, 16, BF, seed=4)
    width = table.shape[1] * 16
    out = torch.full_like(q, 7.0)
    P.paged_attention(torch.nan_to_num(q), torch.nan_to_num(kc), torch.nan_to_num(vc), table,
                      torch.tensor([width + 1000, -5], dtype=torch.int32, device=DEV), cu_new, out=out)
    torch.cuda.synchronize()
    assert bool((out[2:5] == 0).all())                       # a sequence of no tokens: nothing to see
    assert bool(torch.isfinite(out[:2].float()).all()) and bool((out[5:] == 7.0).all())
    out.fill_(7.0)
    P.paged_attention(q, kc, vc, table, ln, torch.tensor([0, 100000, 100000], dtype=torch.int32, device=DEV), out=out)
    torch.cuda.synchronize()


def test_cache_of_more_than_four_gigabytes():
    pages, page, Hkv, d = 40000, 64, 8, 128
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("needs 14 GB of GPU memory")
    kc, vc = (torch.zeros(pages, page, Hkv, d, dtype=BF, device=DEV) for _ in range(2))
    last = [pages - 1, pages - 2, 39000, 5]
    table = torch.tensor([last], dtype=torch.int32, device=DEV)
    K, V = rnd(1, 1, Hkv, 200, d), rnd(2, 1, Hkv, 200, d)
    ln, cu_new = torch.tensor([200], dtype=torch.int32, device=DEV), torch.tensor([0, 200], dtype=torch.int32, device=DEV)
    P.paged_append(K[0].transpose(0, 1).contiguous().to(DEV), V[0].transpose(0, 1).contiguous().to(DEV), kc, vc, table, ln, cu_new)
    for H, new in ((8, 1), (16, 1), (8, 150)):
        q = rnd(3, new, H, d).to(DEV)
        cu = torch.tensor([0, new], dtype=torch.int32, device=DEV)
        o = P.paged_attention(q, kc, vc, table, ln, cu, window=90, sinks=2)
        torch.cuda.synchronize()
        want, tol = attention(q.transpose(0, 1)[None].cpu(), K, V, q_start=200 - new, window=90, sinks=2)
        check(f"H {H} new {new}", o.transpose(0, 1)[None], want["o"], tol["o"])


def layer(q, k, v, wq, wk, inv, do, **opt):
    """Forward and reverse of one layer's attention half."""
    qn, kn = P.qk_norm_rope(q, k, wq, wk, inv)
    vt = v.transpose(1, 2)
    o, lse = P.window_attention(qn, kn, vt, with_lse=True, **opt)
    dqn, dkn, dv = P.window_attention_backward(qn, kn, vt, o, lse, do, **opt)
    dq, dk, dwq, dwk = P.qk_norm_rope_backward(q, k, dqn, dkn, wq, wk, inv)
    return o, dq, dk, dv, dwq, dwk


def layer_inputs(seed=0, B=2, n=150, H=4, Hkv=2, d=64, dtype=BF):
    fused = rnd(seed, B, n, H + 2 * Hkv, d, dtype=dtype).to(DEV)
    wq, wk = (torch.rand(d, generator=torch.Generator().manual_seed(seed + x), dtype=F32).to(DEV) + 0.5 for x in (1, 2))
    inv = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).to(DEV)
    return fused[:, :, :H], fused[:, :, H:H + Hkv], fused[:, :, H + Hkv:], wq, wk, inv, rnd(seed + 3, B, H, n, d, dtype=dtype).to(DEV)


OPT = dict(window=40, sinks=2)


def test_two_runs_are_bitwise_equal():
    x = layer_inputs()
    for a, b in zip(layer(*x, **OPT), layer(*x, **OPT)):
        assert torch.equal(a, b)


def test_chain_in_fp32_against_differences():
    x = q, k, v, wq, wk, inv, do = tuple(t.clone() for t in layer_inputs(5, B=1, n=40, H=2, Hkv=1, d=16, dtype=F32))
    got = layer(*x, **OPT)[1:]
    pos = torch.arange(40)[None]
    see = visible(40, 40, 40, 0, OPT["window"], OPT["sinks"], 0)
    g64 = do.double().cpu()

    def normed(a, w):
        return norm_rope(a, w, inv, pos, 1e-6, False)

    def loss(a, b, c, u, w):      # the layer's definition in 64 bits
        qn, kn = normed(a, u), normed(b, w)
        return float(sum((head(qn[0, h], kn[0, 0], c[0, :, 0], see, 0.25)["o"] * g64[0, h]).sum() for h in range(2)))

    base = [t.double().cpu() for t in (q, k, v, wq, wk)]
    # The attention's bounds for its cotangents, twice for the rounding of its own
    # inputs, through the norm: its reverse is a linear map of norm at most
    # 2 max(r w), and an element of a weight's gradient is a product with a column of x r.
    _, tol = attention(normed(q, wq).float(), normed(k, wk).float(), v.transpose(1, 2), do=do, **OPT)
    unit = [t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt() for t in base[:2]]
    gain = [float(((t.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w).max()) for t, w in zip(base[:2], base[3:])]
    n = [2 * float(tol[y].norm()) for y in ("dq", "dk", "dv")]
    bound = [2 * gain[0] * n[0], 2 * gain[1] * n[1], n[2], *(n[i] * float(unit[i].flatten(0, 2).norm(dim=0).max()) for i in (0, 1))]
    for i, g in enumerate((got[0], got[1], got[2].transpose(1, 2), got[3], got[4])):
        step = rnd(20 + i, *base[i].shape, dtype=torch.float64)
        h = 1e-5
        at = [loss(*(t + (sign * h * step if j == i else 0) for j, t in enumerate(base))) for sign in (1, -1)]
        want = (at[0] - at[1]) / (2 * h)
        have = float((g.double().cpu() * step).sum())
        assert abs(have - want) <= bound[i] * float(step.norm()) + 1e-7 * abs(want), i
        assert bound[i] < 0.02 * float(g.norm()), i      # (a bound that would notice a missing term)


def test_decoding_token_by_token_matches_the_prefill():
    B, n, H, Hkv, d, page = 2, 90, 4, 2, 64, 16
    q, k, v, wq, wk, inv, _ = layer_inputs(7, B, n, H, Hkv, d)
    qn, kn = P.qk_norm_rope(q, k, wq, wk, inv)
    want, tol = attention(qn, kn, v.transpose(1, 2).contiguous(), **OPT)
    width = -(-n // page)
    kc, vc = (torch.full((B * width, page, Hkv, d), float("nan"), dtype=BF, device=DEV) for _ in range(2))
    table = torch.randperm(B * width, generator=torch.Generator().manual_seed(1)).view(B, width).to(DEV, torch.int32)
    done = 0
    got = torch.empty(B, n, H, d, dtype=BF, device=DEV)
    for m in (50, 1, 1, 20, 1, 17):       # a prompt, tokens, a chunk, ...
        at = slice(done, done + m)
        done += m
        qt, kt = P.qk_norm_rope(q[:, at], k[:, at], wq, wk, inv, pos0=done - m)
        rows = lambda t, h: t.transpose(1, 2).reshape(B * m, h, d)
        ln = torch.full((B,), done, dtype=torch.int32, device=DEV)
        cu = torch.arange(0, (B + 1) * m, m, dtype=torch.int32, device=DEV)
        P.paged_append(rows(kt, Hkv), v[:, at].reshape(B * m, Hkv, d), kc, vc, table, ln, cu)
        got[:, at] = P.paged_attention(rows(qt, H), kc, vc, table, ln, cu, **OPT).view(B, m, H, d)
    torch.cuda.synchronize()
    assert done == n
    check("decoded", got.transpose(1, 2), want["o"], tol["o"])


def test_captured_and_replayed_on_another_stream():
    x = layer_inputs(11)
    q, kc, vc, table, ln, cu_new, _, _, cu = paged_setup([300, 90], [1, 4], 4, 2, 64, 16, BF, seed=8)
    kc, vc, q = (torch.nan_to_num(t) for t in (kc, vc, q))
    new = rnd(12, q.shape[0], 2, 64).to(DEV)

    def step():
        P.paged_append(new, new, kc, vc, table, ln, cu_new)
        return (*layer(*x, **OPT), P.paged_attention(q, kc, vc, table, ln, cu_new, window=200, out=torch.zeros_like(q)))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        with torch.no_grad():
            x[0].copy_(rnd(30 + i, *x[0].shape))
            q.copy_(rnd(40 + i, *q.shape))
            new.copy_(rnd(50 + i, *new.shape))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in out]
        for a, b in zip(replayed, step()):
            assert torch.equal(a, b), i


def test_outputs_given_and_bindings_refuse():
    q, k, v = rnd(1, 2, 4, 70, 64).to(DEV), rnd(2, 2, 2, 70, 64).to(DEV), rnd(3, 2, 2, 70, 64).to(DEV)
    o, lse = P.window_attention(q, k, v, with_lse=True, **OPT)
    out = torch.full((2, 70, 4, 64), 9.0, dtype=BF, device=DEV)      # heads behind tokens
    P.window_attention(q, k, v, out=out.transpose(1, 2), **OPT)
    assert torch.equal(out.transpose(1, 2), o)
    do = rnd(4, 2, 4, 70, 64).to(DEV)
    want = P.window_attention_backward(q, k, v, o, lse, do, **OPT)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    fused = torch.full((2, 70, 8, 64), 9.0, dtype=BF, device=DEV)
    parts = [fused[:, :, a:b].transpose(1, 2) for a, b in ((0, 4), (4, 6), (6, 8))]
    P.window_attention_backward(q, k, v, o, lse, do, out=parts, workspace=ws, **OPT)
    for a, b in zip(parts, want):
        assert torch.equal(a, b)
    # keys of one head given to all of a batch's heads by a stride of zero: as if repeated
    kx, vx = k[:, :1].expand(2, 4, 70, 64), v[:, :1].expand(2, 4, 70, 64)
    assert torch.equal(P.window_attention(q, kx, vx, **OPT), P.window_attention(q, kx.contiguous(), vx.contiguous(), **OPT))
    bad = [lambda: P.window_attention(q, k, v.float()), lambda: P.window_attention(q, k, v[:, :, :60]),
           lambda: P.window_attention(q, k[:, :, :, :32], v), lambda: P.window_attention(q[0], k, v),
           lambda: P.window_attention(q.half(), k.half(), v.half()),
           lambda: P.window_attention(q, k, v, lengths=torch.tensor([70, 70], device=DEV)),
           lambda: P.window_attention(q.transpose(2, 3), k, v), lambda: P.window_attention(q, k.cpu(), v),
           lambda: P.window_attention(q, k, v, scale=-1.0), lambda: P.window_attention(q[:, :3], k, v),
           lambda: P.window_attention(q, k, v, out=torch.empty_like(q)[:, :1].expand_as(q)),
           lambda: P.window_attention_backward(q, k, v, o, None, do),
           lambda: P.window_attention_backward(q, k, v, o, lse, do, workspace=ws[:64]),
           lambda: P.qk_norm_rope(q, k, torch.ones(64, device=DEV, dtype=BF)),
           lambda: P.qk_norm_rope(q.transpose(1, 2), k.transpose(1, 2), inv_freq=torch.ones(33, device=DEV, dtype=torch.float64))]
    for i, call in enumerate(bad):
        with pytest.raises(P.LactError):
            call()
            pytest.fail(f"call {i} was taken")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_an_infinite_key_that_weighs_nothing_stays_out_of_the_others(dtype):
    # its score is -inf for every query, so the others' gradients are those without it
    q, k, v, do = (rnd(60 + i, 1, 2, 70, 64, dtype=dtype) for i in range(4))
    q[..., 5] = -q[..., 5].abs() - 0.1
    k[:, :, 30] = k[:, :, 30].abs()
    k[:, :, 30, 5] = math.inf
    without = [j for j in range(70) if j != 30]
    x = [t.to(DEV) for t in (q, k, v)]
    o, lse = P.window_attention(*x, lookahead=None, with_lse=True)
    dq, dk, dv = P.window_attention_backward(*x, o, lse, do.to(DEV), lookahead=None)
    see = torch.ones(70, 69, dtype=torch.bool)
    for h in range(2):
        r = head(q[0, h], k[0, h, without], v[0, h, without], see, 0.125, do[0, h])
        t = bounds(r, q[0, h], k[0, h, without], do, 0.125, dtype)
        check("o", o[0, h], r["o"], t["o"])
        check("dk", dk[0, h][without], r["dk"], t["dk"])
        check("dv", dv[0, h][without], r["dv"], t["dv"])
        assert bool((dv[0, h, 30] == 0).all()) and bool(torch.isnan(dq[0, h, :, 5]).all())


def test_work_on_a_given_stream_beside_the_current_one():
    # outputs and workspaces come from the given stream's memory, so that work of
    # the current stream, still queued, neither overwrites them nor is overwritten
    x = layer_inputs(13, n=400)
    want = layer(*x, **OPT)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    junk = []
    for _ in range(4):
        s = side.cuda_stream
        q, k, v, wq, wk, inv, do = x
        big = torch.full((1 << 22,), 3.0, device=DEV)
        del big                                              # its memory is free for the current stream only
        qn, kn = P.qk_norm_rope(q, k, wq, wk, inv, stream=s)
        vt = v.transpose(1, 2)
        o, lse = P.window_attention(qn, kn, vt, with_lse=True, stream=s, **OPT)
        dqn, dkn, dv = P.window_attention_backward(qn, kn, vt, o, lse, do, stream=s, **OPT)
        junk.append(torch.full((1 << 20,), float("nan"), device=DEV))
        dq, dk, dwq, dwk = P.qk_norm_rope_backward(q, k, dqn, dkn, wq, wk, inv, stream=s)
        side.synchronize()
        for a, b in zip((o, dq, dk, dv, dwq, dwk), want):
            assert torch.equal(a, b)
    torch.cuda.synchronize()


def test_many_sequences_and_mixed_lengths():
    # more sequences than a wave has lanes, and 64 of them: the two ways to find a row's sequence
    for B in (63, 64, 65, 130):
        lens = [1 + (37 * b) % 200 for b in range(B)]
        new = [min(1 + (b % 5) * (b % 3), n) if b % 7 else 0 for b, n in enumerate(lens)]
        q, kc, vc, table, ln, cu_new, K, V, cu = paged_setup(lens, new, 4, 2, 64, 16, BF, seed=B)
        o = P.paged_attention(q, kc, vc, table, ln, cu_new, window=70, sinks=1)
        torch.cuda.synchronize()
        for b in range(0, B, 9):
            if not new[b]:
                continue
            rows = slice(cu[b], cu[b] + new[b])
            want, tol = attention(q[rows].transpose(0, 1)[None].cpu(), K[b][:, :, :lens[b]], V[b][:, :, :lens[b]], window=70, sinks=1)
            check(f"{B} {b}", o[rows].transpose(0, 1)[None], want["o"], tol["o"])


# enough heads that a workgroup takes 128 queries, or keys, in either type
MANY = [
    (8, 20, 4, 150, 150, 64, dict(window=60, sinks=3)),
    (8, 20, 20, 140, 140, 128, dict(window=50, lookahead=7, lengths=[140, 1, 0, 129, 128, 64, 77, 139])),
    (8, 20, 4, 130, 200, 80, dict(window=90, sinks=70)),
    (8, 20, 10, 131, 131, 200, dict(lookahead=None)),
    (4, 80, 16, 129, 270, 128, {}),
    (6, 60, 20, 65, 65, 24, dict(window=1)),
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("i", range(len(MANY)))
def test_window_attention_of_many_heads(i, dtype):
    B, H, Hkv, n_q, n_kv, d, opt = MANY[i]
    opt = dict(opt)
    q, k, v, do = (rnd(10 * i + x, B, h, n, d, dtype=dtype) for x, h, n in
                   ((0, H, n_q), (1, Hkv, n_kv), (2, Hkv, n_kv), (3, H, n_q)))
    want, tol = attention(q, k, v, do=do, **opt)
    if "lengths" in opt:
        opt["lengths"] = torch.tensor(opt["lengths"], dtype=torch.int32, device=DEV)
    q, k, v, do = (strided(x.to(DEV)) if i % 2 else x.to(DEV) for x in (q, k, v, do))
    print(f"[gpu] window of many heads {MANY[i]} {dtype}", flush=True)
    o, lse = P.window_attention(q, k, v, with_lse=True, **opt)
    dq, dk, dv = P.window_attention_backward(q, k, v, o, lse, do, **opt)
    torch.cuda.synchronize()
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        check(name, got, want[name], tol[name])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("d,opt", [(64, dict(window=20, sinks=2)), (128, dict(window=70)), (128, dict(window=10, lookahead=10)),
                                   (200, {})])
def test_infinities_and_nan_of_one_head_of_many(d, opt, value, dtype):
    B, H, G, n, b, hk, rows = 8, 40, 2, 150, 3, 7, [75, 3]
    q, k, v, do = (rnd(x, B, h, n, d, dtype=dtype).to(DEV) for x, h in ((0, H), (1, H // G), (2, H // G), (3, H)))
    see = visible(n, n, n, 0, opt.get("window"), opt.get("sinks", 0), 0 if "lookahead" not in opt else opt["lookahead"])
    hit_q, hit_k = see[:, rows].any(1), see[rows].any(0)
    o0, lse0 = P.window_attention(q, k, v, with_lse=True, **opt)
    g0 = P.window_attention_backward(q, k, v, o0, lse0, do, **opt)
    print(f"[gpu] nonfinite of one head d={d} {opt} {value} {dtype}", flush=True)

    def spoil(x, h):
        x = x.clone()
        x[b, h, rows, 5] = value
        return x

    def same(name, got, want, h, where):      # everything but the rows that are reached in heads h of batch b
        keep = torch.ones(got.shape[:3], dtype=torch.bool, device=DEV)
        for x in h:
            keep[b, x] = ~where.to(DEV)
        assert torch.equal(got[keep], want[keep]), name

    heads = [hk * G, hk * G + 1]
    one = torch.zeros(n, dtype=torch.bool)
    one[rows] = True
    o, lse = P.window_attention(q, k, spoil(v, hk), with_lse=True, **opt)
    same("o", o, o0, heads, hit_q)
    assert torch.equal(lse, lse0)
    assert bool((~torch.isfinite(o[b, heads][:, hit_q.to(DEV), 5].float())).all())
    ks = spoil(k, hk)
    o, lse = P.window_attention(q, ks, v, with_lse=True, **opt)
    same("o of k", o, o0, heads, hit_q)
    dq, dk, dv = P.window_attention_backward(q, ks, v, o, lse, do, **opt)
    reached = see[hit_q].any(0)
    same("dq of k", dq, g0[0], heads, hit_q)
    same("dk of k", dk, g0[1], [hk], reached)
    same("dv of k", dv, g0[2], [hk], reached)
    dq, dk, dv = P.window_attention_backward(q, k, v, o0, lse0, spoil(do, heads[1]), **opt)
    same("dq of do", dq, g0[0], heads[1:], one)
    same("dk of do", dk, g0[1], [hk], hit_k)
    same("dv of do", dv, g0[2], [hk], hit_k)
    assert bool((~torch.isfinite(dv[b, hk, hit_k.to(DEV), 5].float())).all())
    qs = spoil(q, heads[1])
    o, lse = P.window_attention(qs, k, v, with_lse=True, **opt)
    same("o of q", o, o0, heads[1:], one)
    dq, dk, dv = P.window_attention_backward(qs, k, v, o, lse, do, **opt)
    same("dq of q", dq, g0[0], heads[1:], one)
    same("dk of q", dk, g0[1], [hk], hit_k)
    same("dv of q", dv, g0[2], [hk], hit_k)


# long caches: the keys of a row are cut into parts, and these joined
LONG = [
    # lens, new, H, Hkv, d, page, options
    ([5003], [1], 16, 4, 128, 64, dict(window=2048, sinks=4)),
    ([3000, 10, 0, 700], [1, 1, 0, 1], 8, 2, 64, 16, {}),
    ([2100, 40], [3, 2], 8, 8, 256, 32, dict(window=1500)),
    ([1100, 700], [200, 90], 4, 2, 128, 24, dict(sinks=70, window=400)),
    ([1300, 3], [150, 2], 4, 1, 64, 16, {}),
    ([900, 1200], [70, 129], 2, 2, 200, 16, {}),
    ([2500], [2000], 16, 16, 64, 16, {}),
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("i", range(len(LONG)))
def test_paged_attention_in_parts(i, dtype):
    lens, new, H, Hkv, d, page, opt = LONG[i]
    q, kc, vc, table, ln, cu_new, K, V, cu = paged_setup(lens, new, H, Hkv, d, page, dtype, seed=200 + i)
    print(f"[gpu] paged in parts {LONG[i]} {dtype}", flush=True)
    out = torch.full_like(q, 7.0)
    P.paged_attention(q, kc, vc, table, ln, cu_new, out=out, **opt)
    torch.cuda.synchronize()
    for b in range(len(lens)):
        rows = slice(cu[b], cu[b] + new[b])
        if new[b]:
            want, tol = attention(q[rows].transpose(0, 1)[None].cpu(), K[b], V[b], q_start=lens[b] - new[b], **opt)
            check(f"{b}", out[rows].transpose(0, 1)[None], want["o"], tol["o"])
    assert bool((out[cu[-1]:] == 7.0).all())
    again = torch.full_like(q, 7.0)
    P.paged_attention(q, kc, vc, table, ln, cu_new, out=again, **opt)
    assert torch.equal(again, out)


# few heads over long windows: the queries of a tile of keys, and the heads that share it, are cut into parts
PARTS = [
    (1, 2, 1, 1300, 1300, 64, {}),
    (1, 2, 2, 900, 900, 128, dict(window=700, sinks=3)),
    (1, 4, 1, 800, 800, 128, dict(lookahead=None, lengths=[650])),
    (2, 3, 1, 700, 1100, 80, dict(window=600, lookahead=40)),
    (1, 6, 1, 600, 600, 256, {}),
    (1, 1, 1, 1500, 1500, 64, dict(window=50, sinks=200)),
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("i", range(len(PARTS)))
def test_window_attention_backward_in_parts(i, dtype):
    B, H, Hkv, n_q, n_kv, d, opt = PARTS[i]
    opt = dict(opt)
    q, k, v, do = (rnd(500 + 10 * i + x, B, h, n, d, dtype=dtype) for x, h, n in
                   ((0, H, n_q), (1, Hkv, n_kv), (2, Hkv, n_kv), (3, H, n_q)))
    want, tol = attention(q, k, v, do=do, **opt)
    if "lengths" in opt:
        opt["lengths"] = torch.tensor(opt["lengths"], dtype=torch.int32, device=DEV)
    q, k, v, do = (x.to(DEV) for x in (q, k, v, do))
    print(f"[gpu] window in parts {PARTS[i]} {dtype}", flush=True)
    o, lse = P.window_attention(q, k, v, with_lse=True, **opt)
    dq, dk, dv = P.window_attention_backward(q, k, v, o, lse, do, **opt)
    torch.cuda.synchronize()
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        check(name, got, want[name], tol[name])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_scores_of_large_magnitude(dtype):
    # rows that are all but one-hot, and a maximum whose rounding alone is tens of units
    q, k, v = (rnd(700 + x, 2, 2, 200, 64, dtype=dtype) for x in range(3))
    for size in (1e2, 1e4):
        qs, ks = (q.float() * size).to(dtype), (k.float() * size).to(dtype)
        o, lse = P.window_attention(qs.to(DEV), ks.to(DEV), v.to(DEV), window=90, with_lse=True)
        want, tol = attention(qs, ks, v, window=90)
        assert bool(torch.isfinite(o.float()).all())
        # where the second largest score is further off than the scores' own rounding, o is the first's value
        s = qs.double() @ ks.double().transpose(2, 3) / 8
        s = torch.where(visible(200, 200, 200, 0, 90, 0, 0), s, torch.full_like(s, -math.inf))
        top, at = s.topk(2, dim=-1)
        sure = (top[..., 0] - top[..., 1] > 40 + 72 * 2.0 ** -23 * (qs.double().abs() @ ks.double().abs().transpose(2, 3)).amax(-1) / 8)
        sure[..., 0] = True
        first = torch.gather(v.double(), 2, at[..., :1].expand(-1, -1, -1, 64))
        assert sure.float().mean() > 0.5
        err = (o.double().cpu() - first).abs()[sure]
        assert float(err.max()) <= 2 * HALF[dtype] * float(v.abs().max()) + 1e-5      # the weight's and the output's rounding
        # a score is a sum of 64 products in fp32, off by up to 64 2^-24 of their magnitudes however
        # small the sum is, so relative to the magnitudes (attention_reference.head), not to lse
        check("lse", lse, want["lse"], tol["lse"])


@pytest.mark.parametrize("B,n,H,Hkv,d", [(4, 2, 40, 8, 80), (1, 2, 2, 2, 64), (1, 5, 2, 2, 128), (2, 40, 4, 2, 128), (2, 3, 4, 4, 256)])
def test_gradients_of_few_keys_are_rounded_once(B, n, H, Hkv, d):
    # score cotangents of few keys do not average their roundings: beside the output's own half
    # step there is 2^-15 of each term (their two bf16 parts) and the fp32 arithmetic, no more
    q, k, v, do = (rnd(800 + x, B, h, n, d).to(DEV) for x, h in ((0, H), (1, Hkv), (2, Hkv), (3, H)))
    o, lse = P.window_attention(q, k, v, with_lse=True)
    got = P.window_attention_backward(q, k, v, o, lse, do)
    see, scale, u, h = visible(n, n, n, 0, None, 0, 0), d ** -0.5, 2.0 ** -24, HALF[BF]
    want, tol = ([torch.zeros(t.shape, dtype=torch.float64) for t in got] for _ in range(2))
    for b in range(B):
        for i in range(H):
            j = i // (H // Hkv)
            qi, kj, vj, gi = (t.double().cpu() for t in (q[b, i], k[b, j], v[b, j], do[b, i]))
            r = head(qi, kj, vj, see, scale, gi)
            e = r["p"] * (r["e"] + 3 * (d + n + 8) * u) * (r["mdp"] + r["mdelta"]) + r["ds"].abs() * (2.0 ** -15 + r["e"])
            want[0][b, i] = r["dq"]
            tol[0][b, i] = e @ kj.abs() * scale
            want[1][b, j] += r["dk"]
            tol[1][b, j] += e.t() @ qi.abs() * scale
    for name, x, w, t in zip(("dq", "dk"), got, want, tol):
        check(name, x, w, 2 * t + w.abs() * h)      # (twice: the correction of delta carries the same errors)


# lens, new, H, Hkv, d, page, options, the sequence and positions of a value that is no number
SPOILT = [
    ([100], [1], 2, 1, 64, 16, {}, 0, (96, 97, 98, 99, 64, 3)),               # tiles of keys end past the length
    ([70, 130], [1, 3], 4, 2, 128, 24, dict(window=37, sinks=2), 1, (128, 129, 93, 94, 0, 1)),
    ([45], [1], 1, 1, 256, 7, dict(window=20), 0, (32, 35, 40, 44)),
    ([100], [70], 4, 2, 64, 16, {}, 0, (96, 99, 31, 33, 64)),                 # 128 rows a workgroup
    ([300, 9], [150, 9], 2, 2, 128, 16, dict(window=100, sinks=3), 0, (0, 2, 130, 192, 195, 256)),
    ([150], [140], 1, 1, 200, 16, dict(window=50), 0, (1, 64, 67, 96, 149)),
    ([3003], [1], 4, 1, 64, 64, dict(window=1027), 0, (3001, 2976, 2979, 1977, 1984)),      # keys in parts
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("i", range(len(SPOILT)))
def test_infinities_and_nan_in_pages_reach_every_row_that_sees_them(i, value, dtype):
    lens, new, H, Hkv, d, page, opt, b, where = SPOILT[i]
    q, kc, vc, table, ln, cu_new, _, _, cu = paged_setup(lens, new, H, Hkv, d, page, dtype, seed=300 + i)
    q = q[:cu[-1]].contiguous()
    print(f"[gpu] nonfinite in pages {SPOILT[i]} {value} {dtype}", flush=True)
    base = P.paged_attention(q, kc, vc, table, ln, cu_new, **opt)
    assert bool(torch.isfinite(base.float()).all())
    cols = torch.arange(d, device=DEV) % 3 == 1          # of every four, and eight, in a row some
    for at in where:
        spoilt = vc.clone()
        spoilt[table[b, at // page], at % page][:, cols] = value
        got = P.paged_attention(q, kc, spoilt, table, ln, cu_new, **opt)
        see = visible(new[b], lens[b], lens[b], lens[b] - new[b], opt.get("window"), opt.get("sinks", 0), 0)[:, at]
        assert bool(see.any())
        hit = torch.zeros(cu[-1], dtype=torch.bool)
        hit[cu[b]:cu[b + 1]] = see
        hit = hit.to(DEV)
        assert torch.equal(got[~hit], base[~hit]), at
        assert torch.equal(got[hit][..., ~cols], base[hit][..., ~cols]), at
        x = got[hit][..., cols]
        assert bool(torch.isnan(x).all() if math.isnan(value) else (x == value).all()), at


def clamped(B, H, d, n, splits):
    """Sequences whose offsets, but the first one's, lie past the new tokens: all n of them are the first's."""
    lens = [900 if splits else 60] + [40] * (B - 1)
    q, kc, vc, table, ln, _, K, V, _ = paged_setup(lens, [n] + [0] * (B - 1), H, 1, d, 16, BF, seed=B + n)
    q = q[:n].contiguous()
    cu = torch.tensor([-9] + [100000] * B, dtype=torch.int32, device=DEV)
    return q, kc, vc, table, ln, cu, K, V, lens


@pytest.mark.parametrize("B,n,splits", [(2, 5, False), (3, 40, False), (70, 5, False), (70, 90, False), (2, 4, True), (70, 4, True)])
def test_offsets_past_the_new_tokens_give_them_all_to_one_sequence(B, n, splits):
    q, kc, vc, table, ln, cu, K, V, lens = clamped(B, 4, 64, n, splits)
    o = P.paged_attention(q, kc, vc, table, ln, cu)
    torch.cuda.synchronize()
    want, tol = attention(q.transpose(0, 1)[None].cpu(), K[0], V[0], q_start=lens[0] - n)
    check("o", o.transpose(0, 1)[None], want["o"], tol["o"])


@pytest.mark.parametrize("B,n", [(2, 5), (70, 90)])
def test_append_takes_offsets_past_the_new_tokens_as_the_attention_does(B, n):
    _, kc, vc, table, ln, cu, _, _, lens = clamped(B, 4, 64, n, False)
    kc, vc = torch.nan_to_num(kc, nan=3.0), torch.nan_to_num(vc, nan=3.0)
    k, v = rnd(1, n, 1, 64).to(DEV), rnd(2, n, 1, 64).to(DEV)
    kw, vw = kc.clone(), vc.clone()
    for x in range(n):
        p = lens[0] - n + x
        if p >= 0:
            kw[table[0, p // 16].item(), p % 16], vw[table[0, p // 16].item(), p % 16] = k[x], v[x]
    P.paged_append(k, v, kc, vc, table, ln, cu)
    torch.cuda.synchronize()
    assert torch.equal(kc, kw) and torch.equal(vc, vw)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("size,eps", [(1e-14, 0.0), (1e-13, 1e-30), (1e15, 1e-6)])
@pytest.mark.parametrize("per_head", [False, True])
def test_norm_of_small_and_large_vectors(size, eps, per_head, dtype):
    # r = 1 / rms within fp32's range, r^3 past either end of it
    B, n, H, Hkv, d = 2, 9, 3, 1, 64
    q, k = rnd(1, B, n, H, d, dtype=F32).mul(size).to(dtype).to(DEV), rnd(2, B, n, Hkv, d, dtype=F32).mul(size).to(dtype).to(DEV)
    wq, wk = (rnd(s, *((h, d) if per_head else (d,)), dtype=F32).to(DEV) for s, h in ((3, H), (4, Hkv)))
    dqn, dkn = rnd(5, B, H, n, d, dtype=dtype).to(DEV), rnd(6, B, Hkv, n, d, dtype=dtype).to(DEV)
    inv = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).to(DEV)
    pos = torch.arange(n, dtype=torch.int32).repeat(B, 1)
    qn, kn = P.qk_norm_rope(q, k, wq, wk, inv, eps=eps)
    dq, dk, dwq, dwk = P.qk_norm_rope_backward(q, k, dqn, dkn, wq, wk, inv, eps=eps)
    torch.cuda.synchronize()
    h, u = HALF[dtype], 2.0 ** -24
    for x, w, y, dy, dx, dw, name in ((q, wq, qn, dqn, dq, dwq, "q"), (k, wk, kn, dkn, dk, dwk, "k")):
        ry, rdx, rdw, mag, wmag = norm_rope(x, w, inv, pos, eps, False, dy)
        e = (d + 32) * u
        r = 1.0 / torch.sqrt(x.double().cpu().square().mean(-1) + eps)
        amp = ((x.double().cpu() * w.double().cpu()).abs().amax(-1) * r).transpose(1, 2)[..., None]
        check(name + "n", y, ry, ry.abs() * h + amp * e)
        # half a step of the smallest normal number where an element of dx lies below it
        check("d" + name, dx, rdx, rdx.abs() * h + mag.amax(-1, keepdim=True) * e * 2 + 2.0 ** -126 * h)
        if not per_head:
            rdw, wmag = rdw.sum(0), wmag.sum(0)
        check("dw" + name, dw, rdw, wmag.max() * (e + B * n * H * u) + rdw.abs() * u)


def test_norm_of_the_most_tokens_that_a_launch_holds():
    n, d = (1 << 25) - 4, 264                             # pieces of four elements, four tokens a workgroup
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of GPU memory")
    x = rnd(1, 1, 1, 2, d).to(DEV)
    q, k = (x[:, :, i:i + 1].expand(1, n, 1, d) for i in range(2))
    inv = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).to(DEV)
    print(f"[gpu] norm of {n} tokens", flush=True)
    qn, kn = P.qk_norm_rope(q, k, None, None, inv, eps=1e-5)
    torch.cuda.synchronize()
    at = torch.tensor([0, 1, 4097, 1 << 22, (1 << 24) + 1, n - 5, n - 1])
    for t, y in ((q, qn), (k, kn)):
        want = norm_rope(t[:, :1].expand(1, len(at), 1, d).contiguous(), None, inv, at[None], 1e-5, False)
        amp = t[0, 0, 0].double().cpu()
        amp = float(amp.abs().max() / torch.sqrt(amp.square().mean() + 1e-5))
        # the angle's fp32 fraction of a turn: 2 pi 2^-24, as everywhere
        check("y", y[:, :, at.to(DEV)], want, want.abs() * HALF[BF] + amp * (d + 32) * 2.0 ** -24)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("B,H,n,d,cut", [(1, 2, 60, 64, 30), (1, 2, 200, 128, 70), (8, 16, 150, 64, 50), (1, 2, 100, 256, 99)])
def test_reverse_of_a_part_of_the_keys_with_the_whole_rows_lse(B, H, n, d, cut, dtype):
    # keys split over calls: each call's reverse takes the rows' o and lse over all keys, and gives its part
    q, k, v, do = (rnd(950 + x, B, H, n, d, dtype=dtype) for x in range(4))
    want, tol = attention(q, k, v, lookahead=None, do=do)
    qd, kd, vd, gd = (t.to(DEV) for t in (q, k, v, do))
    print(f"[gpu] parts of the keys B={B} H={H} n={n} d={d} cut={cut} {dtype}", flush=True)
    o, lse = P.window_attention(qd, kd, vd, lookahead=None, with_lse=True)
    parts = [P.window_attention_backward(qd, kd[:, :, a:b], vd[:, :, a:b], o, lse, gd, lookahead=None)
             for a, b in ((0, cut), (cut, n))]
    h = HALF[dtype]
    for x, name in ((1, "dk"), (2, "dv")):
        check(name, torch.cat([p[x] for p in parts], 2), want[name], tol[name])
    # dq: each part is rounded by itself, so the two half steps are of their own sizes
    dq = sum(p[0].double().cpu() for p in parts)
    check("dq", dq, want["dq"], tol["dq"] + sum(p[0].double().cpu().abs() for p in parts) * h * 1.01)


def few_keys(q, k, v, o, lse, do, **opt):
    """dq and dk of bf16 calls against 64 bits: rows that see 128 keys at most with the rounding of their outputs and
    2^-15 of each term (the two bf16 parts of a score's cotangent, delta freed of the rounding of o), the others with
    a half step of each cotangent and of o."""
    B, H, n_q, d = q.shape
    Hkv, n_kv = k.shape[1], k.shape[2]
    kw = dict(opt)
    if "lengths" in opt:
        kw["lengths"] = torch.tensor(opt["lengths"], dtype=torch.int32, device=DEV)
    got = P.window_attention_backward(q, k, v, o, lse, do, **kw)
    scale, u, h = d ** -0.5, 2.0 ** -24, HALF[BF]
    want, tol = ([torch.zeros(t.shape, dtype=torch.float64) for t in got] for _ in range(2))
    for b in range(B):
        L = opt["lengths"][b] if "lengths" in opt else n_kv
        see = visible(n_q, n_kv, L, opt.get("q_start", n_kv - n_q), opt.get("window"), opt.get("sinks", 0), opt.get("lookahead", 0))
        few = (see.sum(1, keepdim=True) <= 128).double()
        n = int(see.sum(1).max())
        for i in range(H):
            j = i // (H // Hkv)
            qi, kj, vj, gi = (t.double().cpu() for t in (q[b, i], k[b, j], v[b, j], do[b, i]))
            r = head(qi, kj, vj, see, scale, gi)
            t = bounds(r, qi, kj, gi, scale, BF)
            o_err = (gi.abs() * (t["o"] + r["o"].abs() * h)).sum(1, keepdim=True)
            e = r["p"] * (r["e"] + 3 * (d + n + 8) * u) * (r["mdp"] + r["mdelta"]) + r["ds"].abs() * (2.0 ** -15 + r["e"])
            e = e + (1 - few) * (r["p"] * o_err + r["ds"].abs() * h)
            want[0][b, i] = r["dq"]
            tol[0][b, i] = e @ kj.abs() * scale
            want[1][b, j] += r["dk"]
            tol[1][b, j] += e.t() @ qi.abs() * scale
    for name, x, w, t in zip(("dq", "dk"), got, want, tol):
        check(name, x, w, 2 * t + w.abs() * h)      # (twice: the correction of delta carries the same errors)


# B, H, Hkv, n_q, n_kv, d, options
FEW = [
    (1, 2, 1, 400, 400, 64, dict(window=2)),
    (1, 2, 2, 400, 400, 128, dict(window=8)),
    (1, 4, 2, 300, 300, 128, dict(window=60)),
    (2, 2, 1, 400, 400, 80, dict(window=40, sinks=3)),
    (1, 2, 2, 400, 400, 64, dict(window=128)),
    (1, 2, 1, 400, 400, 64, dict(window=129)),                    # all but the first rows see more
    (1, 2, 1, 300, 300, 128, {}),                                  # the rows around position 128
    (1, 2, 2, 200, 200, 256, dict(window=30)),
    (1, 2, 1, 200, 200, 256, {}),
    (1, 2, 1, 300, 300, 64, dict(window=0, sinks=5)),
    (1, 2, 2, 300, 300, 128, dict(window=70, sinks=90)),           # few by the window, many by the sinks
    (1, 2, 1, 100, 500, 64, dict(window=20)),                      # q_start 400
    (1, 2, 1, 300, 300, 64, dict(window=20, lookahead=15)),
    (1, 2, 1, 300, 300, 64, dict(window=30, lookahead=None)),      # few at the end only
    (1, 2, 1, 300, 300, 128, dict(window=None, lookahead=None)),   # nowhere few, the first positions neither
    (2, 2, 1, 300, 300, 64, dict(window=None, lookahead=None, lengths=[300, 100])),
    (8, 16, 4, 300, 300, 64, dict(window=16)),                     # 128 queries a workgroup
    (4, 32, 8, 300, 300, 128, dict(window=40, sinks=2)),
    (8, 16, 16, 200, 200, 128, {}),
]


@pytest.mark.parametrize("i", range(len(FEW)))
def test_rows_of_few_keys_wherever_they_stand(i):
    B, H, Hkv, n_q, n_kv, d, opt = FEW[i]
    q, k, v, do = (rnd(900 + 10 * i + x, B, h, n, d).to(DEV) for x, h, n in ((0, H, n_q), (1, Hkv, n_kv), (2, Hkv, n_kv), (3, H, n_q)))
    kw = dict(opt)
    if "lengths" in opt:
        kw["lengths"] = torch.tensor(opt["lengths"], dtype=torch.int32, device=DEV)
    print(f"[gpu] few keys {FEW[i]}", flush=True)
    o, lse = P.window_attention(q, k, v, with_lse=True, **kw)
    few_keys(q, k, v, o, lse, do, **opt)


# long calls, tiles and parts at every place: each visible pair is counted once
COUNTED = [
    (1, 2, 1, 2600, 2600, 64, dict(window=600, sinks=70)),
    (1, 4, 2, 2100, 2100, 128, dict(window=300, sinks=4)),
    (1, 2, 2, 1700, 1700, 128, {}),
    (2, 3, 1, 1000, 1300, 80, dict(window=500, lookahead=100, lengths=[1300, 900])),
    (1, 2, 1, 1500, 1500, 96, dict(window=None, lookahead=None)),
    (4, 32, 4, 520, 520, 64, dict(window=130, sinks=3)),
    (1, 2, 1, 900, 900, 256, dict(window=200)),
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("i", range(len(COUNTED)))
def test_every_visible_pair_is_counted_once(i, dtype):
    # Where every score is 0 a row's weights are one number, and with rows of the unit matrix
    # for values, cotangents, keys or queries an element of an output is a sum of equal signs over
    # every d-th pair: its bound is relative to itself, and one pair less or twice is past it.
    B, H, Hkv, n_q, n_kv, d, opt = COUNTED[i]
    opt = dict(opt)
    unit = lambda h, n: torch.eye(d, dtype=dtype)[torch.arange(n) % d].expand(B, h, n, d).contiguous()
    zero = lambda h, n: torch.zeros(B, h, n, d, dtype=dtype)
    first = lambda h, n: torch.zeros(B, h, n, d, dtype=dtype).index_fill(3, torch.tensor([0]), 1.0)
    sign = lambda h, n: first(h, n) * (1.0 - 2.0 * (torch.arange(n) % 2))[:, None].to(dtype)
    ln = opt.get("lengths")
    for q, k, v, do, names in ((zero(H, n_q), unit(Hkv, n_kv), unit(Hkv, n_kv), unit(H, n_q), ("o", "dv")),
                               (zero(H, n_q), unit(Hkv, n_kv), sign(Hkv, n_kv), first(H, n_q), ("dq",)),
                               (unit(H, n_q), zero(Hkv, n_kv), sign(Hkv, n_kv), first(H, n_q), ("dk",))):
        want, tol = attention(q, k, v, do=do, **opt)
        kw = dict(opt, lengths=torch.tensor(ln, dtype=torch.int32, device=DEV)) if ln else opt
        q, k, v, do = (t.to(DEV) for t in (q, k, v, do))
        print(f"[gpu] pairs {COUNTED[i]} {names} {dtype}", flush=True)
        o, lse = P.window_attention(q, k, v, with_lse=True, **kw)
        got = dict(zip(("dq", "dk", "dv"), P.window_attention_backward(q, k, v, o, lse, do, **kw)), o=o)
        for x in names:
            check(x, got[x], want[x], tol[x])


@pytest.mark.parametrize("lens,new,H,Hkv,d,page,opt", [
    ([40, 333], [1, 1], 16, 2, 128, 16, {}), ([700], [1], 4, 4, 64, 24, dict(window=500, sinks=3)), ([300, 90], [4, 2], 4, 1, 80, 16, {}),
    ([200], [3], 2, 2, 256, 32, {}), ([5003], [1], 16, 4, 128, 64, dict(window=2048, sinks=4)), ([1], [1], 2, 1, 64, 16, {})])
def test_tokens_over_pages_are_rounded_once(lens, new, H, Hkv, d, page, opt):
    # up to 32 rows (tokens times heads of a group) a sequence: beside the output's own half step
    # there is 2^-15 of each weight (its two bf16 parts) and the fp32 arithmetic, no more
    q, kc, vc, table, ln, cu_new, K, V, cu = paged_setup(lens, new, H, Hkv, d, page, BF, seed=400 + d)
    print(f"[gpu] tokens {lens} {new} {H} {Hkv} {d}", flush=True)
    o = P.paged_attention(q, kc, vc, table, ln, cu_new, **opt)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        see = visible(new[b], n, n, n - new[b], opt.get("window"), opt.get("sinks", 0), 0)
        for h in range(H):
            x, j = q[cu[b]:cu[b + 1], h].cpu(), h // (H // Hkv)
            r = head(x, K[b][0, j], V[b][0, j], see, d ** -0.5)
            check(f"{b} {h}", o[cu[b]:cu[b + 1], h], r["o"], r["o_mag"] * (r["e"] + 2.0 ** -15 + n * 2.0 ** -24) * 1.01 + r["o"].abs() * HALF[BF])
