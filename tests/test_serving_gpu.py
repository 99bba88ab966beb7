"""The cache in 8 bits and the attention of sequences that share a prefix, on
the GPU against plain 64-bit forms, with bounds derived from the arithmetic."""
import math

import pytest
import torch

import paper_2505_23884_amd as P
from attention_reference import HALF, attention, check, head, visible
from serving_reference import Cache, quantise, values

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
types = pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])


def rnd(seed, *shape, dtype=BF, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=F32) * scale).to(dtype)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def same(got, want, what=""):
    """Bitwise equal, any NaN equal to any (without a print of whole tensors)."""
    got, want = got.cpu(), want.cpu()
    assert got.shape == want.shape and got.dtype == want.dtype, what
    differ = got != want
    if got.dtype.is_floating_point:
        differ &= ~(torch.isnan(got) & torch.isnan(want))
    n = int(differ.sum())
    assert n == 0, f"{what}: {n} of {got.numel()} differ, first at {differ.nonzero()[0].tolist()}"


def offsets(new):
    cu = [0]
    for x in new:
        cu.append(cu[-1] + x)
    return cu


# ---------------------------------------------------------------- into the cache and back

def hard_vectors(d, dtype):
    """Vectors where the scale or the rounding can go wrong."""
    x = rnd(1, 40, d, dtype=F32)
    x[0] = 0
    x[1] = -0.0
    x[2, 3:] = 0
    x[3] *= 2.0 ** -125
    x[4] *= 2.0 ** -132                       # subnormal numbers among them
    x[5] *= 2.0 ** 120
    x[6, 1] = 3.3e38                          # more than 448 2^119
    x[7, 2], x[7, 5] = math.inf, -math.inf
    x[8, 4] = math.nan
    x[9] = math.nan
    for i in range(10, 20):                   # the largest at, just below and just above 448 2^e
        x[i] *= 0.1
        x[i, 0] = (448.0, 446.0, 450.0, 1.75, 1.765625, 1.7421875, -448.0, 2.0, 1.0, -1.75)[i - 10]
    for i in range(20, 30):                   # ties between two numbers, and beside them
        x[i] = torch.tensor([(2 * k + 17) / 32 * (1 + (0, 2.0 ** -7, -2.0 ** -7)[i % 3]) for k in range(d)], dtype=F32) * 0.25
        x[i, 0] = 448.0 if i % 2 else 1.75
    x[30] = torch.tensor([(2 * k + 1) * 2.0 ** -10 for k in range(d)], dtype=F32)      # ties of numbers below the least normal one
    x[30, 0] = 448.0
    return x.to(dtype)


@types
@pytest.mark.parametrize("Hkv,d,page,B", [(1, 16, 1, 1), (2, 64, 7, 3), (3, 80, 16, 5), (4, 128, 24, 70), (1, 256, 64, 2), (5, 144, 8, 65)])
def test_append_quantises_by_the_definition_and_writes_nothing_else(Hkv, d, page, B, dtype):
    hard = hard_vectors(d, dtype)
    new = [(7 * b + 3) % 11 for b in range(B)]
    new[0] = 40
    lens = [n + (5 * b) % 13 for b, n in enumerate(new)]
    cu = offsets(new)
    c = Cache(lens, Hkv, d, page, dtype, True, 3)
    total = cu[-1] + 3
    qkv = rnd(2, total, 2 * Hkv + 1, d, dtype=dtype)             # parts of a fused projection
    qkv[:40, 0] = hard
    qkv[:40, 2 * Hkv] = hard.flip(0)
    k, v = qkv.to(DEV)[:, :Hkv], qkv.to(DEV)[:, Hkv + 1:]
    kc, vc, ks, vs = c.on(DEV)
    want = [x.clone() for x in c.cache], [x.clone() for x in c.scales]
    for w, x in enumerate((k, v)):
        codes, scales = quantise(x)
        for b in range(B):
            for i in range(new[b]):
                p = lens[b] - new[b] + i
                at = c.table[b, p // page].item(), p % page
                want[0][w][at], want[1][w][at] = codes[cu[b] + i], scales[cu[b] + i]
    print(f"[gpu] append e4m3 {Hkv} {d} {page} {B} {dtype}", flush=True)
    P.paged_append_e4m3(k, v, kc, vc, ks, vs, c.table.to(DEV), i32(lens), i32(cu))
    torch.cuda.synchronize()
    for got, x in zip((kc, vc), want[0]):
        same(got.view(torch.uint8), x, "numbers")
    same(ks, want[1][0], "k_scale")
    same(vs, want[1][1], "v_scale")
    # and back: exactly what the numbers stand for
    kr, vr = (torch.full((total, Hkv, d), 7.0, dtype=dtype, device=DEV) for _ in range(2))
    P.paged_read_e4m3(kc, vc, ks, vs, c.table.to(DEV), i32(lens), i32(cu), total, out=(kr, vr))
    for got, x in ((kr, k), (vr, v)):
        same(got[:cu[-1]], values(*quantise(x)).to(dtype)[:cu[-1]], "read back")
        assert bool((got[cu[-1]:] == 7.0).all())


@types
def test_every_number_at_every_scale_is_read_exactly(dtype):
    scales = torch.arange(10, 247, dtype=torch.uint8)
    n = scales.numel()
    codes = torch.arange(256, dtype=torch.uint8).expand(n, 1, 1, 256).contiguous()
    kc = codes.view(torch.float8_e4m3fn).to(DEV)
    vc = codes.flip(-1).contiguous().view(torch.float8_e4m3fn).to(DEV)
    s = scales.view(n, 1, 1).to(DEV)
    k, v = P.paged_read_e4m3(kc, vc, s, s, torch.arange(n, dtype=torch.int32, device=DEV)[None], i32([n]), i32([0, n]), n, dtype=dtype)
    want = values(codes[:, 0], scales[:, None])
    for got, x in ((k, want), (v, want.flip(-1))):
        same(got.double(), x)


@pytest.mark.parametrize("binade", [0, 1, 7, -100])
def test_every_bf16_number_is_rounded_to_the_nearest(binade):
    # all magnitudes from 448 2^binade down: vectors of 16 with that as their first element
    top = torch.tensor([448.0 * 2.0 ** binade], dtype=BF).view(torch.int16).item()
    x = torch.arange(top + 1, dtype=torch.int16).view(BF)
    x = x[: x.numel() // 15 * 15].view(-1, 15)
    x = torch.cat([torch.full((x.shape[0], 1), 448.0 * 2.0 ** binade, dtype=BF), x * torch.tensor([1.0, -1.0] * 7 + [1.0], dtype=BF)], 1)[:, None]
    n = x.shape[0]
    kc, vc = (torch.zeros(1, n, 1, 16, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.zeros(1, n, 1, dtype=torch.uint8, device=DEV) for _ in range(2))
    P.paged_append_e4m3(x.to(DEV), x.to(DEV), kc, vc, ks, vs, i32([[0]]), i32([n]), i32([0, n]))
    codes, scales = quantise(x)
    same(ks[0], scales)
    same(kc[0].view(torch.uint8), codes)
    same(vs, ks)
    same(vc.view(torch.uint8), kc.view(torch.uint8))


def test_read_of_whole_sequences_and_of_what_is_not_there():
    lens, Hkv, d, page = [33, 0, 100, 5], 2, 64, 16
    c = Cache(lens, Hkv, d, page, BF, True, 5)
    table = c.table.clone()
    table[2, 1], table[0, 0], table[3, 0] = -1, 10 ** 6, c.cache[0].shape[0]
    cu = offsets(lens)
    rows = [n + 4 for n in lens]                       # more rows than a sequence holds: zeros before its first
    k, v = P.paged_read_e4m3(*c.on(DEV), c.table.to(DEV), i32(lens), i32(cu), cu[-1])
    for b in range(4):
        for got, x in ((k, c.kv[b][0]), (v, c.kv[b][1])):
            same(got[cu[b]:cu[b + 1]], x.transpose(0, 1))
    cu = offsets(rows)
    out = [torch.full((cu[-1] + 2, Hkv, d), 9.0, dtype=F32, device=DEV).transpose(0, 1).contiguous().transpose(0, 1) for _ in range(2)]
    P.paged_read_e4m3(*c.on(DEV), table.to(DEV), i32(lens), i32(cu), cu[-1] + 2, out=out)
    for w in range(2):
        for b in range(4):
            want = torch.cat([torch.zeros(4, Hkv, d, dtype=F32), c.kv[b][w].transpose(0, 1).float()])
            if b == 2:
                want[4 + 16:4 + 32] = 0
            if b in (0, 3):
                want[4:4 + 16] = 0
            same(out[w][cu[b]:cu[b + 1]], want, (w, b))
        assert bool((out[w][cu[-1]:] == 9.0).all())


# ---------------------------------------------------------------- attention over e4m3 numbers

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
    ([90], [2], 2, 1, 16, 5, {}),
    ([200, 77], [50, 2], 4, 4, 48, 16, {}),
    # keys in parts
    ([5003], [1], 16, 4, 128, 64, dict(window=2048, sinks=4)),
    ([3000, 10, 0, 700], [1, 1, 0, 1], 8, 2, 64, 16, {}),
    ([2100, 40], [3, 2], 8, 8, 256, 32, dict(window=1500)),
    ([1100, 700], [200, 90], 4, 2, 128, 24, dict(sinks=70, window=400)),
    ([900, 1200], [70, 129], 2, 2, 208, 16, {}),
]


def spread(out, fill=7.0):
    """A tensor like `out` whose heads lie behind its tokens, filled."""
    return torch.full((out.shape[1], out.shape[0], out.shape[2]), fill, dtype=out.dtype, device=out.device).transpose(0, 1)


@types
@pytest.mark.parametrize("i", range(len(PAGED)))
def test_attention_over_e4m3_matches_the_formula(i, dtype):
    lens, new, H, Hkv, d, page, opt = PAGED[i]
    c = Cache(lens, Hkv, d, page, dtype, True, 100 + i)
    cu = offsets(new)
    q = rnd(i, cu[-1] + 2, H, d, dtype=dtype).to(DEV)
    out = spread(q) if i % 2 else torch.full_like(q, 7.0)
    print(f"[gpu] e4m3 {PAGED[i]} {dtype}", flush=True)
    P.paged_attention_e4m3(q, *c.on(DEV), c.table.to(DEV), i32(lens), i32(cu), out=out, **opt)
    torch.cuda.synchronize()
    for b in range(len(lens)):
        if new[b]:
            rows = slice(cu[b], cu[b + 1])
            want, tol = attention(q[rows].transpose(0, 1)[None].cpu(), c.kv[b][0][None], c.kv[b][1][None],
                                  q_start=lens[b] - new[b], **opt)
            check(f"sequence {b}", out[rows].transpose(0, 1)[None], want["o"], tol["o"])
    assert bool((out[cu[-1]:] == 7.0).all())
    again = torch.full_like(q, 7.0)
    P.paged_attention_e4m3(q, *c.on(DEV), c.table.to(DEV), i32(lens), i32(cu), out=again, **opt)
    same(again, out)


# ---------------------------------------------------------------- shared prefixes

PREFIX = [
    # prefixes, sequences of each, lens, new, H, Hkv, d, page, options
    ([5], [2], [1, 1], [1, 1], 1, 1, 64, 16, {}),
    ([100], [3], [40, 1, 300], [1, 1, 1], 4, 1, 128, 16, {}),
    ([37, 64, 0], [1, 2, 1], [130, 7, 65, 20], [1, 1, 1, 1], 8, 2, 64, 24, dict(window=50, sinks=3)),
    ([90], [2], [30, 4], [1, 4], 4, 2, 128, 7, dict(window=10, sinks=100)),        # sinks end among a sequence's own keys
    ([90], [2], [30, 44], [2, 1], 4, 2, 96, 8, dict(window=40)),                   # windows that end in the prefix
    ([200], [3], [70, 200, 5], [70, 33, 5], 4, 2, 128, 16, {}),
    ([61], [2], [300, 90], [200, 1], 6, 2, 80, 16, dict(window=140, sinks=70)),
    ([64, 33], [2, 1], [64, 0, 128], [3, 0, 128], 5, 1, 96, 32, {}),
    ([70], [2], [100, 31], [4, 31], 2, 2, 256, 64, dict(window=60)),
    ([20], [3], [3, 10, 6], [5, 2, 6], 2, 1, 64, 4, {}),                           # more new tokens than a sequence holds
    ([20], [2], [0, 4], [3, 4], 2, 1, 64, 4, dict(window=12)),
    ([1500], [4], [9, 1, 2, 3], [1, 1, 1, 1], 16, 4, 128, 64, {}),                 # keys in parts
    ([2000, 700], [3, 2], [90, 10, 200, 300, 1], [1, 2, 1, 1, 1], 8, 2, 64, 16, dict(window=900, sinks=7)),
    ([800], [2], [600, 100], [130, 70], 4, 2, 128, 24, dict(sinks=30, window=400)),
    ([50, 60], [1, 1], [5, 6], [1, 1], 2, 1, 64, 16, dict(window=0)),
    ([300], [10], list(range(1, 11)), [1] * 10, 8, 2, 64, 32, dict(scale=0.3)),    # rows of a group fill several tiles
    ([333], [40], [2] * 40, [2] * 40, 8, 2, 64, 32, {}),
    ([40], [2], [10, 20], [2, 1], 4, 2, 16, 8, {}),
]


def prefix_call(c, q, out, plen, seqs, lens, cu, **opt):
    caches = c.on(DEV)
    kw = dict(opt) if not c.codes else dict(opt, k_scale=caches[2], v_scale=caches[3])
    return P.paged_prefix_attention(q, caches[0], caches[1], c.ptable.to(DEV), i32(plen), i32(seqs), c.table.to(DEV), i32(lens),
                                    i32(cu), out=out, **kw)


def check_prefix(out, q, c, plen, seqs, lens, cu, opt, only=None):
    """Every sequence against the formula over its prefix's keys and its own."""
    group = [-1] * len(lens)
    for g in range(len(plen)):
        for b in range(seqs[g], seqs[g + 1]):
            group[b] = g
    for b, n in enumerate(lens):
        m = cu[b + 1] - cu[b]
        if not m or (only is not None and b not in only):
            continue
        rows, g = slice(cu[b], cu[b + 1]), group[b]
        f = plen[g] if g >= 0 else 0
        k, v = (torch.cat([c.pkv[g][w], c.kv[b][w]], 1) if g >= 0 else c.kv[b][w] for w in range(2))
        held = min(m, n)                        # a token that the sequence does not hold sees nothing
        x = out[rows].transpose(0, 1)[None]
        assert bool((x[:, :, :m - held] == 0).all()), b
        if held:
            want, tol = attention(q[rows][m - held:].transpose(0, 1)[None].cpu(), k[None], v[None], q_start=f + n - held, **opt)
            check(f"sequence {b}", x[:, :, m - held:], want["o"], tol["o"])


@types
@pytest.mark.parametrize("codes", [False, True], ids=["plain", "e4m3"])
@pytest.mark.parametrize("i", range(len(PREFIX)))
def test_prefix_attention_matches_the_formula(i, codes, dtype):
    plen, counts, lens, new, H, Hkv, d, page, opt = PREFIX[i]
    c = Cache(lens, Hkv, d, page, dtype, codes, 200 + i, prefixes=plen)
    cu, seqs = offsets(new), offsets(counts)
    q = rnd(i, cu[-1] + 2, H, d, dtype=dtype).to(DEV)
    out = spread(q) if i % 2 else torch.full_like(q, 7.0)
    print(f"[gpu] prefix {PREFIX[i]} {codes} {dtype}", flush=True)
    prefix_call(c, q, out, plen, seqs, lens, cu, **opt)
    torch.cuda.synchronize()
    check_prefix(out, q, c, plen, seqs, lens, cu, opt)
    assert bool((out[cu[-1]:] == 7.0).all())
    again = torch.full_like(q, 7.0)
    prefix_call(c, q, again, plen, seqs, lens, cu, **opt)
    same(again, out)


@types
@pytest.mark.parametrize("d", [8, 24, 72, 200])
def test_prefix_attention_of_heads_of_eights(d, dtype):
    plen, lens = [70, 33], [40, 3, 90]
    for new in ([1, 1, 1], [4, 3, 9], [40, 3, 80]):
        c = Cache(lens, 2, d, 16, dtype, False, d, prefixes=plen)
        cu = offsets(new)
        q = rnd(d, cu[-1], 4, d, dtype=dtype).to(DEV)
        out = torch.full_like(q, 7.0)
        print(f"[gpu] prefix d {d} {new} {dtype}", flush=True)
        prefix_call(c, q, out, plen, [0, 2, 3], lens, cu, window=100, sinks=5)
        torch.cuda.synchronize()
        check_prefix(out, q, c, plen, [0, 2, 3], lens, cu, dict(window=100, sinks=5))


@pytest.mark.parametrize("codes", [False, True], ids=["plain", "e4m3"])
@pytest.mark.parametrize("B,groups,opt", [(63, 2, {}), (64, 64, dict(window=30, sinks=2)), (65, 3, {}), (130, 70, dict(window=25)), (130, 1, {})])
def test_many_sequences_and_groups(B, groups, opt, codes):
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 40, (B,), generator=g).tolist()
    new = [min(x, n) for x, n in zip(torch.randint(0, 3, (B,), generator=g).tolist(), lens)]
    plen = torch.randint(0, 60, (groups,), generator=g).tolist()
    edges = sorted(torch.randint(1, B, (groups - 1,), generator=g).tolist())      # groups of none among them
    seqs = [2] + [max(x, 2) for x in edges] + [B - 3]                             # sequences of no group at both ends
    seqs = [min(x, B - 3) for x in seqs]
    c = Cache(lens, 1, 64, 16, BF, codes, B, prefixes=plen)
    cu = offsets(new)
    q = rnd(3, cu[-1] + 1, 3, 64).to(DEV)
    out = torch.full_like(q, 7.0)
    print(f"[gpu] many {B} {groups} {codes}", flush=True)
    prefix_call(c, q, out, plen, seqs, lens, cu, **opt)
    torch.cuda.synchronize()
    check_prefix(out, q, c, plen, seqs, lens, cu, opt)
    assert bool((out[cu[-1]:] == 7.0).all())


# ---------------------------------------------------------------- what is not there, or is no number

# lens, new, H, Hkv, d, page, options, the sequence and positions of a value that is no number
SPOILT = [
    ([100], [1], 2, 1, 64, 16, {}, 0, (96, 97, 98, 99, 64, 3)),               # tiles of keys end past the length
    ([70, 130], [1, 3], 4, 2, 128, 24, dict(window=37, sinks=2), 1, (128, 129, 93, 94, 0, 1)),
    ([45], [1], 1, 1, 256, 7, dict(window=20), 0, (32, 35, 40, 44)),
    ([60], [9], 2, 1, 64, 16, dict(window=20), 0, (32, 35, 40, 59)),          # 32 rows a workgroup
    ([100], [70], 4, 2, 64, 16, {}, 0, (96, 99, 31, 33, 64)),                 # 128 rows
    ([300, 9], [150, 9], 2, 2, 128, 16, dict(window=100, sinks=3), 0, (0, 2, 130, 192, 195, 256)),
    ([150], [140], 1, 1, 208, 16, dict(window=50), 0, (1, 64, 67, 96, 149)),
    ([3003], [1], 4, 1, 64, 64, dict(window=1027), 0, (3001, 2976, 2979, 1977, 1984)),      # keys in parts
    ([3003], [1], 4, 2, 64, 64, dict(window=1027), 0, (3001, 2976, 2979, 1977, 1984)),      # two heads a workgroup
]


@types
@pytest.mark.parametrize("codes,prefix", [(True, 0), (True, 1), (False, 1)], ids=["e4m3", "e4m3-prefix", "plain-prefix"])
@pytest.mark.parametrize("i", range(len(SPOILT)))
def test_nan_in_pages_reach_every_row_that_sees_them_and_no_other(i, codes, prefix, dtype):
    lens, new, H, Hkv, d, page, opt, b, where = SPOILT[i]
    f = 75 if prefix else 0                       # keys of a prefix; the spoilt one is then the prefix's, or a sequence's own
    plen, seqs = ([f], [0, len(lens)]) if prefix else ([], [0])
    c = Cache(lens, Hkv, d, page, dtype, codes, 300 + i, prefixes=plen)
    cu = offsets(new)
    q = rnd(i, cu[-1], H, d, dtype=dtype).to(DEV)
    print(f"[gpu] nan in pages {SPOILT[i]} {codes} {prefix} {dtype}", flush=True)

    def call():
        out = torch.full_like(q, 7.0)
        if prefix:
            return prefix_call(c, q, out, plen, seqs, lens, cu, **opt)
        return P.paged_attention_e4m3(q, *c.on(DEV), c.table.to(DEV), i32(lens), i32(cu), out=out, **opt)

    base = call()
    assert bool(torch.isfinite(base.float()).all())
    cols = torch.arange(d) % 3 == 1
    group = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(new))          # a row's sequence
    pos = torch.cat([torch.arange(n - m, n) for n, m in zip(lens, new)])
    for own_key, at in [(True, x) for x in where] + [(False, x) for x in ((0, 31, 64, 74) if prefix else ())]:
        v, table = c.cache[1], c.table[b] if own_key else c.ptable[0]
        saved = v.clone()
        slot = v[table[at // page], at % page]
        slot[..., cols] = 0x7f if codes else math.nan
        p, j = f + pos, f + at if own_key else at
        see = j <= p
        if "window" in opt:
            see &= (j > p - opt["window"]) | (j < opt.get("sinks", 0))
        if own_key:
            see &= group == b
        got = call()
        c.cache[1] = saved
        if own_key and not prefix:        # (behind a prefix the sinks are among its keys)
            assert bool(see.any())
        same(got[~see.to(DEV)], base[~see.to(DEV)], ("rows that do not see it", own_key, at))
        hit = got[see.to(DEV)].cpu()
        same(hit[..., ~cols], base[see.to(DEV)].cpu()[..., ~cols], ("other columns", own_key, at))
        assert bool(torch.isnan(hit[..., cols]).all()), (own_key, at)


# lens, new, H, Hkv, d, options
NO_NUMBERS = [
    ([300, 40], [1, 1], 4, 2, 64, {}),                    # 16 rows, two heads a workgroup
    ([5000, 40], [1, 2], 4, 1, 128, {}),                  # keys in parts
    ([5000], [1], 2, 1, 64, dict(window=3000)),
    ([200, 90], [9, 5], 4, 2, 128, dict(window=50)),      # 32 rows
    ([200, 150], [150, 90], 4, 2, 64, dict(window=50, sinks=2)),
    ([9, 30], [12, 1], 2, 1, 256, {}),                    # rows that their sequence does not hold
]


@types
@pytest.mark.parametrize("codes,prefix", [(True, None), (True, 75), (True, 0), (False, 75), (False, 0)],
                         ids=["e4m3", "e4m3-prefix", "e4m3-empty-prefix", "plain-prefix", "plain-empty-prefix"])
@pytest.mark.parametrize("i", range(len(NO_NUMBERS)))
def test_queries_that_are_no_numbers_give_none(i, codes, prefix, dtype):
    lens, new, H, Hkv, d, opt = NO_NUMBERS[i]
    plen, seqs = ([], [0]) if prefix is None else ([prefix], [0, len(lens)])
    c = Cache(lens, Hkv, d, 16, dtype, codes, 700 + i, prefixes=plen)
    cu = offsets(new)
    q = rnd(i, cu[-1], H, d, dtype=dtype).to(DEV)
    print(f"[gpu] queries of nan {NO_NUMBERS[i]} {codes} {prefix} {dtype}", flush=True)

    def call(q):
        out = torch.full_like(q, 7.0)
        if prefix is not None:
            return prefix_call(c, q, out, plen, seqs, lens, cu, **opt)
        return P.paged_attention_e4m3(q, *c.on(DEV), c.table.to(DEV), i32(lens), i32(cu), out=out, **opt)

    base = call(q)
    for token, head in {(0, 0), (cu[-1] - 1, H - 1), (cu[-1] // 2, H // 2)}:
        spoilt = q.clone()
        spoilt[token, head, d // 2] = math.nan
        got = call(spoilt)
        b = max(x for x in range(len(lens)) if cu[x] <= token)
        if lens[b] - (cu[b + 1] - token) >= 0:            # a row that sees a key
            assert bool(torch.isnan(got[token, head].float()).all()), (token, head)
        else:
            assert bool((got[token, head] == 0).all()), (token, head)
        got[token, head] = base[token, head]
        same(got, base, (token, head))


@types
@pytest.mark.parametrize("codes,prefix", [(True, False), (True, True), (False, True)], ids=["e4m3", "e4m3-prefix", "plain-prefix"])
def test_a_key_of_nan_that_is_all_a_row_sees(codes, prefix, dtype):
    plen, seqs = ([20], [0, 1]) if prefix else ([], [0])
    c = Cache([3000, 30], 1, 64, 16, dtype, codes, 9, prefixes=plen)
    lens, cu = [3000, 30], [0, 1, 2]
    q = rnd(4, 2, 2, 64, dtype=dtype).to(DEV)
    slot = c.cache[0][c.table[0, 2999 // 16], 2999 % 16]
    slot[..., 5] = 0x7f if codes else math.nan
    opt = dict(window=1)
    got = (prefix_call(c, q, torch.full_like(q, 7.0), plen, seqs, lens, cu, **opt) if prefix else
           P.paged_attention_e4m3(q, *c.on(DEV), c.table.to(DEV), i32(lens), i32(cu), **opt))
    assert bool(torch.isnan(got[0].float()).all()) and bool(torch.isfinite(got[1].float()).all())


@pytest.mark.parametrize("codes", [False, True], ids=["plain", "e4m3"])
@pytest.mark.parametrize("new", [[3, 1], [90, 60]])
def test_pages_outside_the_cache_hold_nothing(new, codes):
    lens, H, Hkv, d, page, plen = [100, 70], 4, 2, 64, 16, [90]
    c = Cache(lens, Hkv, d, page, BF, codes, 3, prefixes=plen)
    cu = offsets(new)
    q = rnd(1, cu[-1], H, d).to(DEV)
    c.table[0, 2], c.table[1, 0], c.table[1, 4] = -1, c.cache[0].shape[0], 2 ** 31 - 1
    c.ptable[0, 1], c.ptable[0, 5] = -2 ** 31, c.cache[0].shape[0]
    gone = {0: [(32, 48)], 1: [(0, 16), (64, 80)]}
    for shared in (False, True):
        if not shared and not codes:
            continue
        out = torch.full_like(q, 7.0)
        if shared:
            prefix_call(c, q, out, plen, [0, 2], lens, cu)
        else:
            P.paged_attention_e4m3(q, *c.on(DEV), c.table.to(DEV), i32(lens), i32(cu), out=out)
        torch.cuda.synchronize()
        f = 90 if shared else 0
        for b in range(2):
            keep = torch.ones(f + lens[b], dtype=torch.bool)
            for x, y in gone[b]:
                keep[f + x:f + y] = False
            if shared:
                keep[16:32] = keep[80:90] = False
            K, V = (torch.cat([c.pkv[0][w], c.kv[b][w]], 1) if shared else c.kv[b][w] for w in range(2))
            for i in range(new[b]):
                p = f + lens[b] - new[b] + i
                rows = keep.clone()
                rows[p + 1:] = False
                x = out[cu[b] + i][None, :, None]
                if not rows.any():
                    assert bool((x == 0).all())
                    continue
                want, tol = attention(q[cu[b] + i][None, :, None].cpu(), K[None, :, rows], V[None, :, rows], lookahead=None)
                check(f"{shared} {b} {i}", x, want["o"], tol["o"])


def test_lengths_offsets_and_groups_out_of_range_are_clamped():
    lens, new, H, Hkv, d, page, plen = [40, 50], [2, 3], 2, 1, 64, 16, [30]
    c = Cache(lens, Hkv, d, page, BF, True, 4, prefixes=plen)
    for x in c.cache:
        x[:] = torch.where(x & 0x7f == 0x7f, torch.zeros_like(x), x)      # (slots of none are read below)
    for x in c.scales:
        x[:] = torch.where(x == 255, torch.full_like(x, 127), x)
    cu = offsets(new)
    q = rnd(1, cu[-1] + 2, H, d).to(DEV)
    wide, pwide = c.table.shape[1] * page, c.ptable.shape[1] * page
    big = 2 ** 31 - 1
    for ln in ([wide + 1000, -5], [big, -big]):
        out = torch.full_like(q, 7.0)
        P.paged_attention_e4m3(q, *c.on(DEV), c.table.to(DEV), i32(ln), i32(cu), out=out)
        assert bool((out[2:5] == 0).all()) and bool(torch.isfinite(out[:2].float()).all()) and bool((out[5:] == 7.0).all())
        k, v = (torch.full((7, Hkv, d), 9.0, dtype=BF, device=DEV) for _ in range(2))
        P.paged_read_e4m3(*c.on(DEV), c.table.to(DEV), i32(ln), i32(cu), 7, out=(k, v))
        assert bool((k[2:5] == 0).all()) and bool((v[5:] == 9.0).all()) and bool(torch.isfinite(k.float()).all())
        out = torch.full_like(q, 7.0)
        prefix_call(c, q, out, [pwide + 99], [0, 2], ln, cu)
        assert bool((out[2:5] == 0).all()) and bool(torch.isfinite(out.float()).all()) and bool((out[5:] == 7.0).all())
    caches = c.on(DEV)
    before = [x.clone() for x in caches]
    kv = rnd(2, cu[-1] + 2, Hkv, d).to(DEV)
    P.paged_append_e4m3(kv, kv, *caches, c.table.to(DEV), i32([-5, -big]), i32(cu))
    for x, y in zip(caches, before):
        same(x.view(torch.uint8), y.view(torch.uint8), "an append of no tokens")
    # offsets past the tokens: all of them are the first sequence's; groups past the sequences end with them
    one = Cache([60, 40], Hkv, d, page, BF, True, 5, prefixes=[33, 12])
    out = torch.full_like(q, 7.0)
    prefix_call(one, q, out, [33, 12], [-7, 1, big], [60, 40], [-9, 100000, 100000])
    torch.cuda.synchronize()
    check_prefix(out, q, one, [33, 12], [0, 1, 2], [60, 40], [0, 7, 7], {})
    out.fill_(7.0)
    prefix_call(one, q, out, [33, -12], [1, 1, 1], [60, 40], [0, 4, 7])      # groups of nothing
    torch.cuda.synchronize()
    check_prefix(out, q, one, [33, 0], [1, 1, 1], [60, 40], [0, 4, 7], {})
    prefix_call(one, q, out, [33, 12], [2, 1, 0], [60, 40], [7, 3, 0])       # falling offsets: nothing is out of range
    torch.cuda.synchronize()


# ---------------------------------------------------------------- sizes, layouts, streams

@pytest.mark.parametrize("B", [511, 512, 700])
def test_hundreds_of_sequences(B):
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 9, (B,), generator=g).tolist()
    new = [min(x, n) for x, n in zip(torch.randint(0, 3, (B,), generator=g).tolist(), lens)]
    plen = [20, 0, 35]
    seqs = [0, 100, 100, B - 1]
    for codes in (False, True):
        c = Cache(lens, 1, 64, 8, BF, codes, B, prefixes=plen)
        cu = offsets(new)
        q = rnd(3, cu[-1] + 1, 2, 64).to(DEV)
        for opt in ({}, dict(window=15, sinks=3)):
            out = torch.full_like(q, 7.0)
            prefix_call(c, q, out, plen, seqs, lens, cu, **opt)
            torch.cuda.synchronize()
            check_prefix(out, q, c, plen, seqs, lens, cu, opt, only=set(range(0, B, 17)) | {B - 1, B - 2, 99, 100})
        if codes:
            k, v = P.paged_read_e4m3(*c.on(DEV), c.table.to(DEV), i32(lens), i32(offsets(lens)), sum(lens))
            same(v, torch.cat([x[1].transpose(0, 1) for x in c.kv]))
            rows = rnd(5, cu[-1], 1, 64)
            caches = c.on(DEV)
            P.paged_append_e4m3(rows.to(DEV), rows.to(DEV), *caches, c.table.to(DEV), i32(lens), i32(cu))
            k, v = P.paged_read_e4m3(*caches, c.table.to(DEV), i32(lens), i32(cu), cu[-1])
            same(k, values(*quantise(rows)).to(BF))
            same(v, k)


@types
@pytest.mark.parametrize("d,Hkv", [(64, 2), (128, 3), (96, 1)])
def test_caches_of_other_layouts(d, Hkv, dtype):
    # heads before slots, a gap behind each vector, scales with pages last
    lens, new, H, page, plen = [70, 33], [3, 1], 2 * Hkv, 16, [40]
    c = Cache(lens, Hkv, d, page, dtype, True, 9, prefixes=plen)
    kc, vc, ks, vs = c.on(DEV)
    pages = kc.shape[0]
    cu = offsets(new)
    q = rnd(1, cu[-1], H, d, dtype=dtype).to(DEV)
    tables = (c.table.to(DEV), i32(lens), i32(cu))

    def laid(x):
        big = torch.full((pages, Hkv, page, d + 16), 0x7f, dtype=torch.uint8, device=DEV)
        y = big[..., :d].transpose(1, 2).view(torch.float8_e4m3fn)
        y.view(torch.uint8).copy_(x.view(torch.uint8))
        return y

    def laid_s(x):
        return x.permute(2, 1, 0).contiguous().permute(2, 1, 0)

    other = (laid(kc), laid(vc), laid_s(ks), laid_s(vs))
    assert other[0].stride() != kc.stride() and other[2].stride() != ks.stride()
    for new_ in (new, [60, 20]):
        cu = offsets(new_)
        q = rnd(1, cu[-1], H, d, dtype=dtype).to(DEV)
        tables = (c.table.to(DEV), i32(lens), i32(cu))
        same(P.paged_attention_e4m3(q, *other, *tables), P.paged_attention_e4m3(q, kc, vc, ks, vs, *tables))
        kw = lambda x: dict(k_scale=x[2], v_scale=x[3])
        pre = (c.ptable.to(DEV), i32(plen), i32([0, 2]))
        same(P.paged_prefix_attention(q, *other[:2], *pre, *tables, **kw(other)),
             P.paged_prefix_attention(q, kc, vc, *pre, *tables, **kw((kc, vc, ks, vs))))
        for x, y in zip(P.paged_read_e4m3(*other, *tables, cu[-1]), P.paged_read_e4m3(kc, vc, ks, vs, *tables, cu[-1])):
            same(x, y)
        kv = rnd(7, 2, cu[-1], Hkv, d, dtype=dtype).to(DEV)
        for to in (other, (kc, vc, ks, vs)):
            P.paged_append_e4m3(kv[0], kv[1], *to, *tables)
        for x, y in zip(other, (kc, vc, ks, vs)):
            same(x.view(torch.uint8) if x.dtype != torch.uint8 else x, y.view(torch.uint8) if y.dtype != torch.uint8 else y)


def test_cache_of_more_than_four_gigabytes():
    pages, page, Hkv, d = 80000, 64, 8, 128
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("needs 14 GB of GPU memory")
    kc, vc = (torch.zeros(pages, page, Hkv, d, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.full((pages, page, Hkv), 127, dtype=torch.uint8, device=DEV) for _ in range(2))
    table = i32([[pages - 1, pages - 2, 79000, 5]])
    K, V = rnd(1, 200, Hkv, d), rnd(2, 200, Hkv, d)
    ln, cu = i32([200]), i32([0, 200])
    P.paged_append_e4m3(K.to(DEV), V.to(DEV), kc, vc, ks, vs, table, ln, cu)
    k, v = P.paged_read_e4m3(kc, vc, ks, vs, table, ln, cu, 200)
    K, V = (values(*quantise(x)).to(BF) for x in (K, V))
    same(k, K)
    same(v, V)
    K, V = (x.transpose(0, 1)[None] for x in (K, V))
    for H, new in ((8, 1), (16, 1), (8, 150)):
        q = rnd(3, new, H, d).to(DEV)
        want, tol = attention(q.transpose(0, 1)[None].cpu(), K, V, q_start=200 - new, window=90, sinks=2)
        o = P.paged_attention_e4m3(q, kc, vc, ks, vs, table, ln, i32([0, new]), window=90, sinks=2)
        check(f"H {H} new {new}", o.transpose(0, 1)[None], want["o"], tol["o"])
        if new < 100:     # the first 100 as a prefix of another call: 64 + 36 on its second page
            o = P.paged_prefix_attention(q, kc, vc, table[:, :1].contiguous(), i32([64]), i32([0, 1]), table[:, 1:].contiguous(),
                                         i32([136]), i32([0, new]), k_scale=ks, v_scale=vs, window=90, sinks=2)
            check(f"prefix, H {H} new {new}", o.transpose(0, 1)[None], want["o"], tol["o"])


def serve(c, q, kv, plen, seqs, lens, cu, out):
    """Serving as it goes: new tokens into the cache, the attention of each over its own and behind the prefix, and the rows back."""
    caches = c["caches"]
    tables = (c["table"], i32(lens) if isinstance(lens, list) else lens, cu)
    P.paged_append_e4m3(kv[0], kv[1], *caches, *tables)
    P.paged_attention_e4m3(q, *caches, *tables, window=60, out=out[0])
    P.paged_prefix_attention(q, *caches[:2], c["ptable"], plen, seqs, *tables, k_scale=caches[2], v_scale=caches[3], sinks=2,
                             window=200, out=out[1])
    P.paged_read_e4m3(*caches, *tables, q.shape[0], out=out[2:])


def serving(seed=8, lens=(300, 90, 40), new=(1, 4, 1), plen=(700, 60), seqs=(0, 2, 3), H=4, Hkv=2, d=64):
    c = Cache(list(lens), Hkv, d, 16, BF, True, seed, prefixes=list(plen))
    n = sum(new)
    x = {"caches": c.on(DEV), "table": c.table.to(DEV), "ptable": c.ptable.to(DEV)}
    args = [x, rnd(seed, n, H, d).to(DEV), rnd(seed + 1, 2, n, Hkv, d).to(DEV), i32(list(plen)), i32(list(seqs)), i32(list(lens)),
            i32(offsets(new))]
    out = [torch.zeros(n, H, d, dtype=BF, device=DEV) for _ in range(2)] + [torch.zeros(n, Hkv, d, dtype=BF, device=DEV) for _ in range(2)]
    return c, args, out


def test_a_run_of_them_matches_the_formula():
    # decoding step by step: what is appended is what later tokens see
    c, args, out = serving(lens=(40, 41, 42), new=(1, 1, 1))
    K = [[x.clone() for x in kv] for kv in c.kv]
    lens = [40, 41, 42]
    for t in range(3):
        lens = [n + 1 for n in lens]
        args[1], args[2], args[5] = rnd(50 + t, 3, 4, 64).to(DEV), rnd(60 + t, 2, 3, 2, 64).to(DEV), i32(lens)
        serve(*args, out)
        torch.cuda.synchronize()
        held = [values(*quantise(args[2][w])).to(BF) for w in range(2)]
        for w in range(2):
            same(out[2 + w], held[w])
            for b in range(3):
                K[b][w] = torch.cat([K[b][w], held[w][b][:, None]], 1)
        for b in range(3):
            q = args[1][b][None, :, None].cpu()
            want, tol = attention(q, K[b][0][None], K[b][1][None], window=60)
            check(f"own {t} {b}", out[0][b][None, :, None], want["o"], tol["o"])
            g = 0 if b < 2 else 1
            k, v = (torch.cat([c.pkv[g][w], K[b][w]], 1)[None] for w in range(2))
            want, tol = attention(q, k, v, window=200, sinks=2)
            check(f"behind the prefix {t} {b}", out[1][b][None, :, None], want["o"], tol["o"])


def test_captured_and_replayed():
    _, args, out = serving()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        serve(*args, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        serve(*args, out)
    second = torch.cuda.CUDAGraph()          # two graphs of the same calls, replayed in turn
    with torch.cuda.graph(second):
        serve(*args, out)
    eager = [torch.zeros_like(x) for x in out]
    for i in range(4):
        args[1].copy_(rnd(30 + i, *args[1].shape))
        args[2].copy_(rnd(40 + i, *args[2].shape))
        args[5].copy_(i32([[300, 90, 40], [200, 4, 41], [320, 12, 1], [17, 90, 40]][i]))
        (graph if i % 2 else second).replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        serve(*args, eager)
        torch.cuda.synchronize()
        for a, b in zip(got, eager):
            same(a, b, i)


def test_work_on_a_given_stream_beside_the_current_one():
    _, (c, q, kv, plen, seqs, lens, cu), out = serving()
    serve(c, q, kv, plen, seqs, lens, cu, out)
    want = [x.clone() for x in out]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    junk = []
    for _ in range(4):
        s = side.cuda_stream
        big = torch.full((1 << 22,), 3.0, dtype=F32, device=DEV)
        del big                                              # its memory is free for the current stream only
        tables = (c["table"], lens, cu)
        o = P.paged_attention_e4m3(q, *c["caches"], *tables, window=60, stream=s)
        p = P.paged_prefix_attention(q, *c["caches"][:2], c["ptable"], plen, seqs, *tables, k_scale=c["caches"][2],
                                     v_scale=c["caches"][3], sinks=2, window=200, stream=s)
        junk.append(torch.full((1 << 20,), float("nan"), dtype=F32, device=DEV))
        k, v = P.paged_read_e4m3(*c["caches"], *tables, q.shape[0], stream=s)
        P.paged_append_e4m3(kv[0], kv[1], *c["caches"], *tables, stream=s)
        side.synchronize()
        for a, b in zip((o, p, k, v), want):
            same(a, b)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,codes", [(BF, True), (F32, True), (BF, False)])
@pytest.mark.parametrize("d,Hkv,G,n", [(128, 2, 8, 1), (64, 2, 4, 3), (64, 1, 6, 5), (128, 4, 4, 2), (256, 1, 3, 1)])
def test_few_rows_are_rounded_once(d, Hkv, G, n, dtype, codes):
    # up to 32 rows of a key head: beside the output's own half step there is what two or
    # three bf16 parts leave of each weight, and of a score, and the fp32 arithmetic
    lens, plen = [333, 90], [140]
    H = Hkv * G
    c = Cache(lens, Hkv, d, 16, dtype, codes, 21, prefixes=plen)
    cu = offsets([n, n])
    q = rnd(2, cu[-1], H, d, dtype=dtype).to(DEV)
    left = 2.0 ** -15 if dtype is BF else 2.0 ** -22       # of a weight: two parts, or three (and a score's)
    outs = [("prefix", 140, prefix_call(c, q, torch.full_like(q, 7.0), plen, [0, 2], lens, cu))]
    if 2 * n * G > 32:
        outs = []                                         # (the group's rows go together)
    if codes:
        outs.append(("own", 0, P.paged_attention_e4m3(q, *c.on(DEV), c.table.to(DEV), i32(lens), i32(cu))))
    for name, f, o in outs:
        for b, m in enumerate(lens):
            k, v = (torch.cat([c.pkv[0][w], c.kv[b][w]], 1) if f else c.kv[b][w] for w in range(2))
            see = visible(n, f + m, f + m, f + m - n, None, 0, 0)
            for h in range(H):
                x = q[cu[b]:cu[b + 1], h].cpu()
                r = head(x, k[h // G], v[h // G], see, d ** -0.5)
                mag = (x.double().abs() @ k[h // G].double().abs().t()).amax(1, keepdim=True) * d ** -0.5
                e = r["e"] + left + (left * mag if dtype is F32 else 0.0)
                check(f"{name} {b} {h}", o[cu[b]:cu[b + 1], h], r["o"],
                      r["o_mag"] * (e + (f + m) * 2.0 ** -24) * 1.01 + r["o"].abs() * HALF[dtype])


@types
def test_scores_of_large_magnitude(dtype):
    lens, plen = [150, 40], [130]
    for codes in (False, True):
        c = Cache(lens, 2, 64, 16, dtype, codes, 31, prefixes=plen, scale=30.0)
        cu = offsets([2, 40])
        q = rnd(3, cu[-1], 4, 64, dtype=dtype, scale=30.0).to(DEV)
        out = torch.full_like(q, 7.0)
        prefix_call(c, q, out, plen, [0, 2], lens, cu)
        check_prefix(out, q, c, plen, [0, 2], lens, cu, {})


def test_one_prefix_is_a_table_that_begins_with_its_pages():
    # 64 keys on 4 pages: the same keys as one table of pages, over either kind of cache
    lens, new, H, Hkv, d, page, plen = [37, 90, 5], [1, 2, 1], 8, 2, 128, 16, [64]
    for codes in (False, True):
        c = Cache(lens, Hkv, d, page, BF, codes, 13, prefixes=plen)
        cu = offsets(new)
        q = rnd(4, cu[-1], H, d).to(DEV)
        whole = torch.cat([c.ptable[0, :4].expand(3, 4), c.table], 1).contiguous().to(DEV)
        full = i32([n + 64 for n in lens])
        a = prefix_call(c, q, torch.zeros_like(q), plen, [0, 3], lens, cu, window=90, sinks=3)
        if codes:
            b = P.paged_attention_e4m3(q, *c.on(DEV), whole, full, i32(cu), window=90, sinks=3)
        else:
            b = P.paged_attention(q, *c.on(DEV), whole, full, i32(cu), window=90, sinks=3)
        # each is within its half step of the formula and what the weights' rounding leaves (2^-8 of the magnitudes)
        assert float((a.double() - b.double()).norm() / b.double().norm()) < 2 * (2.0 ** -9 + 2.0 ** -9)


def test_outputs_and_workspaces_given_and_bindings_refuse():
    c, (x, q, kv, plen, seqs, lens, cu), _ = serving()
    t = (x["table"], lens, cu)
    caches = x["caches"]
    attend = lambda **k: P.paged_attention_e4m3(q, *caches, *t, **k)
    shared = lambda **k: P.paged_prefix_attention(q, *caches[:2], x["ptable"], plen, seqs, *t,
                                                  **dict(dict(k_scale=caches[2], v_scale=caches[3]), **k))
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    for f in (attend, shared):
        want = f()
        out = spread(q)
        same(f(out=out, workspace=ws), want)
    with pytest.raises(P.LactError):
        shared(workspace=ws[:64])
    kc, vc, ks, vs = caches
    n = q.shape[0]
    bad = [lambda: P.paged_attention_e4m3(q, kc.view(torch.uint8), vc, ks, vs, *t),
           lambda: P.paged_attention_e4m3(q, kc, vc, ks.float(), vs, *t), lambda: P.paged_attention_e4m3(q, kc, vc, ks[:-1], vs, *t),
           lambda: P.paged_attention_e4m3(q, kc, vc, ks, None, *t), lambda: P.paged_attention_e4m3(q.half(), *caches, *t),
           lambda: P.paged_attention_e4m3(q[..., :48], *caches, *t), lambda: P.paged_attention_e4m3(q[0], *caches, *t),
           lambda: P.paged_attention_e4m3(q[:, :3], *caches, *t), lambda: P.paged_attention_e4m3(q, kc[..., :24], vc[..., :24], ks, vs, *t),
           lambda: P.paged_attention_e4m3(q, kc, vc, ks, vs.transpose(1, 2), *t), lambda: attend(scale=-1.0),
           lambda: attend(window=-2), lambda: attend(out=q[:1].expand_as(q)), lambda: shared(v_scale=None),
           lambda: shared(k_scale=None, v_scale=None), lambda: P.paged_attention_e4m3(q, *caches, x["table"].long(), lens, cu),
           lambda: P.paged_prefix_attention(q, kc, vc, x["ptable"][:0], plen[:0], seqs[:1], *t, k_scale=ks, v_scale=vs),
           lambda: P.paged_prefix_attention(q, kc, vc, x["ptable"], plen[:1], seqs, *t, k_scale=ks, v_scale=vs),
           lambda: P.paged_prefix_attention(q, kc, vc, x["ptable"], plen, seqs[:2], *t, k_scale=ks, v_scale=vs),
           lambda: P.paged_prefix_attention(q, kc, vc, x["ptable"][0], plen, seqs, *t, k_scale=ks, v_scale=vs),
           lambda: P.paged_prefix_attention(q, kc, vc, x["ptable"], None, seqs, *t, k_scale=ks, v_scale=vs),
           lambda: P.paged_append_e4m3(kv[0], kv[1].float(), *caches, *t), lambda: P.paged_append_e4m3(kv[0], kv[1, :2], *caches, *t),
           lambda: P.paged_append_e4m3(kv[0], kv[1], kc, vc, ks[:1].expand_as(ks), vs, *t),
           lambda: P.paged_append_e4m3(kv[0].half(), kv[1].half(), *caches, *t),
           lambda: P.paged_read_e4m3(*caches, *t, n, dtype=torch.float16), lambda: P.paged_read_e4m3(*caches, *t, -1),
           lambda: P.paged_read_e4m3(*caches, *t, n, dtype=F32, out=(kv[0], kv[1])),
           lambda: P.paged_read_e4m3(kc.cpu(), vc, ks, vs, *t, n)]
    for i, call in enumerate(bad):
        with pytest.raises(P.LactError):
            call()
            pytest.fail(f"call {i} was taken")
    # nothing to do
    none = torch.empty(0, 4, 64, dtype=BF, device=DEV)
    assert P.paged_attention_e4m3(none, *caches, *t).shape == none.shape
    assert P.paged_prefix_attention(none, kc, vc, x["ptable"], plen, seqs, *t, k_scale=ks, v_scale=vs).shape == none.shape
    assert P.paged_read_e4m3(*caches, *t, 0)[0].shape == (0, 2, 64)
    P.paged_append_e4m3(kv[0][:0], kv[1][:0], *caches, *t)
    # a cache of no pages, tables of no width: nothing is seen, nothing written
    kc, vc, ks, vs = (y[:0] for y in caches)
    for tab in (x["table"], x["table"][:, :0].contiguous()):
        assert bool((P.paged_attention_e4m3(q, kc, vc, ks, vs, tab, lens, cu) == 0).all())
        assert bool((P.paged_prefix_attention(q, kc, vc, x["ptable"], plen, seqs, tab, lens, cu, k_scale=ks, v_scale=vs) == 0).all())
        assert bool((P.paged_read_e4m3(kc, vc, ks, vs, tab, lens, cu, n)[0] == 0).all())
        P.paged_append_e4m3(kv[0], kv[1], kc, vc, ks, vs, tab, lens, cu)
    # a prefix of no pages
    same(P.paged_prefix_attention(q, *caches[:2], x["ptable"][:, :0].contiguous(), plen, seqs, *t, k_scale=caches[2], v_scale=caches[3]),
         P.paged_prefix_attention(q, *caches[:2], x["ptable"], plen * 0, seqs, *t, k_scale=caches[2], v_scale=caches[3]))


@types
@pytest.mark.parametrize("prefix", [False, True], ids=["own", "prefix"])
@pytest.mark.parametrize("new,Hkv,d", [([1, 1], 2, 64), ([1, 1], 1, 128), ([5, 9], 1, 64), ([9, 7], 2, 256), ([60, 30], 2, 128)])
def test_scores_of_zero_at_any_scale(new, Hkv, d, prefix, dtype):
    # keys of the largest magnitudes that a cache holds, times a scale over 355: past fp32 before a score is
    lens, plen, H = [100, 60], [40], 2 * Hkv
    c = Cache(lens, Hkv, d, 16, dtype, True, 51, prefixes=plen)
    c.scales[0] = torch.where(c.scales[0] == 255, c.scales[0], torch.full_like(c.scales[0], 246))
    cu = offsets(new)
    q = torch.zeros(cu[-1], H, d, dtype=dtype, device=DEV)
    print(f"[gpu] scores of zero {new} {Hkv} {d} {prefix} {dtype}", flush=True)
    for scale in (1.0, 1e3, 1e12):
        if prefix:
            o = prefix_call(c, q, torch.full_like(q, 7.0), plen, [0, 2], lens, cu, scale=scale)
        else:
            o = P.paged_attention_e4m3(q, *c.on(DEV), c.table.to(DEV), i32(lens), i32(cu), scale=scale)
        for b in range(2):
            k, v = (torch.cat([c.pkv[0][w], c.kv[b][w]], 1) if prefix else c.kv[b][w] for w in range(2))
            rows = slice(cu[b], cu[b + 1])
            want, tol = attention(q[rows].transpose(0, 1)[None].cpu(), torch.zeros_like(k)[None], v[None],
                                  q_start=k.shape[1] - new[b])
            check(f"{scale} {b}", o[rows].transpose(0, 1)[None], want["o"], tol["o"])


# prefixes, sequences of each, lens, new, H, Hkv, d: up to 32 rows of a key head in a sequence, and as many
# in a group as come together
FEW = [
    ([140, 90], [1, 1], [333, 90], [5, 5], 6, 1, 64),            # sequences of more than 16 rows, in groups of their own
    ([140, 90], [1, 1], [33, 90], [3, 4], 6, 2, 128),
    ([300], [2], [333, 90], [5, 5], 6, 1, 64),                   # more than 32 rows a group
    ([300], [2], [20, 90], [5, 5], 6, 1, 256),
    ([1700], [40], list(range(1, 41)), [1] * 40, 8, 2, 128),     # a decoding batch, the prefix in parts
    ([700, 40], [30, 10], [5] * 40, [1] * 40, 4, 2, 64),
    ([400], [20], [9] * 20, [1] * 20, 8, 1, 256),
    ([200], [12], [6] * 12, [3] * 12, 4, 2, 80),
]


@pytest.mark.parametrize("dtype,codes", [(BF, True), (F32, True), (BF, False)], ids=["bf16-e4m3", "fp32-e4m3", "bf16"])
@pytest.mark.parametrize("i", range(len(FEW)))
def test_few_rows_behind_a_prefix_are_rounded_once(i, dtype, codes):
    # as test_few_rows_are_rounded_once(): two or three parts of a weight, however many rows share the prefix
    plen, counts, lens, new, H, Hkv, d = FEW[i]
    G = H // Hkv
    assert sum(new) * G <= 32 * len(lens)
    c = Cache(lens, Hkv, d, 16, dtype, codes, 40 + i, prefixes=plen)
    cu, seqs = offsets(new), offsets(counts)
    q = rnd(2, cu[-1], H, d, dtype=dtype).to(DEV)
    left = 2.0 ** -15 if dtype is BF else 2.0 ** -22
    print(f"[gpu] few rows behind a prefix {FEW[i]} {dtype} {codes}", flush=True)
    o = prefix_call(c, q, torch.full_like(q, 7.0), plen, seqs, lens, cu).cpu()
    for g, f in enumerate(plen):
        for b in range(seqs[g], seqs[g + 1]):
            n, m = new[b], lens[b]
            k, v = (torch.cat([c.pkv[g][w], c.kv[b][w]], 1) for w in range(2))
            see = visible(n, f + m, f + m, f + m - n, None, 0, 0)
            for h in range(H):
                x = q[cu[b]:cu[b + 1], h].cpu()
                r = head(x, k[h // G], v[h // G], see, d ** -0.5)
                mag = (x.double().abs() @ k[h // G].double().abs().t()).amax(1, keepdim=True) * d ** -0.5
                e = r["e"] + left + (left * mag if dtype is F32 else 0.0)
                check(f"{b} {h}", o[cu[b]:cu[b + 1], h], r["o"],
                      r["o_mag"] * (e + (f + m) * 2.0 ** -24) * 1.01 + r["o"].abs() * HALF[dtype])


@types
@pytest.mark.parametrize("value", [math.inf, -math.inf])
@pytest.mark.parametrize("i", range(len(SPOILT)))
def test_infinities_in_pages_behind_a_prefix_stay_what_they_are(i, value, dtype):
    # as test_nan_in_pages_..., where a part of a weight that became zero, or a sign that was lost, would show
    lens, new, H, Hkv, d, page, opt, b, where = SPOILT[i]
    f, plen, seqs = 75, [75], [0, len(lens)]
    c = Cache(lens, Hkv, d, page, dtype, False, 300 + i, prefixes=plen)
    cu = offsets(new)
    q = rnd(i, cu[-1], H, d, dtype=dtype).to(DEV)
    print(f"[gpu] infinities behind a prefix {SPOILT[i]} {value} {dtype}", flush=True)

    def call():
        return prefix_call(c, q, torch.full_like(q, 7.0), plen, seqs, lens, cu, **opt)

    base = call()
    assert bool(torch.isfinite(base.float()).all())
    cols = torch.arange(d) % 3 == 1
    group = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(new))
    pos = torch.cat([torch.arange(n - m, n) for n, m in zip(lens, new)])
    seen = 0
    for own_key, at in [(True, x) for x in where] + [(False, x) for x in (0, 31, 64, 74)]:
        v, table = c.cache[1], c.table[b] if own_key else c.ptable[0]
        saved = v.clone()
        v[table[at // page], at % page][..., cols] = value
        p, j = f + pos, f + at if own_key else at
        see = j <= p
        if "window" in opt:
            see &= (j > p - opt["window"]) | (j < opt.get("sinks", 0))
        if own_key:
            see &= group == b
        got = call()
        c.cache[1] = saved
        seen += int(see.sum())
        see = see.to(DEV)
        same(got[~see], base[~see], ("rows that do not see it", own_key, at))
        same(got[see].cpu()[..., ~cols], base[see].cpu()[..., ~cols], ("other columns", own_key, at))
        assert bool((got[see].cpu()[..., cols] == value).all()), (own_key, at)
    assert seen
