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
        x[i] = torch.tensor([(2 * k + 17) / 32 * (1 + (0, 2.0 ** -7, -2.0 ** -7)[i % 3]) for k in range(d)]) * 0.25
        x[i, 0] = 448.0 if i % 2 else 1.75
    x[30] = torch.tensor([(2 * k + 1) * 2.0 ** -10 for k in range(d)])      # ties of numbers below the least normal one
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
            want = torch.cat([torch.zeros(4, Hkv, d), c.kv[b][w].transpose(0, 1).float()])
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
