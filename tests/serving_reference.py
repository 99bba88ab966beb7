"""Plain 64-bit forms of the cache in 8 bits, on the CPU, and caches for the
tests of the entry points that read them."""
import math

import torch

CODES = torch.tensor([math.nan if c & 127 == 127 else (-1.0 if c & 128 else 1.0) *
                      ((c & 7) * 2.0 ** -9 if c >> 3 & 15 == 0 else (8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10))
                      for c in range(256)], dtype=torch.float64)
POSITIVE = CODES[:127]          # ascending: 0 to 448


def values(codes, scales):
    """What codes [.., d] (uint8) with scales [..] (uint8) stand for, in 64 bits."""
    return CODES[codes.long()] * torch.pow(torch.tensor(2.0, dtype=torch.float64), scales.double() - 127)[..., None]


def nearest(x):
    """The code of the e4m3 number nearest to each |x| <= 448 (64 bits), ties to the even one, sign apart."""
    a = x.abs()
    hi = torch.searchsorted(POSITIVE, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = a - POSITIVE[lo], POSITIVE[hi] - a
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return torch.where(up, hi, lo)


def quantise(x):
    """Codes and scales of vectors [.., d] of any type, by the definition."""
    x = x.detach().cpu().double()
    fine = torch.isfinite(x)
    a = torch.where(fine, x.abs(), torch.zeros_like(x)).amax(-1)
    e = torch.full_like(a, -117)
    for k in range(-117, 120):
        e = torch.where(448 * 2.0 ** k < a, torch.full_like(e, min(k + 1, 119)), e)
    y = torch.where(fine, x, torch.zeros_like(x)) / torch.pow(torch.tensor(2.0, dtype=torch.float64), e)[..., None]
    c = nearest(y.clamp(-448, 448)) + 128 * torch.signbit(x).long()
    c = torch.where(fine, c, torch.full_like(c, 127))
    return c.to(torch.uint8), (e + 127).to(torch.uint8)


class Cache:
    """Pages of keys and values of sequences (and of prefixes): `k`, `v` lists of
    [Hkv, n, d] tensors, in pages that are shuffled; slots of none hold NaN.
    codes: e4m3 numbers, and then `k`, `v` are what they stand for."""

    def __init__(self, lens, Hkv, d, page, dtype, codes, seed, prefixes=(), extra=2, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.page, self.codes, self.dtype, self.d, self.Hkv = page, codes, dtype, d, Hkv
        width, pwidth = (max([-(-x // page) for x in n] + [0]) + 1 for n in (lens, prefixes))
        B, P = len(lens), len(prefixes)
        pages = B * width + P * pwidth + extra
        perm = torch.randperm(pages, generator=g)
        self.table, self.ptable = perm[:B * width].view(B, width).int(), perm[B * width:B * width + P * pwidth].view(P, pwidth).int()
        shape = (pages, page, Hkv, d)
        if codes:
            self.cache = [torch.full(shape, 0x7f, dtype=torch.uint8) for _ in range(2)]
            self.scales = [torch.full(shape[:3], 255, dtype=torch.uint8) for _ in range(2)]
        else:
            self.cache, self.scales = [torch.full(shape, math.nan, dtype=dtype) for _ in range(2)], None
        self.kv, self.pkv = [], []
        for ns, table, out in ((lens, self.table, self.kv), (prefixes, self.ptable, self.pkv)):
            for b, n in enumerate(ns):
                both = []
                for w in range(2):
                    x = torch.randn(max(n, 0), Hkv, d, generator=g, dtype=torch.float32)
                    x = x * torch.exp(0.3 * torch.randn(max(n, 0), Hkv, 1, generator=g, dtype=torch.float32))
                    x = (x * scale).to(dtype)
                    j = torch.arange(max(n, 0))
                    at = (table[b, j // page].long(), j % page)
                    if codes:
                        c, s = quantise(x)
                        self.cache[w][at], self.scales[w][at] = c, s
                        x = values(c, s).to(dtype)
                    else:
                        self.cache[w][at] = x
                    both.append(x.transpose(0, 1))
                out.append(both)

    def on(self, device):
        """(caches and, with codes, scales) on a device, as the entry points take them."""
        c = [x.to(device) for x in self.cache]
        if not self.codes:
            return c
        return [x.view(torch.float8_e4m3fn) for x in c] + [x.to(device) for x in self.scales]
