"""The cache in 8 bits and the attention behind shared prefixes without a GPU:
refusals before any HIP call, workspace sizes, and the plain forms against
other ways to the same."""
import ctypes
import math

import pytest
import torch

import paper_2505_23884_amd as P
from paper_2505_23884_amd.binding import LactPagedDesc, LactPrefix, LactView
from serving_reference import CODES, Cache, nearest, quantise, values

EINVAL, EALIGN, EWORKSPACE, EUNSUPPORTED = -1, -2, -3, -4
PAGED = dict(B=3, H=4, Hkv=2, d=128, n_new=5, pages=10, page=16, max_pages=4, window=-1, sinks=0, scale=0.1, io_dtype=0)


def view(at=0x10000, batch=1 << 16, head=1 << 13, token=128):
    return LactView(at, batch, head, token)


def small(at=0x10001, batch=32, head=16, token=1):      # scales: any alignment
    return LactView(at, batch, head, token)


def call(which, desc=None, ws=None, **a):
    d = LactPagedDesc(**dict(PAGED, **(desc or {})))
    g = lambda n, v: a.get(n, v)
    L = P.lib()
    tail = [g("table", 0x1000), g("lens", 0x1000), g("cu_new", 0x1000)]
    cache = [g("k_cache", view()), g("v_cache", view()), g("k_scale", small()), g("v_scale", small())]
    if which == "append":
        return L.lact_paged_append_e4m3(d, g("k", view()), g("v", view()), *cache, *tail, None)
    if which == "read":
        return L.lact_paged_read_e4m3(d, *cache, *tail, g("k", view()), g("v", view()), None)
    if which == "attend":
        need = L.lact_paged_attention_e4m3_workspace_bytes(d, None)
        return L.lact_paged_attention_e4m3(d, g("q", view()), *cache, *tail, g("o", view()), g("workspace", 0x10000),
                                           need if ws is None else ws, None)
    p = g("prefix", prefix())
    if which == "plain":
        cache[2] = cache[3] = None
    need = L.lact_paged_prefix_attention_workspace_bytes(d, p, int(which == "shared"), None)
    return L.lact_paged_prefix_attention(d, p, g("q", view()), *cache, *tail, g("o", view()), g("workspace", 0x10000),
                                         need if ws is None else ws, None)


def prefix(groups=2, max_pages=3, table=0x1000, lens=0x1000, cu_seq=0x1000):
    return LactPrefix(groups, max_pages, table, lens, cu_seq)


ALL = ["append", "read", "attend", "shared", "plain"]


@pytest.mark.parametrize("which", ALL)
@pytest.mark.parametrize("field,value,code", [
    ("B", 0, EINVAL), ("Hkv", 0, EINVAL), ("d", 12, EUNSUPPORTED), ("d", 264, EUNSUPPORTED), ("io_dtype", 2, EINVAL),
    ("n_new", -1, EINVAL), ("pages", -1, EINVAL), ("page", 0, EINVAL), ("max_pages", -1, EINVAL),
    ("max_pages", 1 << 26, EUNSUPPORTED), ("n_new", 1 << 30, EUNSUPPORTED), ("n_new", (1 << 26) + 1, EUNSUPPORTED)])
def test_descriptor_is_refused(field, value, code, which):
    assert call(which, {field: value}, ws=1 << 50) == code


@pytest.mark.parametrize("which", ALL[:4])
def test_vectors_of_e4m3_numbers_are_whole_chunks(which):
    assert call(which, {"d": 72}, ws=1 << 50, k=view(token=144), v=view(token=144), k_cache=view(token=144),
                v_cache=view(token=144)) == EUNSUPPORTED


@pytest.mark.parametrize("which", ALL[2:])
def test_attention_fields_are_refused(which):
    for f, v in (("window", -2), ("sinks", -1), ("scale", 0.0), ("scale", math.nan), ("scale", math.inf), ("H", 3)):
        assert call(which, {f: v}) == EINVAL
    for name in ("q", "o"):
        assert call(which, **{name: view(0)}) == EINVAL
        assert call(which, **{name: None}) == EINVAL
        assert call(which, **{name: view(0x10008)}) == EALIGN
    assert call(which, o=view(token=0)) == EINVAL
    long = {"max_pages": 4096}
    assert call(which, long, ws=16) == EWORKSPACE
    assert call(which, long, workspace=None) == EWORKSPACE
    assert call(which, long, workspace=0x10010) == EALIGN
    assert call(which, {"n_new": 0}, q=view(0), o=view(0)) == 0


@pytest.mark.parametrize("which", ALL)
def test_caches_and_tables_are_refused(which):
    for name in ("k_cache", "v_cache"):
        assert call(which, **{name: None}) == EINVAL
        assert call(which, **{name: view(0)}) == EINVAL
        assert call(which, **{name: view(0x10004)}) == EALIGN
        assert call(which, **{name: view(head=(1 << 13) + 4)}) in (EALIGN, EINVAL)
        assert call(which, **{name: view(head=1 << 12)}) == EINVAL          # another layout than the other's
    if which != "plain":
        for name in ("k_scale", "v_scale"):
            assert call(which, **{name: None}) == EINVAL
            assert call(which, **{name: small(0)}) == EINVAL
            assert call(which, **{name: small(batch=64)}) == EINVAL
            assert call(which, **{name: small(token=-1)}) == EINVAL
    for name in ("table", "lens", "cu_new"):
        assert call(which, **{name: None}) == EINVAL
        assert call(which, **{name: 0x1002}) == EALIGN


def test_append_and_read_arguments_are_refused():
    for which in ("append", "read"):
        for name in ("k", "v"):
            assert call(which, **{name: view(0)}) == EINVAL
            assert call(which, **{name: view(0x10008)}) == EALIGN
        assert call(which, {"n_new": 0}, k=view(0), v=view(0)) == 0
        assert call(which, {"n_new": (1 << 25) + 1}) == EUNSUPPORTED          # times 2 heads of 128
    over = dict(batch=0), dict(token=64), dict(head=0)
    for bad in over:                                                          # written: vectors must not overlap
        assert call("append", k_cache=view(**bad), v_cache=view(**bad)) == EINVAL
    for bad in (dict(batch=0), dict(batch=16), dict(head=0), dict(token=0)):
        assert call("append", k_scale=small(**bad), v_scale=small(**bad)) == EINVAL
    assert call("read", k=view(head=64)) == EINVAL


@pytest.mark.parametrize("which", ["shared", "plain"])
def test_prefixes_are_refused(which):
    assert call(which, prefix=None, ws=1 << 40) == EINVAL
    assert call(which, prefix=prefix(groups=0), ws=1 << 40) == EINVAL
    assert call(which, prefix=prefix(max_pages=-1), ws=1 << 40) == EINVAL
    assert call(which, prefix=prefix(groups=1 << 20), ws=1 << 50) == EUNSUPPORTED       # times 2 heads
    assert call(which, prefix=prefix(max_pages=(1 << 25) - 3), ws=1 << 50) == EUNSUPPORTED     # 4 pages of the sequence beside it
    for name in ("table", "lens", "cu_seq"):
        assert call(which, prefix=prefix(**{name: None})) == EINVAL
        assert call(which, prefix=prefix(**{name: 0x1002})) == EALIGN


def test_workspaces():
    L = P.lib()
    f = lambda **k: L.lact_paged_attention_e4m3_workspace_bytes(LactPagedDesc(**dict(PAGED, **k)), None)
    assert f(n_new=0) == 0 and f(max_pages=0) == 0
    assert 0 < f(max_pages=2048) <= 64 * 5 * 4 * 130 * 4 + 256
    err = ctypes.c_int(0)
    assert L.lact_paged_attention_e4m3_workspace_bytes(LactPagedDesc(**dict(PAGED, d=24)), ctypes.byref(err)) == 0
    assert err.value == EUNSUPPORTED
    g = lambda p, **k: L.lact_paged_prefix_attention_workspace_bytes(LactPagedDesc(**dict(PAGED, **k)), p, 1, ctypes.byref(err))
    assert g(prefix()) >= 2 * 5 * 4 * 130 * 4 and err.value == 0               # a part of each at least
    assert g(None) == 0 and err.value == EINVAL
    # the parts stay few for the largest calls, whose launches hold fewer than 2^32 threads
    for T, B in ((1 << 24, 1), (1 << 22, 1 << 18)):
        n = g(prefix(groups=1, max_pages=1 << 20), n_new=T, B=B, max_pages=1 << 20)
        assert 0 < n <= (T * 4 * 130 * 4) * 8


def test_tensors_of_the_host_are_refused():
    f8 = torch.float8_e4m3fn
    t = torch.zeros(8, 2, 64, dtype=torch.bfloat16)
    c, s = torch.zeros(4, 16, 2, 64, dtype=torch.uint8).view(f8), torch.zeros(4, 16, 2, dtype=torch.uint8)
    i = torch.zeros(1, 2, dtype=torch.int32)
    lens, cu = i[0, :1], i[0]
    for f in (lambda: P.paged_append_e4m3(t, t, c, c, s, s, i, lens, cu), lambda: P.paged_read_e4m3(c, c, s, s, i, lens, cu, 3),
              lambda: P.paged_attention_e4m3(t, c, c, s, s, i, lens, cu),
              lambda: P.paged_prefix_attention(t, c, c, i, lens, cu, i, lens, cu, k_scale=s, v_scale=s),
              lambda: P.paged_prefix_attention(t, t[None], t[None], i, lens, cu, i, lens, cu)):
        with pytest.raises(P.LactError):
            f()


def test_codes_are_the_type_that_torch_has():
    c = torch.arange(256, dtype=torch.uint8)
    want = c.view(torch.float8_e4m3fn).double()
    assert torch.equal(torch.isnan(want), torch.isnan(CODES)) and torch.equal(torch.nan_to_num(want), torch.nan_to_num(CODES))


def test_rounding_is_that_of_the_type():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(4000, generator=g, dtype=torch.float32) * 2.0 ** torch.randint(-12, 7, (4000,), generator=g).float()
    x = torch.cat([x, torch.tensor([448.0, 0.0, 2.0 ** -10, 3 * 2.0 ** -10, 17 / 16, 19 / 16, 2.0 ** -9 * 2.5], dtype=torch.float32)]).clamp(-448, 448)
    code = nearest(x.double()) + 128 * torch.signbit(x).long()
    assert torch.equal(code.to(torch.uint8), x.to(torch.float8_e4m3fn).view(torch.uint8))


def test_a_scale_is_the_smallest_that_takes_the_largest_element():
    g = torch.Generator().manual_seed(2)
    x = torch.randn(300, 32, generator=g, dtype=torch.float32) * 2.0 ** torch.randint(-140, 127, (300, 1), generator=g).float()
    x[:5] = 0
    c, s = quantise(x)
    a = x.double().abs().amax(-1)
    p = 2.0 ** (s.double() - 127)
    top = s.int() == 246
    assert bool((s >= 10).all()) and bool((s <= 246).all()) and bool((s[:5] == 10).all())
    assert bool(((a <= 448 * p) | top).all()) and bool(((a > 448 * p / 2) | (s == 10)).all())
    y = values(c, s)
    err = (y - x.double()).abs()
    # half a step: 2^-4 of the number, or 2^-10 of the scale below the normal ones; magnitudes over 448 2^119 become that
    assert bool((err <= torch.maximum(x.double().abs() * 2.0 ** -4, p[:, None] * 2.0 ** -10))[~top].all())


def test_prefix_and_own_keys_add_up_to_one_sequence():
    # the parts that the operator joins, in 64 bits: maxima, sums and outputs over two sets of keys
    g = torch.Generator().manual_seed(3)
    s, v = torch.randn(5, 40, generator=g, dtype=torch.float64) * 3, torch.randn(40, 8, generator=g, dtype=torch.float64)
    want = torch.softmax(s, 1) @ v
    parts = []
    for a, b in ((0, 25), (25, 40)):
        m = s[:, a:b].amax(1, keepdim=True)
        p = torch.exp(s[:, a:b] - m)
        parts.append((m, p.sum(1, keepdim=True), p @ v[a:b]))
    m = torch.maximum(parts[0][0], parts[1][0])
    o = sum(torch.exp(x[0] - m) * x[2] for x in parts) / sum(torch.exp(x[0] - m) * x[1] for x in parts)
    assert torch.allclose(o, want, rtol=0, atol=1e-14)


def test_caches_of_the_tests_hold_what_they_say():
    c = Cache([5, 0, 20], 2, 16, 4, torch.bfloat16, True, 7, prefixes=[9])
    for b, n in enumerate((5, 0, 20)):
        for p in range(n):
            pg = c.table[b, p // 4]
            got = values(c.cache[1][pg, p % 4], c.scales[1][pg, p % 4])
            assert torch.equal(got.to(torch.bfloat16), c.kv[b][1][:, p])


# io_dtype, whether the cache is one of e4m3 numbers, heads, new tokens, sequences, groups: calls of a launch that holds
# fewer than 2^24 workgroups of 256, and of one that does not
@pytest.mark.parametrize("io_dtype,which,H,Hkv,d,n_new,B,groups,fits", [
    (1, "shared", 4, 2, 32, 1 << 26, 1, 1, False),            # fp32 queries over e4m3: 32 rows a workgroup in both roles
    (1, "shared", 4, 2, 32, (1 << 26) - 4096, 1, 1, True),
    (1, "shared", 1, 1, 32, 1 << 28, 1, 1, False),
    (1, "attend", 4, 2, 32, 1 << 26, 1, 0, True),
    (0, "shared", 4, 2, 32, 1 << 26, 1, 1, True),             # 128 rows
    (0, "plain", 4, 2, 32, 1 << 26, 1, 1, True),
    (1, "plain", 4, 2, 32, 1 << 26, 1, 1, True),
    (1, "shared", 1, 1, 32, (1 << 28) - (1 << 21), 1 << 20, 1 << 20, False),
    (1, "shared", 2, 1, 16, (1 << 26) - 7, 1 << 19, 1 << 20, True)])
def test_launches_of_too_many_workgroups_are_refused(io_dtype, which, H, Hkv, d, n_new, B, groups, fits):
    L, err = P.lib(), ctypes.c_int(7)
    desc = LactPagedDesc(**dict(PAGED, io_dtype=io_dtype, H=H, Hkv=Hkv, d=d, n_new=n_new, B=B))
    if which == "attend":
        need = L.lact_paged_attention_e4m3_workspace_bytes(desc, ctypes.byref(err))
    else:
        need = L.lact_paged_prefix_attention_workspace_bytes(desc, prefix(groups=groups), int(which == "shared"), ctypes.byref(err))
    assert err.value == (0 if fits else EUNSUPPORTED)
    if not fits:
        assert need == 0
        v = view(token=H * d, head=d)
        c = view(batch=16 * Hkv * d, head=d, token=Hkv * d)
        assert call(which, dict(io_dtype=io_dtype, H=H, Hkv=Hkv, d=d, n_new=n_new, B=B), ws=1 << 60, q=v, o=v, k_cache=c, v_cache=c,
                    prefix=prefix(groups=groups)) == EUNSUPPORTED


@pytest.mark.parametrize("B,H,Hkv,d,n_new,page,max_pages,io_dtype", [
    (501, 64, 8, 16, 1 << 21, 1, 74581363, 1), (30, 8, 8, 64, 1 << 24, 128, 1781422, 1), (199, 1, 1, 80, 107374182, 16, 13517319, 1),
    (1018890, 1, 1, 16, 3056670, 1, 265423107, 0), (2110, 8, 8, 16, 1 << 24, 16, 15340556, 0)])
def test_parts_of_wide_tables_stay_within_a_launch(B, H, Hkv, d, n_new, page, max_pages, io_dtype):
    # keys by the hundred million: every part is worth its sums, but some of them fill a launch
    L, err = P.lib(), ctypes.c_int(7)
    desc = LactPagedDesc(**dict(PAGED, B=B, H=H, Hkv=Hkv, d=d, n_new=n_new, page=page, max_pages=max_pages, io_dtype=io_dtype))
    n = L.lact_paged_attention_e4m3_workspace_bytes(desc, ctypes.byref(err))
    parts = max(1, n // (n_new * H * (d + 2) * 4))
    rows = n_new * (H // Hkv)
    size = 32 if io_dtype else 128 if rows > 32 * B else 16       # rows a workgroup
    assert err.value == 0 and parts * (rows // size + B) * Hkv < 1 << 24


def test_workspaces_of_refused_vectors():
    L, err = P.lib(), ctypes.c_int(7)
    f = lambda e4m3: L.lact_paged_prefix_attention_workspace_bytes(LactPagedDesc(**dict(PAGED, d=24)), prefix(), e4m3, ctypes.byref(err))
    assert f(1) == 0 and err.value == EUNSUPPORTED       # as the call
    assert f(0) > 0 and err.value == 0
