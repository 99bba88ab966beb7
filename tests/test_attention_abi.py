"""The attention entry points without a GPU: refusals before any HIP call,
workspace sizes, and the plain 64-bit forms against differences."""
import ctypes
import math

import pytest
import torch

import paper_2505_23884_amd as P
from attention_reference import head, norm_rope, visible
from paper_2505_23884_amd.binding import LactAttnDesc, LactPagedDesc, LactRopeDesc, LactView

EINVAL, EALIGN, EWORKSPACE, EUNSUPPORTED = -1, -2, -3, -4
vp = ctypes.c_void_p


def view(at=0x10000, batch=1 << 16, head=1 << 13, token=128):
    return LactView(at, batch, head, token)


ROPE = dict(B=2, H=4, Hkv=2, d=128, n=33, pos0=0, rot=64, interleaved=0, weight_per_head=0, io_dtype=0, eps=1e-6,
            reserved=0)
ATTN = dict(B=2, H=4, Hkv=2, d=128, n_q=33, n_kv=33, q_start=0, window=16, lookahead=0, sinks=1, scale=0.1, io_dtype=0)
PAGED = dict(B=3, H=4, Hkv=2, d=128, n_new=5, pages=10, page=16, max_pages=4, window=-1, sinks=0, scale=0.1, io_dtype=0)


def rope(desc=None, back=False, ws=None, **a):
    d = LactRopeDesc(**dict(ROPE, **(desc or {})))
    g = lambda n, v: a.get(n, v)
    L = P.lib()
    head_ = [g("q", view()), g("k", view()), g("wq", 0x1000), g("wk", 0x1000), g("inv_freq", 0x1000), g("positions", None)]
    if not back:
        return L.lact_qk_norm_rope(d, *head_, g("qn", view()), g("kn", view()), None)
    need = L.lact_qk_norm_rope_backward_workspace_bytes(d, None)
    return L.lact_qk_norm_rope_backward(d, *head_, g("dqn", view()), g("dkn", view()), g("dq", view()), g("dk", view()),
                                        g("dwq", 0x1000), g("dwk", 0x1000), g("workspace", 0x10000), need if ws is None else ws,
                                        None)


def attn(desc=None, back=False, ws=None, **a):
    d = LactAttnDesc(**dict(ATTN, **(desc or {})))
    g = lambda n, v: a.get(n, v)
    L = P.lib()
    if not back:
        return L.lact_window_attention(d, g("q", view()), g("k", view()), g("v", view()), g("lengths", None),
                                       g("o", view()), g("lse", None), None)
    need = L.lact_window_attention_backward_workspace_bytes(d, None)
    return L.lact_window_attention_backward(d, g("q", view()), g("k", view()), g("v", view()), g("o", view()),
                                            g("lse", 0x1000), g("dout", view()), g("lengths", None), g("dq", view()),
                                            g("dk", view()), g("dv", view()), g("workspace", 0x10000),
                                            need if ws is None else ws, None)


def paged(desc=None, append=False, ws=None, **a):
    d = LactPagedDesc(**dict(PAGED, **(desc or {})))
    g = lambda n, v: a.get(n, v)
    L = P.lib()
    tail = [g("table", 0x1000), g("lens", 0x1000), g("cu_new", 0x1000)]
    if append:
        return L.lact_paged_append(d, g("k", view()), g("v", view()), g("k_cache", view()), g("v_cache", view()), *tail, None)
    need = L.lact_paged_attention_workspace_bytes(d, None)
    return L.lact_paged_attention(d, g("q", view()), g("k_cache", view()), g("v_cache", view()), *tail, g("o", view()),
                                  g("workspace", 0x10000), need if ws is None else ws, None)


HEADS = [("B", 0, EINVAL), ("H", 0, EINVAL), ("Hkv", 3, EINVAL), ("Hkv", 0, EINVAL), ("d", 0, EINVAL), ("d", 12, EUNSUPPORTED),
         ("io_dtype", 2, EINVAL), ("B", 1 << 19, EUNSUPPORTED)]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("field,value,code", HEADS + [
    ("d", 520, EUNSUPPORTED), ("n", -1, EINVAL), ("rot", -2, EINVAL), ("rot", 7, EINVAL), ("rot", 130, EINVAL),
    ("rot", 12, EUNSUPPORTED), ("interleaved", 2, EINVAL), ("weight_per_head", -1, EINVAL), ("eps", -1.0, EINVAL),
    ("eps", math.inf, EINVAL), ("eps", math.nan, EINVAL), ("reserved", 1, EINVAL), ("n", 1 << 31, EUNSUPPORTED),
    ("pos0", 1 << 41, EUNSUPPORTED), ("rot", 0, EINVAL)])
def test_rope_descriptor_is_refused(field, value, code, back):
    assert rope({field: value}, back, ws=1 << 40) == code      # (rot 0 with frequencies given)


def test_rope_arguments_are_refused():
    for back in (False, True):
        assert rope(back=back, inv_freq=None) == EINVAL
        assert rope(back=back, q=None) == EINVAL
        assert rope(back=back, k=view(0)) == EINVAL
        assert rope(back=back, q=view(0x10008)) == EALIGN
        assert rope(back=back, q=view(token=132)) == EALIGN
        assert rope(back=back, q=view(head=-8)) == EINVAL
        assert rope(back=back, wq=0x1002) == EALIGN
        assert rope(back=back, inv_freq=0x1004) == EALIGN
        assert rope(back=back, positions=0x1002) == EALIGN
        assert rope(back=back, q=view(token=1 << 23)) == EUNSUPPORTED
    assert rope(qn=view(token=64)) == EINVAL                   # overlapping outputs
    assert rope(kn=view(head=0)) == EINVAL
    assert rope(back=True, dq=view(batch=0)) == EINVAL
    assert rope(back=True, wq=None) == EINVAL                  # a weight's cotangent without the weight
    assert rope(back=True, ws=16) == EWORKSPACE
    assert rope(back=True, workspace=None) == EWORKSPACE
    assert rope(back=True, workspace=0x10010) == EALIGN
    assert rope({"n": 0}, q=view(0), k=view(0), qn=view(0), kn=view(0)) == 0


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("field,value,code", HEADS + [
    ("d", 264, EUNSUPPORTED), ("n_q", -1, EINVAL), ("n_kv", -1, EINVAL), ("window", -2, EINVAL), ("lookahead", -2, EINVAL),
    ("sinks", -1, EINVAL), ("scale", 0.0, EINVAL), ("scale", -1.0, EINVAL), ("scale", math.inf, EINVAL),
    ("scale", math.nan, EINVAL), ("scale", 1e-13, EUNSUPPORTED), ("scale", 1e13, EUNSUPPORTED),
    ("n_kv", (1 << 29) + 1, EUNSUPPORTED), ("q_start", 1 << 30, EUNSUPPORTED), ("q_start", -(1 << 30), EUNSUPPORTED)])
def test_window_descriptor_is_refused(field, value, code, back):
    assert attn({field: value}, back, ws=1 << 40) == code


def test_window_arguments_are_refused():
    for back in (False, True):
        for name in ("q", "k", "v", "o"):
            assert attn(back=back, **{name: None}) == EINVAL
            assert attn(back=back, **{name: view(0)}) == EINVAL
            assert attn(back=back, **{name: view(0x10008)}) == EALIGN
            assert attn(back=back, **{name: view(head=(1 << 13) + 4)}) == EALIGN
            assert attn(back=back, **{name: view(token=(1 << 22) + 8)}) == EUNSUPPORTED
        assert attn(back=back, lengths=0x1002) == EALIGN
        assert attn(back=back, lse=0x1001) == EALIGN
    assert attn(o=view(token=0)) == EINVAL
    for head_, token in ((128, 256), (128, 128), (1 << 12, 128), (128, 504)):      # 4 heads of 33 tokens, over each other
        assert attn(o=view(head=head_, token=token)) == EINVAL
    assert attn(o=view(batch=33 * 128 + 64, head=33 * 128)) == EINVAL                  # a batch within the heads
    assert attn(o=view(batch=1 << 62, head=1 << 62)) == EINVAL
    for name in ("dq", "dk", "dv"):
        assert attn(back=True, **{name: view(head=64)}) == EINVAL
    assert attn(back=True, dout=view(0)) == EINVAL
    assert attn(back=True, lse=None) == EINVAL
    assert attn(back=True, ws=64) == EWORKSPACE
    assert attn(back=True, workspace=None) == EWORKSPACE
    assert attn(back=True, workspace=0x10010) == EALIGN
    assert attn({"n_q": 0}, q=view(0), o=view(0)) == 0


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("field,value,code", [
    ("B", 0, EINVAL), ("Hkv", 0, EINVAL), ("d", 12, EUNSUPPORTED), ("d", 264, EUNSUPPORTED), ("io_dtype", 2, EINVAL),
    ("n_new", -1, EINVAL), ("pages", -1, EINVAL), ("page", 0, EINVAL), ("max_pages", -1, EINVAL),
    ("max_pages", 1 << 26, EUNSUPPORTED), ("n_new", 1 << 30, EUNSUPPORTED)])
def test_paged_descriptor_is_refused(field, value, code, append):
    assert paged({field: value}, append, ws=1 << 40) == code


def test_paged_arguments_are_refused():
    for append in (False, True):
        for name in ("k_cache", "v_cache"):
            assert paged(append=append, **{name: None}) == EINVAL
            assert paged(append=append, **{name: view(0)}) == EINVAL
            assert paged(append=append, **{name: view(0x10004)}) == EALIGN
            assert paged(append=append, **{name: view(head=1 << 12)}) == EINVAL      # another layout than the other's
        for name in ("table", "lens", "cu_new"):
            assert paged(append=append, **{name: None}) == EINVAL
            assert paged(append=append, **{name: 0x1002}) == EALIGN
    assert paged(append=True, k=view(0)) == EINVAL
    assert paged(append=True, k_cache=view(batch=0), v_cache=view(batch=0)) == EINVAL
    for f, v in (("window", -2), ("sinks", -1), ("scale", 0.0), ("scale", math.nan), ("H", 3)):
        assert paged({f: v}) == EINVAL
    assert paged(q=view(0)) == EINVAL
    assert paged(o=view(token=0)) == EINVAL
    long = {"max_pages": 4096}
    d = LactPagedDesc(**dict(PAGED, **long))
    assert P.lib().lact_paged_attention_workspace_bytes(d, None) > 0
    assert paged(long, ws=16) == EWORKSPACE
    assert paged(long, workspace=0x10010) == EALIGN
    assert paged({"n_new": 0}, q=view(0), o=view(0)) == 0
    assert paged({"n_new": 0}, append=True, k=view(0), v=view(0)) == 0


def test_calls_past_the_largest_launch_are_refused():
    assert rope({"B": 1, "n": (1 << 25) + 1}) == EUNSUPPORTED
    assert rope({"B": 1 << 10, "n": (1 << 15) + 1}) == EUNSUPPORTED
    for back in (False, True):
        assert attn({"B": 1 << 10, "n_q": 1 << 19}, back, ws=1 << 50) == EUNSUPPORTED
        assert attn({"B": 1 << 10, "n_kv": 1 << 19}, back, ws=1 << 50) == EUNSUPPORTED
    assert paged({"n_new": (1 << 26) + 1}, ws=1 << 50) == EUNSUPPORTED
    assert paged({"n_new": (1 << 25) + 1}, append=True) == EUNSUPPORTED       # times 2 heads of 128


def test_many_sink_tiles_stay_within_a_workspace():
    # every key a sink: no tile is cut into parts, so the workspace holds rows only
    L = P.lib()
    a = dict(ATTN, B=1, n_q=1 << 18, n_kv=1 << 18, window=64, sinks=1 << 18)
    n = L.lact_window_attention_backward_workspace_bytes(LactAttnDesc(**a), None)
    assert 0 < n < 2 * 4 * (4 << 18) + (1 << 20)


def test_workspaces_grow_with_the_call():
    L = P.lib()
    f = lambda **k: L.lact_window_attention_backward_workspace_bytes(LactAttnDesc(**dict(ATTN, **k)), None)
    assert 0 < f() < f(n_q=4096, n_kv=4096)
    err = ctypes.c_int(0)
    assert L.lact_window_attention_backward_workspace_bytes(LactAttnDesc(**dict(ATTN, d=12)), ctypes.byref(err)) == 0
    assert err.value == EUNSUPPORTED


def test_tensors_of_the_host_are_refused():
    t = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    c, i = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16), torch.zeros(1, 2, dtype=torch.int32)
    for call in (lambda: P.window_attention(t, t, t), lambda: P.qk_norm_rope(t, t),
                 lambda: P.paged_attention(t[0], c, c, i, i[0, :1], i[0]), lambda: P.paged_append(t[0], t[0], c, c, i, i[0, :1], i[0])):
        with pytest.raises(P.LactError):
            call()


def test_numbers_that_no_field_holds_are_refused():
    t = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    for opt in (dict(window=1 << 70), dict(q_start=-(1 << 64)), dict(sinks=1 << 63)):
        with pytest.raises(P.LactError, match="out of range"):
            P.window_attention(t, t, t, **opt)


@pytest.mark.parametrize("window,sinks,look", [(None, 0, 0), (3, 1, 0), (4, 0, 2), (None, 0, None)])
def test_attention_gradients_against_differences(window, sinks, look):
    g = torch.Generator().manual_seed(1)
    q, k, v, do = (torch.randn(7, 8, generator=g, dtype=torch.float64) for _ in range(4))
    see = visible(7, 7, 6, 0, window, sinks, look)
    r = head(q, k, v, see, 0.4, do)
    loss = lambda a, b, c: float((head(a, b, c, see, 0.4)["o"] * do).sum())
    h = 1e-5
    for which, grad in ((0, r["dq"]), (1, r["dk"]), (2, r["dv"])):
        for i, j in ((0, 0), (3, 5), (6, 7), (5, 2)):
            x = [q, k, v]
            at = []
            for s in (h, -h):
                y = x[which].clone()
                y[i, j] += s
                at.append(loss(*(y if n == which else x[n] for n in range(3))))
            assert abs((at[0] - at[1]) / (2 * h) - float(grad[i, j])) < 1e-8


@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope_gradients_against_differences(interleaved):
    g = torch.Generator().manual_seed(2)
    x = torch.randn(2, 3, 2, 16, generator=g, dtype=torch.float64)
    dy = torch.randn(2, 2, 3, 16, generator=g, dtype=torch.float64)
    w = torch.rand(16, generator=g, dtype=torch.float64) + 0.5
    f = torch.tensor([1.0, 0.3, 0.01, 2.0], dtype=torch.float64)
    pos = torch.tensor([[0, 5, 9], [100000, 2, -3]])
    _, dx, dw, _, _ = norm_rope(x, w, f, pos, 1e-3, interleaved, dy)
    loss = lambda a, b: float((norm_rope(a, b, f, pos, 1e-3, interleaved) * dy).sum())
    h = 1e-5
    for at in ((0, 0, 0, 0), (1, 0, 1, 3), (1, 2, 0, 9), (0, 1, 1, 15)):
        y = [x.clone(), x.clone()]
        y[0][at] += h
        y[1][at] -= h
        assert abs((loss(y[0], w) - loss(y[1], w)) / (2 * h) - float(dx[at])) < 1e-8
    for i in (0, 7, 15):
        u = [w.clone(), w.clone()]
        u[0][i] += h
        u[1][i] -= h
        assert abs((loss(x, u[0]) - loss(x, u[1])) / (2 * h) - float(dw.sum(0)[i])) < 1e-8


def test_norm_of_more_tokens_than_one_launch_holds_is_refused():
    # q's and k's workgroups share a launch of fewer than 2^32 threads, four tokens in 256 of them at least
    for n in (1 << 25, (1 << 25) - 3):
        for back in (False, True):
            assert rope({"B": 1, "n": n}, back, ws=1 << 50) == EUNSUPPORTED
    assert rope({"B": 1 << 10, "n": 1 << 15}) == EUNSUPPORTED


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("desc", [{"B": 1 << 10, "H": 1 << 10, "Hkv": 1 << 10, "n_q": 1, "n_kv": 897},
                                  {"B": 1 << 10, "H": 1 << 10, "n_q": 1 << 10, "n_kv": 1}, {"B": 2, "H": 1, "Hkv": 1, "n_q": 1 << 29}])
def test_window_attention_of_more_tiles_than_one_launch_holds_is_refused(desc, back):
    # 2^23 tiles of 128 in workgroups of 512: 2^32 threads
    assert attn(desc, back, ws=1 << 50) == EUNSUPPORTED


def test_views_of_more_elements_than_an_integer_counts_are_looked_at():
    # pages x heads x slots = 2^64, or a multiple of it
    for pages, heads, page in ((1 << 30, 1 << 20, 1 << 14), (1 << 30, 1 << 19, 1 << 16)):
        big = {"B": 1, "H": heads, "Hkv": heads, "pages": pages, "page": page, "n_new": 1}
        for bad in (view(0), view(0x10008)):
            assert paged(big, ws=1 << 50, k_cache=bad) in (EINVAL, EALIGN)
            assert paged(big, append=True, k_cache=bad) in (EINVAL, EALIGN)
