"""ctypes binding of liblact.so with the names of the C ABI (include/lact.h)."""
from __future__ import annotations

import ctypes
import os
import struct

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "liblact.so")

APPLY_THEN_UPDATE, UPDATE_THEN_APPLY = 0, 1
IO_BF16, IO_FP32 = 0, 1
KCLASS_NAMES = ("fwd", "bwd", "update", "ns", "prep", "io", "attn")

_ERRORS = {0: "LACT_OK", -1: "LACT_EINVAL", -2: "LACT_EALIGN", -3: "LACT_EWORKSPACE",
           -4: "LACT_EUNSUPPORTED", -5: "LACT_EHIP", -6: "LACT_ESCRATCH"}
NOALLOC_SCRATCH_BYTES = 128 << 20   # LACT_NOALLOC_SCRATCH_BYTES


class LactError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{_ERRORS.get(code, code)}: {msg}")
        self.code = code


class LactDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32),
                ("h", ctypes.c_int32), ("n_kv", ctypes.c_int64), ("n_q", ctypes.c_int64),
                ("chunk", ctypes.c_int64), ("order", ctypes.c_int32), ("use_muon", ctypes.c_int32),
                ("ns_steps", ctypes.c_int32), ("io_dtype", ctypes.c_int32), ("eta_per_matrix", ctypes.c_int32),
                ("fast_weight", ctypes.c_int32)]


FW_SWIGLU, FW_LINEAR = 0, 1


SEG_APPLY_THEN_UPDATE, SEG_UPDATE_THEN_APPLY, SEG_UPDATE_ONLY, SEG_APPLY_ONLY = 0, 1, 2, 3
SEG_MODES = {"apply_then_update": 0, "update_then_apply": 1, "update_only": 2, "apply_only": 3}


class LactSegment(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int32), ("reserved", ctypes.c_int32), ("begin", ctypes.c_int64),
                ("end", ctypes.c_int64)]


class LactView(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("head", ctypes.c_int64),
                ("token", ctypes.c_int64)]


class LactRopeDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("n", ctypes.c_int64), ("pos0", ctypes.c_int64), ("rot", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("weight_per_head", ctypes.c_int32), ("io_dtype", ctypes.c_int32),
                ("eps", ctypes.c_float), ("reserved", ctypes.c_int32)]


class LactAttnDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("n_q", ctypes.c_int64), ("n_kv", ctypes.c_int64), ("q_start", ctypes.c_int64),
                ("window", ctypes.c_int64), ("lookahead", ctypes.c_int64), ("sinks", ctypes.c_int64),
                ("scale", ctypes.c_float), ("io_dtype", ctypes.c_int32)]


class LactPagedDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("n_new", ctypes.c_int64), ("pages", ctypes.c_int64), ("page", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("window", ctypes.c_int64), ("sinks", ctypes.c_int64),
                ("scale", ctypes.c_float), ("io_dtype", ctypes.c_int32)]


class LactPrefix(ctypes.Structure):
    _fields_ = [("groups", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("table", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("cu_seq", ctypes.c_void_p)]


_lib = None


def load_library(path: str | None = None):
    """Load liblact.so (raises if it has not been built: there is no fallback)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise LactError(-5, f"{p} is missing; build it with paper_2505_23884_amd.build.build()")
    L = ctypes.CDLL(p)
    vp, sz, i32, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int64
    dp = ctypes.POINTER(LactDesc)
    L.lact_workspace_bytes.argtypes = [dp, ctypes.POINTER(i32)]
    L.lact_workspace_bytes.restype = sz
    L.lact_check_desc.argtypes = [dp]
    L.lact_check_desc.restype = i32
    L.lact_forward.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.lact_forward.restype = i32
    L.lact_forward_noalloc.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.lact_forward_noalloc.restype = i32
    L.lact_forward_momentum.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.lact_forward_momentum.restype = i32
    L.lact_forward_schedule.argtypes = [dp, ctypes.POINTER(LactSegment), i64] + [vp] * 13 + [sz, vp]
    L.lact_forward_schedule.restype = i32
    L.lact_backward_workspace_bytes.argtypes = [dp, ctypes.POINTER(i32)]
    L.lact_backward_workspace_bytes.restype = sz
    L.lact_backward_linear.argtypes = [dp] + [vp] * 12 + [vp, sz, vp]
    L.lact_backward_linear.restype = i32
    L.lact_backward.argtypes = [dp] + [vp] * 19 + [sz, vp]
    L.lact_backward.restype = i32
    L.lact_backward_momentum_workspace_bytes.argtypes = [dp, ctypes.POINTER(i32)]
    L.lact_backward_momentum_workspace_bytes.restype = sz
    L.lact_backward_momentum.argtypes = [dp] + [vp] * 30 + [sz, vp]
    L.lact_backward_momentum.restype = i32
    L.lact_backward_schedule_workspace_bytes.argtypes = [dp, ctypes.POINTER(LactSegment), i64, i32,
                                                         ctypes.POINTER(i32)]
    L.lact_backward_schedule_workspace_bytes.restype = sz
    L.lact_backward_schedule.argtypes = [dp, ctypes.POINTER(LactSegment), i64] + [vp] * 30 + [sz, vp]
    L.lact_backward_schedule.restype = i32
    f32 = ctypes.c_float
    L.lact_prologue.argtypes = [dp, vp, vp, f32, vp, vp, vp, vp, vp, vp, vp]
    L.lact_prologue.restype = i32
    L.lact_rmsnorm_out.argtypes = [dp, vp, vp, f32, vp, vp]
    L.lact_prologue_backward.argtypes = [dp, vp, vp, f32] + [vp] * 10
    L.lact_prologue_backward.restype = i32
    L.lact_rmsnorm_out_backward_workspace_bytes.argtypes = [dp, i32, ctypes.POINTER(i32)]
    L.lact_rmsnorm_out_backward_workspace_bytes.restype = sz
    L.lact_rmsnorm_out_backward.argtypes = [dp, vp, vp, f32, vp, vp, vp, vp, sz, vp]
    L.lact_rmsnorm_out_backward.restype = i32
    L.lact_rmsnorm_out.restype = i32
    vw, ip = ctypes.POINTER(LactView), ctypes.POINTER(i32)
    rp, ap, pp = ctypes.POINTER(LactRopeDesc), ctypes.POINTER(LactAttnDesc), ctypes.POINTER(LactPagedDesc)
    L.lact_qk_norm_rope.argtypes = [rp, vw, vw, vp, vp, vp, vp, vw, vw, vp]
    L.lact_qk_norm_rope_backward.argtypes = [rp, vw, vw, vp, vp, vp, vp, vw, vw, vw, vw, vp, vp, vp, sz, vp]
    L.lact_window_attention.argtypes = [ap, vw, vw, vw, vp, vw, vp, vp]
    L.lact_window_attention_backward.argtypes = [ap, vw, vw, vw, vw, vp, vw, vp, vw, vw, vw, vp, sz, vp]
    L.lact_paged_append.argtypes = [pp, vw, vw, vw, vw, vp, vp, vp, vp]
    L.lact_paged_attention.argtypes = [pp, vw, vw, vw, vp, vp, vp, vw, vp, sz, vp]
    xp = ctypes.POINTER(LactPrefix)
    L.lact_paged_append_e4m3.argtypes = [pp] + [vw] * 6 + [vp] * 4
    L.lact_paged_read_e4m3.argtypes = [pp] + [vw] * 4 + [vp] * 3 + [vw, vw, vp]
    L.lact_paged_attention_e4m3.argtypes = [pp] + [vw] * 5 + [vp] * 3 + [vw, vp, sz, vp]
    L.lact_paged_prefix_attention.argtypes = [pp, xp] + [vw] * 5 + [vp] * 3 + [vw, vp, sz, vp]
    L.lact_paged_prefix_attention_workspace_bytes.argtypes = [pp, xp, i32, ip]
    L.lact_paged_prefix_attention_workspace_bytes.restype = sz
    for f in ("lact_qk_norm_rope", "lact_qk_norm_rope_backward", "lact_window_attention",
              "lact_window_attention_backward", "lact_paged_append", "lact_paged_attention", "lact_paged_append_e4m3",
              "lact_paged_read_e4m3", "lact_paged_attention_e4m3", "lact_paged_prefix_attention"):
        getattr(L, f).restype = i32
    for f, desc in (("lact_qk_norm_rope_backward_workspace_bytes", rp),
                    ("lact_window_attention_backward_workspace_bytes", ap),
                    ("lact_paged_attention_workspace_bytes", pp),
                    ("lact_paged_attention_e4m3_workspace_bytes", pp)):
        getattr(L, f).argtypes = [desc, ip]
        getattr(L, f).restype = sz
    L.lact_timing_enable.argtypes = [i32]
    L.lact_timing_enable.restype = i32
    L.lact_timing_reset.argtypes = []
    L.lact_timing_reset.restype = i32
    L.lact_timing_read.argtypes = [i32, ctypes.POINTER(i64), ctypes.POINTER(ctypes.c_double),
                                   ctypes.POINTER(ctypes.c_double)]
    L.lact_timing_read.restype = i32
    for f in ("lact_strerror",):
        getattr(L, f).argtypes = [i32]
        getattr(L, f).restype = ctypes.c_char_p
    for f in ("lact_last_hip_error", "lact_version"):
        getattr(L, f).argtypes = []
        getattr(L, f).restype = ctypes.c_char_p
    if path is None:
        _lib = L
    return L


def lib():
    return load_library()


def _raise(code: int):
    L = lib()
    msg = L.lact_strerror(code).decode()
    if code == -5:
        msg += ": " + L.lact_last_hip_error().decode()
    raise LactError(code, msg)


def make_desc(B, H, d, h, n_kv, n_q, chunk, order=0, use_muon=False, ns_steps=5, io_dtype=IO_BF16,
              eta_per_matrix=False, fast_weight=FW_SWIGLU):
    return LactDesc(int(B), int(H), int(d), int(h), int(n_kv), int(n_q), int(chunk), int(order),
                    int(bool(use_muon)), int(ns_steps), int(io_dtype), int(bool(eta_per_matrix)), int(fast_weight))


def check_desc(desc: LactDesc) -> int:
    return lib().lact_check_desc(ctypes.byref(desc))


def workspace_bytes(desc: LactDesc) -> int:
    err = ctypes.c_int(0)
    n = lib().lact_workspace_bytes(ctypes.byref(desc), ctypes.byref(err))
    if err.value:
        _raise(err.value)
    return int(n)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)


def _marshal(q, k, v, eta, W1, W2, W3, extra, chunk, order, use_muon, ns_steps, out, workspace, stream,
             fast_weight=FW_SWIGLU, need_workspace=True):
    """Checks shapes and dtypes; returns (desc, out, workspace, stream handle)
    (workspace None when need_workspace is False)."""
    import torch
    if q.dim() == 4:
        B, H = q.shape[0], q.shape[1]
    elif q.dim() == 3:
        B, H = q.shape[0], 1
    else:
        raise LactError(-1, "q must be [B, H, n_q, d] or [BH, n_q, d]")
    n_q, d = q.shape[-2], q.shape[-1]
    n_kv = k.shape[-2]
    h = W1.shape[-2]
    if q.dtype == torch.bfloat16:
        io = IO_BF16
    elif q.dtype == torch.float32:
        io = IO_FP32
    else:
        raise LactError(-1, f"unsupported q dtype {q.dtype}")
    named = [(q, "q"), (k, "k"), (v, "v"), (eta, "eta"), (W1, "W1"), (W2, "W2"), (W3, "W3"), *extra]
    for t, name in named:
        if not t.is_cuda or not t.is_contiguous():
            raise LactError(-1, f"{name} must be a contiguous device tensor")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise LactError(-1, "q, k, v must share one dtype")
    if eta.dtype != torch.float32 or any(t.dtype != torch.float32 for t, _ in named[4:]):
        raise LactError(-1, "eta, beta, the fast weights and the momentum are fp32")
    BH = B * H
    # per-matrix rates: eta [.., n_kv, 3] (one more trailing dim than k's token axis)
    lr3 = eta.dim() == k.dim() and eta.shape[-1] == 3
    if (k.numel() != BH * n_kv * d or v.numel() != BH * n_kv * d or eta.numel() != BH * n_kv * (3 if lr3 else 1)
            or W1.numel() != BH * h * d or W3.numel() != BH * h * d or W2.numel() != BH * d * h
            or W2.shape[-2] != d or W2.shape[-1] != h or W1.shape[-1] != d):
        raise LactError(-1, "inconsistent tensor shapes")
    desc = make_desc(B, H, d, h, n_kv, n_q, chunk, order, use_muon, ns_steps, io, lr3, fast_weight)
    if need_workspace and workspace is None:
        workspace = torch.empty(max(workspace_bytes(desc), 1), dtype=torch.uint8, device=q.device)
    if out is None:
        out = torch.empty_like(q)
    if stream is None:
        stream = torch.cuda.current_stream(q.device).cuda_stream
    return desc, out, workspace, stream


def forward(q, k, v, eta, W1, W2, W3, chunk, order=APPLY_THEN_UPDATE, use_muon=False,
            ns_steps=5, out=None, workspace=None, stream=None):
    """LaCT fast-weight path on the GPU (see include/lact.h for the semantics).

    q [B, H, n_q, d] (or [BH, n_q, d]); k, v [.., n_kv, d]; bf16 or fp32 (same dtype);
    eta [.., n_kv] fp32; W1, W3 [.., h, d], W2 [.., d, h] fp32, updated IN PLACE.
    Returns o with q's shape and dtype. Runs on torch's current stream unless a
    stream is given; allocates the workspace unless one is passed.
    """
    desc, out, workspace, stream = _marshal(q, k, v, eta, W1, W2, W3, [], chunk, order, use_muon,
                                            ns_steps, out, workspace, stream)
    rc = lib().lact_forward(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(eta), _ptr(W1),
                            _ptr(W2), _ptr(W3), _ptr(out), _ptr(workspace),
                            ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                            ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    return out


def forward_noalloc(q, k, v, eta, W1, W2, W3, chunk, order=APPLY_THEN_UPDATE, use_muon=False, ns_steps=5,
                    out=None, stream=None):
    """forward() through lact_forward_noalloc: no workspace argument; the
    library's fixed per-device scratch array serves as the workspace (calls
    that may overlap on one device race on it). ``out`` is allocated here
    when not given (pass it to allocate nothing)."""
    desc, out, _, stream = _marshal(q, k, v, eta, W1, W2, W3, [], chunk, order, use_muon, ns_steps, out, None,
                                    stream, need_workspace=False)
    rc = lib().lact_forward_noalloc(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(eta), _ptr(W1),
                                    _ptr(W2), _ptr(W3), _ptr(out), ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    return out


def forward_momentum(q, k, v, eta, beta, W1, W2, W3, M1=None, M2=None, M3=None, *, chunk,
                     order=APPLY_THEN_UPDATE, use_muon=False, ns_steps=5, out=None, workspace=None,
                     stream=None):
    """The path with the momentum test-time optimizer (lact_forward_momentum).

    beta [.., n_kv] fp32 per-token momentum factor; M1, M3 [.., h, d], M2 [.., d, h]
    fp32 momentum, updated IN PLACE (zeros are allocated when omitted). W as in
    forward(). Returns (o, (M1, M2, M3)).
    """
    import torch
    if M1 is None and M2 is None and M3 is None:
        M1, M2, M3 = (torch.zeros_like(w) for w in (W1, W2, W3))
    if M1 is None or M2 is None or M3 is None:
        raise LactError(-1, "pass all three momentum tensors or none")
    for m, w, name in ((M1, W1, "M1"), (M2, W2, "M2"), (M3, W3, "M3")):
        if m.shape != w.shape:
            raise LactError(-1, f"{name} must have the shape of its fast weight")
    if beta.numel() != k.numel() // k.shape[-1]:
        raise LactError(-1, "beta must be [.., n_kv]")
    extra = [(beta, "beta"), (M1, "M1"), (M2, "M2"), (M3, "M3")]
    desc, out, workspace, stream = _marshal(q, k, v, eta, W1, W2, W3, extra, chunk, order, use_muon,
                                            ns_steps, out, workspace, stream)
    rc = lib().lact_forward_momentum(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(eta),
                                     _ptr(beta), _ptr(W1), _ptr(W2), _ptr(W3), _ptr(M1), _ptr(M2),
                                     _ptr(M3), _ptr(out), _ptr(workspace),
                                     ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                                     ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    return out, (M1, M2, M3)


def forward_linear(q, k, v, eta, W, chunk, order=APPLY_THEN_UPDATE, use_muon=False, ns_steps=5, beta=None, M=None,
                   out=None, workspace=None, stream=None):
    """The path with the linear fast weight f_W(x) = W x (lact_desc.fast_weight =
    LACT_FW_LINEAR): W [.., d, d] fp32, updated IN PLACE; q, k, v, eta as in
    forward(). With ``beta`` the updates use momentum (M [.., d, d] updated in
    place, zeros allocated when omitted) and the return is (o, M); else o.
    """
    import torch
    if W.shape[-1] != W.shape[-2]:
        raise LactError(-1, "the linear fast weight is square, [.., d, d]")
    extra = []
    if beta is not None:
        M = torch.zeros_like(W) if M is None else M
        if M.shape != W.shape:
            raise LactError(-1, "M must have W's shape")
        extra = [(beta, "beta"), (M, "M")]
    # W stands in for all three matrices in the shape checks (h = d)
    desc, out, workspace, stream = _marshal(q, k, v, eta, W, W, W, extra, chunk, order, use_muon, ns_steps, out,
                                            workspace, stream, FW_LINEAR)
    wsb = ctypes.c_size_t(workspace.numel() * workspace.element_size())
    if beta is None:
        rc = lib().lact_forward(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(eta), _ptr(W), ctypes.c_void_p(0),
                                ctypes.c_void_p(0), _ptr(out), _ptr(workspace), wsb, ctypes.c_void_p(stream))
    else:
        rc = lib().lact_forward_momentum(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(eta), _ptr(beta), _ptr(W),
                                         ctypes.c_void_p(0), ctypes.c_void_p(0), _ptr(M), ctypes.c_void_p(0),
                                         ctypes.c_void_p(0), _ptr(out), _ptr(workspace), wsb, ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    return (out, M) if beta is not None else out


def backward_workspace_bytes(desc: LactDesc) -> int:
    err = ctypes.c_int(0)
    n = lib().lact_backward_workspace_bytes(ctypes.byref(desc), ctypes.byref(err))
    if err.value:
        _raise(err.value)
    return int(n)


def backward_linear(q, k, v, eta, W0, dout, chunk, order=APPLY_THEN_UPDATE, dW_final=None, use_muon=False,
                    ns_steps=5, out=None, workspace=None, stream=None):
    """Backward of forward_linear (lact_backward_linear): the cotangents of q,
    k, v, eta and of the initial fast weight W0 [.., d, d] (fp32, not written)
    given dout (q's shape and dtype) and, optionally, the cotangent of the
    final fast weight. Returns (dq, dk, dv, deta, dW0), written into ``out``
    (a tuple of five tensors of those shapes) when it is given."""
    import torch
    if W0.shape[-1] != W0.shape[-2]:
        raise LactError(-1, "the linear fast weight is square, [.., d, d]")
    extra = [(dout, "dout")] + ([(dW_final, "dW_final")] if dW_final is not None else [])
    if dout.shape != q.shape or dout.dtype != q.dtype:
        raise LactError(-1, "dout must have q's shape and dtype")
    if dW_final is not None and (dW_final.shape != W0.shape or dW_final.dtype != torch.float32):
        raise LactError(-1, "dW_final must have W0's shape, fp32")
    desc, dq, _, stream = _marshal(q, k, v, eta, W0, W0, W0, extra[1:], chunk, order, use_muon, ns_steps,
                                   None if out is None else out[0], None, stream, FW_LINEAR, need_workspace=False)
    if not dout.is_cuda or not dout.is_contiguous():
        raise LactError(-1, "dout must be a contiguous device tensor")
    if workspace is None:
        workspace = torch.empty(max(backward_workspace_bytes(desc), 1), dtype=torch.uint8, device=q.device)
    if out is None:
        dk, dv = torch.empty_like(k), torch.empty_like(v)
        deta = torch.empty_like(eta)
        dW0 = torch.empty_like(W0)
    else:
        _, dk, dv, deta, dW0 = out
        for t, ref, name in ((dq, q, "dq"), (dk, k, "dk"), (dv, v, "dv"), (deta, eta, "deta"), (dW0, W0, "dW0")):
            if t.shape != ref.shape or t.dtype != ref.dtype or not t.is_cuda or not t.is_contiguous():
                raise LactError(-1, f"{name} must be a contiguous device tensor shaped like its input")
    rc = lib().lact_backward_linear(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(eta), _ptr(W0), _ptr(dout),
                                    _ptr(dW_final), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(deta), _ptr(dW0),
                                    _ptr(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                                    ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    return dq, dk, dv, deta, dW0


def backward(q, k, v, eta, W1, W2, W3, dout, chunk, order=APPLY_THEN_UPDATE, dW_final=None, use_muon=False,
             ns_steps=5, out=None, workspace=None, stream=None):
    """Backward of forward() for the SwiGLU fast weight (lact_backward), with
    or without Muon, one rate per token or per matrix, no momentum: the cotangents of q, k, v, eta and of the initial fast
    weights W1, W2, W3 (fp32, not written) given dout (q's shape and dtype)
    and, optionally, dW_final = (dW1, dW2, dW3) of the final fast weights (any
    of them None). Returns (dq, dk, dv, deta, dW1, dW2, dW3), written into
    ``out`` (a tuple of seven tensors of those shapes) when it is given."""
    import torch
    dWf = tuple(dW_final) if dW_final is not None else (None, None, None)
    extra = [(t, name) for t, name in zip(dWf, ("dW1_final", "dW2_final", "dW3_final")) if t is not None]
    if dout.shape != q.shape or dout.dtype != q.dtype:
        raise LactError(-1, "dout must have q's shape and dtype")
    for t, ref in zip(dWf, (W1, W2, W3)):
        if t is not None and (t.shape != ref.shape or t.dtype != torch.float32):
            raise LactError(-1, "dW_final tensors must have the fast weights' shapes, fp32")
    desc, dq, _, stream = _marshal(q, k, v, eta, W1, W2, W3, extra, chunk, order, use_muon, ns_steps,
                                   None if out is None else out[0], None, stream, FW_SWIGLU, need_workspace=False)
    if not dout.is_cuda or not dout.is_contiguous():
        raise LactError(-1, "dout must be a contiguous device tensor")
    if workspace is None:
        workspace = torch.empty(max(backward_workspace_bytes(desc), 1), dtype=torch.uint8, device=q.device)
    if out is None:
        res = (dq, torch.empty_like(k), torch.empty_like(v), torch.empty_like(eta), torch.empty_like(W1),
               torch.empty_like(W2), torch.empty_like(W3))
    else:
        res = tuple(out)
        for t, ref, name in zip(res, (q, k, v, eta, W1, W2, W3), ("dq", "dk", "dv", "deta", "dW1", "dW2", "dW3")):
            if t.shape != ref.shape or t.dtype != ref.dtype or not t.is_cuda or not t.is_contiguous():
                raise LactError(-1, f"{name} must be a contiguous device tensor shaped like its input")
    rc = lib().lact_backward(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(eta), _ptr(W1), _ptr(W2), _ptr(W3),
                             _ptr(dout), _ptr(dWf[0]), _ptr(dWf[1]), _ptr(dWf[2]), *(_ptr(t) for t in res),
                             _ptr(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                             ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    return res


def backward_momentum_workspace_bytes(desc: LactDesc) -> int:
    err = ctypes.c_int(0)
    n = lib().lact_backward_momentum_workspace_bytes(ctypes.byref(desc), ctypes.byref(err))
    if err.value:
        _raise(err.value)
    return int(n)


def backward_momentum(q, k, v, eta, beta, W0, M0, dout, chunk, order=APPLY_THEN_UPDATE, dW_final=None,
                      dM_final=None, use_muon=False, ns_steps=5, out=None, workspace=None, stream=None):
    """Backward of the momentum optimizer's path (lact_backward_momentum).

    W0, M0: the fast weights and momentum before the forward (fp32, not
    written): triples (W1, W2, W3), (M1, M2, M3) for SwiGLU, single [.., d, d]
    tensors for the linear fast weight; dW_final, dM_final the same (any of
    them None: zero). Returns (dq, dk, dv, deta, dbeta, dW0, dM0) with dW0,
    dM0 shaped like W0, M0; written into ``out`` (that tuple) when given."""
    import torch
    linear = not isinstance(W0, (tuple, list))
    Ws = (W0,) if linear else tuple(W0)
    Ms = (M0,) if linear else tuple(M0)
    nm = len(Ws)
    if nm not in (1, 3) or len(Ms) != nm:
        raise LactError(-1, "W0 and M0: three tensors (SwiGLU) or one (linear)")
    if linear and W0.shape[-1] != W0.shape[-2]:
        raise LactError(-1, "the linear fast weight is square, [.., d, d]")
    dWf = (None,) * nm if dW_final is None else ((dW_final,) if linear else tuple(dW_final))
    dMf = (None,) * nm if dM_final is None else ((dM_final,) if linear else tuple(dM_final))
    if len(dWf) != nm or len(dMf) != nm:
        raise LactError(-1, "dW_final and dM_final must match W0")
    for t, ref in zip(Ms + dWf + dMf, Ws * 3):
        if t is not None and (t.shape != ref.shape or t.dtype != torch.float32):
            raise LactError(-1, "momentum and final cotangents must have the fast weights' shapes, fp32")
    if dout.shape != q.shape or dout.dtype != q.dtype:
        raise LactError(-1, "dout must have q's shape and dtype")
    if beta.numel() != k.numel() // k.shape[-1] or beta.dtype != torch.float32:
        raise LactError(-1, "beta must be [.., n_kv] fp32")
    extra = [(beta, "beta")] + [(t, "M") for t in Ms] + [(t, "d_final") for t in dWf + dMf if t is not None]
    W1, W2, W3 = (Ws[0],) * 3 if linear else Ws
    desc, dq, _, stream = _marshal(q, k, v, eta, W1, W2, W3, extra, chunk, order, use_muon, ns_steps,
                                   None if out is None else out[0], None, stream,
                                   FW_LINEAR if linear else FW_SWIGLU, need_workspace=False)
    if not dout.is_cuda or not dout.is_contiguous():
        raise LactError(-1, "dout must be a contiguous device tensor")
    if workspace is None:
        workspace = torch.empty(max(backward_momentum_workspace_bytes(desc), 1), dtype=torch.uint8, device=q.device)
    if out is None:
        dW = tuple(torch.empty_like(w) for w in Ws)
        dM = tuple(torch.empty_like(m) for m in Ms)
        head = (dq, torch.empty_like(k), torch.empty_like(v), torch.empty_like(eta), torch.empty_like(beta))
    else:
        head = tuple(out[:5])
        dW = (out[5],) if linear else tuple(out[5])
        dM = (out[6],) if linear else tuple(out[6])
        refs = (q, k, v, eta, beta) + Ws + Ms
        for t, ref in zip(head + dW + dM, refs):
            if t.shape != ref.shape or t.dtype != ref.dtype or not t.is_cuda or not t.is_contiguous():
                raise LactError(-1, "outputs must be contiguous device tensors shaped like their inputs")
    pad = (lambda xs: tuple(xs) + (None,) * (3 - len(xs)))
    args = ([_ptr(q), _ptr(k), _ptr(v), _ptr(eta), _ptr(beta)] + [_ptr(t) for t in pad(Ws)] +
            [_ptr(t) for t in pad(Ms)] + [_ptr(dout)] + [_ptr(t) for t in pad(dWf)] + [_ptr(t) for t in pad(dMf)] +
            [_ptr(t) for t in head[:4]] + [_ptr(head[4])] + [_ptr(t) for t in pad(dW)] + [_ptr(t) for t in pad(dM)])
    rc = lib().lact_backward_momentum(ctypes.byref(desc), *args, _ptr(workspace),
                                      ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                                      ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    if linear:
        return head + (dW[0], dM[0])
    return head + (dW, dM)


def forward_schedule(q, k, v, eta, W1, W2, W3, schedule, *, use_muon=False, ns_steps=5, beta=None,
                     M1=None, M2=None, M3=None, chunk=None, out=None, workspace=None, stream=None):
    """The path over a general schedule (lact_forward_schedule): ``schedule`` is a
    sequence of (mode, begin, end) with mode a name of SEG_MODES or its code.
    ``chunk`` (the workspace bound) defaults to the longest update segment.
    With ``beta`` the updates use momentum (M1..M3 updated in place, zeros
    allocated when omitted). Returns o, or (o, (M1, M2, M3)) with beta.
    With W2 and W3 None the fast weight is the linear one (W1 [.., d, d];
    M1 its state, returned alone; M2 and M3 unused).
    """
    import torch
    segs, longest = _segments(schedule)
    linear = W2 is None and W3 is None
    extra = []
    if beta is not None:
        if linear:
            M1 = torch.zeros_like(W1) if M1 is None else M1
            if M1.shape != W1.shape:
                raise LactError(-1, "M1 must have W1's shape")
            extra = [(beta, "beta"), (M1, "M1")]
        else:
            if M1 is None and M2 is None and M3 is None:
                M1, M2, M3 = (torch.zeros_like(w) for w in (W1, W2, W3))
            if M1 is None or M2 is None or M3 is None:
                raise LactError(-1, "pass all three momentum tensors or none")
            extra = [(beta, "beta"), (M1, "M1"), (M2, "M2"), (M3, "M3")]
    if linear and W1.shape[-1] != W1.shape[-2]:
        raise LactError(-1, "the linear fast weight is square, [.., d, d]")
    Wm = (W1, W1, W1) if linear else (W1, W2, W3)
    desc, out, workspace, stream = _marshal(q, k, v, eta, *Wm, extra, chunk or longest, 0, use_muon,
                                            ns_steps, out, workspace, stream, FW_LINEAR if linear else FW_SWIGLU)
    M = (M1, M2, M3) if beta is not None else (None, None, None)
    rc = lib().lact_forward_schedule(ctypes.byref(desc), segs, ctypes.c_int64(len(schedule)), _ptr(q), _ptr(k),
                                     _ptr(v), _ptr(eta), _ptr(beta), _ptr(W1), _ptr(W2), _ptr(W3),
                                     *[_ptr(m) for m in M], _ptr(out), _ptr(workspace),
                                     ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                                     ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    if beta is not None:
        return out, (M1 if linear else M)
    return out


def _segments(schedule):
    """ctypes segments of a (mode, begin, end) sequence, and the longest update."""
    segs = (LactSegment * max(len(schedule), 1))()
    longest = 1
    for i, (mode, b, e) in enumerate(schedule):
        m = SEG_MODES[mode] if isinstance(mode, str) else int(mode)
        segs[i] = LactSegment(m, 0, int(b), int(e))
        if m != SEG_APPLY_ONLY:
            longest = max(longest, int(e) - int(b))
    return segs, longest


def backward_schedule_workspace_bytes(desc: LactDesc, schedule, momentum=False) -> int:
    segs, _ = _segments(schedule)
    err = ctypes.c_int(0)
    n = lib().lact_backward_schedule_workspace_bytes(ctypes.byref(desc), segs, ctypes.c_int64(len(schedule)),
                                                     int(bool(momentum)), ctypes.byref(err))
    if err.value:
        _raise(err.value)
    return int(n)


def backward_schedule(q, k, v, eta, W1, W2, W3, dout, schedule, *, dW_final=None, use_muon=False, ns_steps=5,
                      beta=None, M=None, dM_final=None, chunk=None, out=None, workspace=None, stream=None):
    """Backward of forward_schedule (lact_backward_schedule), SwiGLU fast
    weight: the cotangents of q, k, v, eta and of the initial W1, W2, W3 (not
    written) given dout and, optionally, dW_final = (dW1, dW2, dW3). With
    ``beta`` the momentum optimizer (M = (M1, M2, M3) the initial state, zeros
    when omitted; dM_final its final cotangents). Returns (dq, dk, dv, deta,
    (dW1, dW2, dW3)) or, with beta, (dq, dk, dv, deta, dbeta, (dW1, dW2, dW3),
    (dM1, dM2, dM3)); written into ``out`` (that tuple) when given. With W2
    and W3 None the fast weight is the linear one: W1 [.., d, d], and M,
    dW_final, dM_final and the returned dW, dM single tensors."""
    import torch
    segs, longest = _segments(schedule)
    linear = W2 is None and W3 is None
    if linear and W1.shape[-1] != W1.shape[-2]:
        raise LactError(-1, "the linear fast weight is square, [.., d, d]")
    one = lambda t: None if t is None else (t,)
    W = (W1,) if linear else (W1, W2, W3)
    mom = beta is not None
    if linear:
        M, dW_final, dM_final = one(M), one(dW_final), one(dM_final)
        if out is not None:
            out = tuple(out[:-2]) + ((out[-2],), (out[-1],)) if mom else tuple(out[:-1]) + ((out[-1],),)
    if mom and M is None:
        M = tuple(torch.zeros_like(w) for w in W)
    dWf = (None,) * len(W) if dW_final is None else tuple(dW_final)
    dMf = (None,) * len(W) if (dM_final is None or not mom) else tuple(dM_final)
    for t, ref in zip(dWf + dMf + (tuple(M) if mom else ()), W * 3):
        if t is not None and (t.shape != ref.shape or t.dtype != torch.float32):
            raise LactError(-1, "momentum and final cotangents must have the fast weights' shapes, fp32")
    if dout.shape != q.shape or dout.dtype != q.dtype:
        raise LactError(-1, "dout must have q's shape and dtype")
    extra = [(t, "d_final") for t in dWf + dMf if t is not None]
    if mom:
        extra += [(beta, "beta")] + [(m, "M") for m in M]
    Wm = (W1, W1, W1) if linear else W
    desc, dq, _, stream = _marshal(q, k, v, eta, *Wm, extra, chunk or longest, 0, use_muon, ns_steps,
                                   None if out is None else out[0], None, stream,
                                   FW_LINEAR if linear else FW_SWIGLU, need_workspace=False)
    if not dout.is_cuda or not dout.is_contiguous():
        raise LactError(-1, "dout must be a contiguous device tensor")
    if workspace is None:
        nb = backward_schedule_workspace_bytes(desc, schedule, mom)
        workspace = torch.empty(max(nb, 1), dtype=torch.uint8, device=q.device)
    if out is None:
        head = (dq, torch.empty_like(k), torch.empty_like(v), torch.empty_like(eta))
        dW = tuple(torch.empty_like(w) for w in W)
        dbeta = torch.empty_like(beta) if mom else None
        dM = tuple(torch.empty_like(w) for w in W) if mom else (None,) * len(W)
    else:
        head = tuple(out[:4])
        dbeta = out[4] if mom else None
        dW = tuple(out[5] if mom else out[4])
        dM = tuple(out[6]) if mom else (None,) * len(W)
    Ms = tuple(M) if mom else (None,) * len(W)
    pad = lambda t: tuple(t) + (None,) * (3 - len(t))
    args = ([_ptr(q), _ptr(k), _ptr(v), _ptr(eta), _ptr(beta)] + [_ptr(w) for w in pad(W)] +
            [_ptr(m) for m in pad(Ms)] + [_ptr(dout)] + [_ptr(t) for t in pad(dWf)] + [_ptr(t) for t in pad(dMf)] +
            [_ptr(t) for t in head] + [_ptr(dbeta)] + [_ptr(t) for t in pad(dW)] + [_ptr(t) for t in pad(dM)])
    rc = lib().lact_backward_schedule(ctypes.byref(desc), segs, ctypes.c_int64(len(schedule)), *args, _ptr(workspace),
                                      ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                                      ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    if linear:
        dW, dM = dW[0], dM[0]
    if mom:
        return head + (dbeta, dW, dM)
    return head + (dW,)


def prologue(qkv, lr_raw, lr_bias, beta_raw=None, n_kv=None, out=None, stream=None):
    """The layer's prologue (lact_prologue): qkv [B, L, 3, H, d] (bf16 or fp32),
    lr_raw [B, L, H] or [B, L, H, 3] fp32, beta_raw [B, L, H] fp32 or None.
    Returns (q [B, H, L, d], k, v [B, H, n_kv, d], eta [B, H, n_kv(, 3)], beta
    [B, H, n_kv] or None); ``out`` may hold preallocated tensors of those shapes.
    """
    import torch
    if qkv.dim() != 5 or qkv.shape[2] != 3:
        raise LactError(-1, "qkv must be [B, L, 3, H, d]")
    B, L, _, H, d = qkv.shape
    n_kv = L if n_kv is None else int(n_kv)
    lr3 = lr_raw.dim() == 4
    if lr_raw.shape[:3] != (B, L, H) or (lr3 and lr_raw.shape[3] != 3):
        raise LactError(-1, "lr_raw must be [B, L, H] or [B, L, H, 3]")
    if beta_raw is not None and beta_raw.shape != (B, L, H):
        raise LactError(-1, "beta_raw must be [B, L, H]")
    for t, name in ((qkv, "qkv"), (lr_raw, "lr_raw"), (beta_raw, "beta_raw")):
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise LactError(-1, f"{name} must be a contiguous device tensor")
    if lr_raw.dtype != torch.float32 or (beta_raw is not None and beta_raw.dtype != torch.float32):
        raise LactError(-1, "lr_raw and beta_raw are fp32")
    io = IO_BF16 if qkv.dtype == torch.bfloat16 else IO_FP32 if qkv.dtype == torch.float32 else None
    if io is None:
        raise LactError(-1, f"unsupported qkv dtype {qkv.dtype}")
    if out is None:
        e = lambda *sh, dt=qkv.dtype: torch.empty(*sh, dtype=dt, device=qkv.device)
        out = (e(B, H, L, d), e(B, H, n_kv, d), e(B, H, n_kv, d),
               e(B, H, n_kv, *((3,) if lr3 else ()), dt=torch.float32),
               e(B, H, n_kv, dt=torch.float32) if beta_raw is not None else None)
    q, k, v, eta, beta = out
    desc = make_desc(B, H, d, d, n_kv, L, 1, 0, False, 0, io, lr3)   # h unused: any valid value
    if stream is None:
        stream = torch.cuda.current_stream(qkv.device).cuda_stream
    rc = lib().lact_prologue(ctypes.byref(desc), _ptr(qkv), _ptr(lr_raw), ctypes.c_float(lr_bias), _ptr(beta_raw),
                             _ptr(q), _ptr(k), _ptr(v), _ptr(eta), _ptr(beta), ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    return q, k, v, eta, beta


def rmsnorm_out(o, weight=None, eps=1e-6, out=None, stream=None):
    """Per-head RMSNorm of the path output (lact_rmsnorm_out): o [B, H, L, d]
    -> y [B, L, H, d]; weight [H, d] fp32 or None."""
    import torch
    if o.dim() != 4:
        raise LactError(-1, "o must be [B, H, L, d]")
    B, H, L, d = o.shape
    if not o.is_cuda or not o.is_contiguous():
        raise LactError(-1, "o must be a contiguous device tensor")
    if weight is not None and (weight.shape != (H, d) or weight.dtype != torch.float32 or not weight.is_contiguous()):
        raise LactError(-1, "weight must be a contiguous fp32 [H, d] tensor")
    io = IO_BF16 if o.dtype == torch.bfloat16 else IO_FP32 if o.dtype == torch.float32 else None
    if io is None:
        raise LactError(-1, f"unsupported o dtype {o.dtype}")
    y = torch.empty(B, L, H, d, dtype=o.dtype, device=o.device) if out is None else out
    desc = make_desc(B, H, d, d, 0, L, 1, 0, False, 0, io)
    if stream is None:
        stream = torch.cuda.current_stream(o.device).cuda_stream
    rc = lib().lact_rmsnorm_out(ctypes.byref(desc), _ptr(o), _ptr(weight), ctypes.c_float(eps), _ptr(y),
                                ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    return y


def prologue_backward(qkv, lr_raw, lr_bias, beta_raw, dq, dk, dv, deta, dbeta=None, out=None, stream=None):
    """Reverse of prologue() (lact_prologue_backward): the cotangents (dqkv
    [B, L, 3, H, d], dlr_raw like lr_raw, dbeta_raw [B, L, H] or None) of the
    prologue's inputs given those of its outputs (dq [B, H, L, d], dk, dv
    [B, H, n_kv, d], deta like eta, dbeta [B, H, n_kv] or None)."""
    import torch
    if qkv.dim() != 5 or qkv.shape[2] != 3:
        raise LactError(-1, "qkv must be [B, L, 3, H, d]")
    B, L, _, H, d = qkv.shape
    n_kv = dk.shape[-2]
    lr3 = lr_raw.dim() == 4
    if dq.shape != (B, H, L, d) or dk.shape != (B, H, n_kv, d) or dv.shape != dk.shape:
        raise LactError(-1, "dq must be [B, H, L, d], dk and dv [B, H, n_kv, d]")
    if deta.shape != (B, H, n_kv, *((3,) if lr3 else ())):
        raise LactError(-1, "deta must be shaped like eta")
    if (beta_raw is None) != (dbeta is None):
        raise LactError(-1, "pass beta_raw and dbeta together")
    for t in (qkv, lr_raw, beta_raw, dq, dk, dv, deta, dbeta):
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise LactError(-1, "inputs must be contiguous device tensors")
    if any(t.dtype != qkv.dtype for t in (dq, dk, dv)):
        raise LactError(-1, "dq, dk, dv must have qkv's dtype")
    io = IO_BF16 if qkv.dtype == torch.bfloat16 else IO_FP32 if qkv.dtype == torch.float32 else None
    if io is None:
        raise LactError(-1, f"unsupported qkv dtype {qkv.dtype}")
    if out is None:
        out = (torch.empty_like(qkv), torch.empty_like(lr_raw),
               torch.empty_like(beta_raw) if beta_raw is not None else None)
    dqkv, dlr, dbr = out
    desc = make_desc(B, H, d, d, n_kv, L, 1, 0, False, 0, io, lr3)   # h unused: any valid value
    if stream is None:
        stream = torch.cuda.current_stream(qkv.device).cuda_stream
    rc = lib().lact_prologue_backward(ctypes.byref(desc), _ptr(qkv), _ptr(lr_raw), ctypes.c_float(lr_bias),
                                      _ptr(beta_raw), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(deta), _ptr(dbeta),
                                      _ptr(dqkv), _ptr(dlr), _ptr(dbr), ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    return dqkv, dlr, dbr


def rmsnorm_out_backward(o, dy, weight=None, eps=1e-6, with_dweight=True, out=None, workspace=None, stream=None):
    """Reverse of rmsnorm_out() (lact_rmsnorm_out_backward): from dy [B, L,
    H, d], returns (d_o [B, H, L, d], dweight [H, d] or None; dweight only
    with a weight and with_dweight)."""
    import torch
    if o.dim() != 4:
        raise LactError(-1, "o must be [B, H, L, d]")
    B, H, L, d = o.shape
    if dy.shape != (B, L, H, d) or dy.dtype != o.dtype:
        raise LactError(-1, "dy must be [B, L, H, d] of o's dtype")
    for t in (o, dy, weight):
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise LactError(-1, "inputs must be contiguous device tensors")
    io = IO_BF16 if o.dtype == torch.bfloat16 else IO_FP32 if o.dtype == torch.float32 else None
    if io is None:
        raise LactError(-1, f"unsupported o dtype {o.dtype}")
    want_dw = weight is not None and with_dweight
    if out is None:
        out = (torch.empty_like(o), torch.empty_like(weight) if want_dw else None)
    d_o, dw = out
    desc = make_desc(B, H, d, d, 0, L, 1, 0, False, 0, io)
    if workspace is None and want_dw:
        err = ctypes.c_int(0)
        nb = lib().lact_rmsnorm_out_backward_workspace_bytes(ctypes.byref(desc), 1, ctypes.byref(err))
        if err.value:
            _raise(err.value)
        workspace = torch.empty(max(int(nb), 1), dtype=torch.uint8, device=o.device)
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if stream is None:
        stream = torch.cuda.current_stream(o.device).cuda_stream
    rc = lib().lact_rmsnorm_out_backward(ctypes.byref(desc), _ptr(o), _ptr(weight), ctypes.c_float(eps), _ptr(dy),
                                         _ptr(d_o), _ptr(dw), _ptr(workspace), ctypes.c_size_t(nbytes),
                                         ctypes.c_void_p(stream))
    if rc:
        _raise(rc)
    return d_o, dw


# ---- the attention half of a hybrid layer (strided tensors are taken as they lie)

# These calls can be as short as a kernel launch, which the host then cannot
# keep up with: their checks read each property of a tensor once, and
# descriptors and views go to the library as packed bytes. One token's norm and
# rotation takes 14.8 us with ctypes structures, 12.1 so (the C call 4 of them).

_pack_view = struct.Struct("Pqqq").pack
_pack_rope = struct.Struct("4i2q4ifi").pack
_pack_attn = struct.Struct("4i6qfi").pack
_pack_paged = struct.Struct("4i2q2i2qfi").pack
_pack_prefix = struct.Struct("2i3P").pack
_packed = {}


def _fn(name):
    """The entry point taking descriptors and views as bytes."""
    f = _packed.get(name)
    if f is None:
        L = lib()
        f = L[name]      # a function object of its own: the attribute keeps its prototype
        f.restype = getattr(L, name).restype
        f.argtypes = [ctypes.c_char_p if issubclass(t, ctypes._Pointer) and issubclass(t._type_, ctypes.Structure) else t
                      for t in getattr(L, name).argtypes]
        _packed[name] = f
    return f


def _pack(pack, *fields):
    try:
        return pack(*fields)
    except struct.error as e:
        raise LactError(-1, f"an argument is out of range: {e}") from None


def _refuse(t, name, shape, dtype, dev):
    if t.shape != shape:
        raise LactError(-1, f"{name} must be {list(shape)}, not {list(t.shape)}")
    if t.dtype != dtype:
        raise LactError(-1, f"{name} must be {dtype}, not {t.dtype}")
    if dev < 0 or t.get_device() != dev:
        raise LactError(-1, f"{name} must be a device tensor, on the first one's device")
    raise LactError(-1, f"{name}'s last dimension must be contiguous")


def _view(t, name, shape, dtype, dev):
    """lact_view of a tensor [batch, head, token, d] of that shape, type and
    device, vectors consecutive."""
    if t.shape == shape and t.dtype is dtype and t.get_device() == dev >= 0:
        s = t.stride()
        if s[3] == 1:
            return _pack_view(t.data_ptr(), s[0], s[1], s[2])
    _refuse(t, name, shape, dtype, dev)


def _view_t(t, name, shape, dtype, dev):
    """The same of a tensor [batch, token, head, d]."""
    if t.shape == shape and t.dtype is dtype and t.get_device() == dev >= 0:
        s = t.stride()
        if s[3] == 1:
            return _pack_view(t.data_ptr(), s[0], s[2], s[1])
    _refuse(t, name, shape, dtype, dev)


def _view_n(t, name, shape, dtype, dev):
    """The same of a tensor [token, head, d]."""
    if t.shape == shape and t.dtype is dtype and t.get_device() == dev >= 0:
        s = t.stride()
        if s[2] == 1:
            return _pack_view(t.data_ptr(), 0, s[1], s[0])
    _refuse(t, name, shape, dtype, dev)


def _view_s(t, name, shape, dtype, dev):
    """The same of scales [page, slot, head], one element each."""
    if t is not None and t.shape == shape and t.dtype is dtype and t.get_device() == dev >= 0:
        s = t.stride()
        return _pack_view(t.data_ptr(), s[0], s[2], s[1])
    raise LactError(-1, f"{name} must be a {dtype} tensor {list(shape)}, on the first one's device")


def _aux(t, name, shape, dtype, dev):
    """The address of a contiguous tensor of that shape, type and device, or None."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        raise LactError(-1, f"{name} must be a contiguous {dtype} tensor {list(shape)} on device {dev}")
    return t.data_ptr()


def _io(t, name, torch):
    if t.dtype is torch.bfloat16:
        return IO_BF16
    if t.dtype is torch.float32:
        return IO_FP32
    raise LactError(-1, f"unsupported {name} dtype {t.dtype}")


def _call(name, dev, stream, torch, *args):
    """The entry point on device `dev` and its current stream (or `stream`)."""
    C = torch._C
    f = _packed.get(name) or _fn(name)
    if C._cuda_getDevice() == dev:
        rc = f(*args, C._cuda_getCurrentRawStream(dev) if stream is None else stream)
    else:
        with torch.cuda.device(dev):
            rc = f(*args, C._cuda_getCurrentRawStream(dev) if stream is None else stream)
    if rc:
        _raise(rc)


def _new(like, shape, stream, torch, dtype=None):
    """An uninitialised tensor of like's device, from the memory of the stream
    that works on it."""
    if stream is None:
        return like.new_empty(shape) if dtype is None else like.new_empty(shape, dtype=dtype)
    dev = like.device
    s = torch.cuda.ExternalStream(stream, device=dev) if stream else torch.cuda.default_stream(dev)
    with torch.cuda.stream(s):
        return like.new_empty(shape, dtype=dtype or like.dtype)


def _workspace(name, desc, workspace, like, stream, torch, *more):
    """(tensor that stays alive, address, bytes) of the caller's workspace, or of
    a new one of the size that the call needs (0 too where the descriptor is
    refused, which the call itself then says)."""
    if workspace is None:
        n = (_packed.get(name) or _fn(name))(desc, *more, None)
        if not n:
            return None, None, 0
        workspace = _new(like, n, stream, torch, torch.uint8)
        return workspace, workspace.data_ptr(), n
    if workspace.device != like.device or not workspace.is_contiguous():
        raise LactError(-1, f"workspace must be a contiguous tensor on {like.device}")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _rope_args(q, k, wq, wk, inv_freq, positions, pos0, eps, interleaved, torch):
    """Shapes, device and the first arguments of the norm and rotation and its reverse."""
    if q.dim() != 4 or k.dim() != 4:
        raise LactError(-1, "q must be [B, n, H, d] and k [B, n, Hkv, d]")
    B, n, H, d = q.shape
    Hkv = k.shape[2]
    dt, dev = q.dtype, q.get_device()
    io = _io(q, "q", torch)
    qv = _view_t(q, "q", (B, n, H, d), dt, dev)
    kv = _view_t(k, "k", (B, n, Hkv, d), dt, dev)
    per_head = (wq is not None and wq.dim() == 2) or (wk is not None and wk.dim() == 2)
    wqp = _aux(wq, "wq", (H, d) if per_head else (d,), torch.float32, dev)
    wkp = _aux(wk, "wk", (Hkv, d) if per_head else (d,), torch.float32, dev)
    rot, ip = 0, None
    if inv_freq is not None:
        if inv_freq.dim() != 1:
            raise LactError(-1, "inv_freq must be [rot / 2]")
        half = inv_freq.shape[0]
        rot = 2 * half
        if half:
            ip = _aux(inv_freq, "inv_freq", (half,), torch.float64, dev)
    desc = _pack(_pack_rope, B, H, Hkv, d, n, int(pos0), rot, 1 if interleaved else 0, 1 if per_head else 0, io,
                 float(eps), 0)
    return (B, n, H, Hkv, d), dt, dev, (desc, qv, kv, wqp, wkp, ip, _aux(positions, "positions", (B, n), torch.int32, dev))


def qk_norm_rope(q, k, wq=None, wk=None, inv_freq=None, *, positions=None, pos0=0, eps=1e-6, interleaved=False,
                 out=None, stream=None):
    """RMS norm of queries and keys for each head with the position rotation
    (lact_qk_norm_rope): q [B, n, H, d], k [B, n, Hkv, d] (bf16 or fp32; any
    strides with contiguous vectors, such as parts of a fused projection); wq,
    wk fp32 [d], or [H, d] and [Hkv, d], or None; inv_freq fp64 [rot / 2]
    radians a position, or None (norm only); positions int32 [B, n], or None
    (pos0 + token). Returns (qn [B, H, n, d], kn [B, Hkv, n, d]), into ``out``
    (two tensors of those shapes, any strides) when it is given."""
    import torch
    (B, n, H, Hkv, d), dt, dev, args = _rope_args(q, k, wq, wk, inv_freq, positions, pos0, eps, interleaved, torch)
    qn, kn = (_new(q, (B, H, n, d), stream, torch), _new(q, (B, Hkv, n, d), stream, torch)) if out is None else out
    _call("lact_qk_norm_rope", dev, stream, torch, *args, _view(qn, "qn", (B, H, n, d), dt, dev),
          _view(kn, "kn", (B, Hkv, n, d), dt, dev))
    return qn, kn


def qk_norm_rope_backward(q, k, dqn, dkn, wq=None, wk=None, inv_freq=None, *, positions=None, pos0=0, eps=1e-6,
                          interleaved=False, with_dweight=True, out=None, workspace=None, stream=None):
    """Reverse of qk_norm_rope() (lact_qk_norm_rope_backward): from the
    cotangents dqn [B, H, n, d], dkn [B, Hkv, n, d], returns (dq [B, n, H, d],
    dk [B, n, Hkv, d], dwq, dwk); the weights' cotangents are None without a
    weight or with_dweight. ``out`` may hold that tuple."""
    import torch
    (B, n, H, Hkv, d), dt, dev, args = _rope_args(q, k, wq, wk, inv_freq, positions, pos0, eps, interleaved, torch)
    if out is None:
        dw = [_new(w, w.shape, stream, torch) if w is not None and with_dweight else None for w in (wq, wk)]
        out = (_new(q, (B, n, H, d), stream, torch), _new(q, (B, n, Hkv, d), stream, torch), *dw)
    dq, dk, dwq, dwk = out
    dwp = []
    for t, w, name in ((dwq, wq, "dwq"), (dwk, wk, "dwk")):
        if t is not None and w is None:
            raise LactError(-1, f"{name} needs its weight")
        dwp.append(None if t is None else _aux(t, name, w.shape, torch.float32, dev))
    wp, nb = None, 0
    if dwq is not None or dwk is not None:
        workspace, wp, nb = _workspace("lact_qk_norm_rope_backward_workspace_bytes", args[0], workspace, q, stream, torch)
    _call("lact_qk_norm_rope_backward", dev, stream, torch, *args, _view(dqn, "dqn", (B, H, n, d), dt, dev),
          _view(dkn, "dkn", (B, Hkv, n, d), dt, dev), _view_t(dq, "dq", (B, n, H, d), dt, dev),
          _view_t(dk, "dk", (B, n, Hkv, d), dt, dev), *dwp, wp, nb)
    return dq, dk, dwq, dwk


def _attn_args(q, k, v, window, sinks, lookahead, lengths, scale, q_start, torch):
    """Shapes of q and of k and v, type, device and the first arguments of
    window attention and its reverse."""
    if q.dim() != 4 or k.dim() != 4:
        raise LactError(-1, "q must be [B, H, n_q, d], k and v [B, Hkv, n_kv, d]")
    sq = B, H, n_q, d = q.shape
    Hkv, n_kv = k.shape[1], k.shape[2]
    sk = (B, Hkv, n_kv, d)
    dt, dev = q.dtype, q.get_device()
    desc = _pack(_pack_attn, B, H, Hkv, d, n_q, n_kv, n_kv - n_q if q_start is None else int(q_start),
                 -1 if window is None else int(window), -1 if lookahead is None else int(lookahead), int(sinks),
                 d ** -0.5 if scale is None else float(scale), _io(q, "q", torch))
    return sq, sk, dt, dev, (desc, _view(q, "q", sq, dt, dev), _view(k, "k", sk, dt, dev), _view(v, "v", sk, dt, dev)), \
        _aux(lengths, "lengths", (B,), torch.int32, dev)


def window_attention(q, k, v, *, window=None, sinks=0, lookahead=0, lengths=None, scale=None, q_start=None,
                     with_lse=False, out=None, stream=None):
    """Softmax attention with a sliding window and first tokens that stay
    visible (lact_window_attention): q [B, H, n_q, d], k, v [B, Hkv, n_kv, d]
    (bf16 or fp32, any strides with contiguous vectors). Query i stands at
    position p = q_start + i (q_start: n_kv - n_q) and sees key j when
    j <= p + lookahead and (j > p - window or j < sinks), both below
    lengths[b] (int32 [B], or None: n_kv). None for window or lookahead: no
    bound. scale: d ** -0.5. A query that sees nothing gives 0 (lse -inf).
    Returns o like q, or (o, lse fp32 [B, H, n_q]) with_lse; ``out`` may hold o,
    or that pair."""
    import torch
    sq, _, dt, dev, args, lp = _attn_args(q, k, v, window, sinks, lookahead, lengths, scale, q_start, torch)
    if out is None:
        o = _new(q, sq, stream, torch)
        lse = _new(q, sq[:3], stream, torch, torch.float32) if with_lse else None
    else:
        o, lse = out if with_lse else (out, None)
    _call("lact_window_attention", dev, stream, torch, *args, lp, _view(o, "o", sq, dt, dev),
          _aux(lse, "lse", sq[:3], torch.float32, dev))
    return (o, lse) if with_lse else o


def window_attention_backward(q, k, v, o, lse, dout, *, window=None, sinks=0, lookahead=0, lengths=None, scale=None,
                              q_start=None, out=None, workspace=None, stream=None):
    """Reverse of window_attention() (lact_window_attention_backward): from its
    o and lse and the cotangent dout of o, returns (dq, dk, dv), written into
    ``out`` (that tuple) when it is given."""
    import torch
    sq, sk, dt, dev, args, lp = _attn_args(q, k, v, window, sinks, lookahead, lengths, scale, q_start, torch)
    if lse is None:
        raise LactError(-1, "lse of the forward is needed")
    dq, dk, dv = tuple(_new(q, x, stream, torch) for x in (sq, sk, sk)) if out is None else out
    workspace, wp, nb = _workspace("lact_window_attention_backward_workspace_bytes", args[0], workspace, q, stream, torch)
    _call("lact_window_attention_backward", dev, stream, torch, *args, _view(o, "o", sq, dt, dev),
          _aux(lse, "lse", sq[:3], torch.float32, dev), _view(dout, "dout", sq, dt, dev), lp,
          _view(dq, "dq", sq, dt, dev), _view(dk, "dk", sk, dt, dev), _view(dv, "dv", sk, dt, dev), wp, nb)
    return dq, dk, dv


def _paged_args(x, H, k_cache, v_cache, table, lens, cu_new, window, sinks, scale, torch):
    """The descriptor, the caches' views and the addresses of the tables."""
    if k_cache.dim() != 4 or table.dim() != 2:
        raise LactError(-1, "new tokens are [n_new, heads, d], caches [pages, page, Hkv, d], table [B, max_pages]")
    sc = pages, page, Hkv, d = k_cache.shape
    B, max_pages = table.shape
    dt, dev, i32 = x.dtype, x.get_device(), torch.int32
    desc = _pack(_pack_paged, B, H, Hkv, d, x.shape[0], pages, page, max_pages, -1 if window is None else int(window),
                 int(sinks), d ** -0.5 if scale is None else float(scale), _io(x, "new tokens", torch))
    return d, dt, dev, desc, (_view_t(k_cache, "k_cache", sc, dt, dev), _view_t(v_cache, "v_cache", sc, dt, dev),
                              _aux(table, "table", (B, max_pages), i32, dev), _aux(lens, "lens", (B,), i32, dev),
                              _aux(cu_new, "cu_new", (B + 1,), i32, dev))


def paged_append(k, v, k_cache, v_cache, table, lens, cu_new, *, stream=None):
    """Writes new keys and values k, v [n_new, Hkv, d] into the pages of a
    cache (lact_paged_append): k_cache, v_cache [pages, page, Hkv, d] (in
    place), table int32 [B, max_pages], lens int32 [B] (tokens of a sequence,
    the new ones included), cu_new int32 [B + 1] (rows of a sequence's new
    tokens, which are its last positions)."""
    import torch
    if k.dim() != 3 or k_cache.dim() != 4:
        raise LactError(-1, "k and v are [n_new, Hkv, d], caches [pages, page, Hkv, d]")
    Hkv = k_cache.shape[2]
    d, dt, dev, desc, tail = _paged_args(k, Hkv, k_cache, v_cache, table, lens, cu_new, None, 0, 1.0, torch)
    s = (k.shape[0], Hkv, d)
    _call("lact_paged_append", dev, stream, torch, desc, _view_n(k, "k", s, dt, dev), _view_n(v, "v", s, dt, dev), *tail)


def paged_attention(q, k_cache, v_cache, table, lens, cu_new, *, window=None, sinks=0, scale=None, out=None,
                    workspace=None, stream=None):
    """Causal attention of new tokens q [n_new, H, d] over a cache of pages
    (lact_paged_attention): the cache, table, lens and cu_new of
    paged_append(), window and sinks of window_attention(). Returns o like q
    (rows of no sequence are left as they were), into ``out`` when given."""
    import torch
    if q.dim() != 3:
        raise LactError(-1, "q must be [n_new, H, d]")
    T, H, _ = q.shape
    d, dt, dev, desc, tail = _paged_args(q, H, k_cache, v_cache, table, lens, cu_new, window, sinks, scale, torch)
    s = (T, H, d)
    qv = _view_n(q, "q", s, dt, dev)
    o = _new(q, s, stream, torch) if out is None else out
    workspace, wp, nb = _workspace("lact_paged_attention_workspace_bytes", desc, workspace, q, stream, torch)
    _call("lact_paged_attention", dev, stream, torch, desc, qv, *tail, _view_n(o, "o", s, dt, dev), wp, nb)
    return o


def _code_args(x, H, n, dtype, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new, window, sinks, scale, torch):
    """As _paged_args() for a cache of e4m3 numbers: x is a tensor of the call's device, n its new tokens."""
    sc, st = k_cache.shape, table.shape
    if len(sc) != 4 or len(st) != 2:
        raise LactError(-1, "new tokens are [n_new, heads, d], caches [pages, page, Hkv, d], table [B, max_pages]")
    pages, page, Hkv, d = sc
    B, max_pages = st
    dev, i32, u8, f8 = x.get_device(), torch.int32, torch.uint8, torch.float8_e4m3fn
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise LactError(-1, f"unsupported dtype {dtype}")
    desc = _pack(_pack_paged, B, H, Hkv, d, n, pages, page, max_pages, -1 if window is None else int(window),
                 int(sinks), d ** -0.5 if scale is None else float(scale), IO_BF16 if dtype is torch.bfloat16 else IO_FP32)
    return d, dev, desc, (_view_t(k_cache, "k_cache", sc, f8, dev), _view_t(v_cache, "v_cache", sc, f8, dev),
                          _view_s(k_scale, "k_scale", sc[:3], u8, dev), _view_s(v_scale, "v_scale", sc[:3], u8, dev),
                          _aux(table, "table", st, i32, dev), _aux(lens, "lens", (B,), i32, dev),
                          _aux(cu_new, "cu_new", (B + 1,), i32, dev))


def paged_append_e4m3(k, v, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new, *, stream=None):
    """paged_append() into a cache in 8 bits (lact_paged_append_e4m3): k_cache,
    v_cache float8_e4m3fn [pages, page, Hkv, d] (d a multiple of 16) and
    k_scale, v_scale uint8 [pages, page, Hkv], in place. A vector is held as
    numbers c and a byte x, and stands for c 2^(x - 127), the smallest power of
    two that takes its largest element."""
    import torch
    if k.dim() != 3 or k_cache.dim() != 4:
        raise LactError(-1, "k and v are [n_new, Hkv, d], caches [pages, page, Hkv, d]")
    n, Hkv, dt = k.shape[0], k_cache.shape[2], k.dtype
    d, dev, desc, tail = _code_args(k, Hkv, n, dt, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new, None, 0, 1.0,
                                    torch)
    s = (n, Hkv, d)
    _call("lact_paged_append_e4m3", dev, stream, torch, desc, _view_n(k, "k", s, dt, dev), _view_n(v, "v", s, dt, dev),
          *tail)


def paged_read_e4m3(k_cache, v_cache, k_scale, v_scale, table, lens, cu_new, n_new, *, dtype=None, out=None, stream=None):
    """What the cache of paged_append_e4m3() holds for the last positions of
    sequences (lact_paged_read_e4m3): returns (k, v) [n_new, Hkv, d] of
    ``dtype`` (bf16 or fp32; bf16), exactly, where rows cu_new[b] ..
    cu_new[b + 1] - 1 are sequence b's last positions (with cu_new the sums of
    lens: whole sequences); rows of no sequence are left as they were,
    positions that hold nothing are zeros. ``out`` may hold that pair."""
    import torch
    if k_cache.dim() != 4:
        raise LactError(-1, "caches are [pages, page, Hkv, d]")
    Hkv = k_cache.shape[2]
    dt = dtype if dtype is not None else torch.bfloat16 if out is None else out[0].dtype
    n = int(n_new)
    d, dev, desc, tail = _code_args(k_cache, Hkv, n, dt, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new, None, 0,
                                    1.0, torch)
    s = (n, Hkv, d)
    if n < 0:
        raise LactError(-1, "n_new must not be negative")
    k, v = (_new(k_cache, s, stream, torch, dt), _new(k_cache, s, stream, torch, dt)) if out is None else out
    _call("lact_paged_read_e4m3", dev, stream, torch, desc, *tail, _view_n(k, "k", s, dt, dev),
          _view_n(v, "v", s, dt, dev))
    return k, v


def paged_attention_e4m3(q, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new, *, window=None, sinks=0, scale=None,
                         out=None, workspace=None, stream=None):
    """paged_attention() over the cache of paged_append_e4m3()
    (lact_paged_attention_e4m3)."""
    import torch
    if q.dim() != 3:
        raise LactError(-1, "q must be [n_new, H, d]")
    T, H, _ = q.shape
    dt = q.dtype
    d, dev, desc, tail = _code_args(q, H, T, dt, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new, window, sinks,
                                    scale, torch)
    s = (T, H, d)
    qv = _view_n(q, "q", s, dt, dev)
    o = _new(q, s, stream, torch) if out is None else out
    workspace, wp, nb = _workspace("lact_paged_attention_e4m3_workspace_bytes", desc, workspace, q, stream, torch)
    _call("lact_paged_attention_e4m3", dev, stream, torch, desc, qv, *tail, _view_n(o, "o", s, dt, dev), wp, nb)
    return o


def paged_prefix_attention(q, k_cache, v_cache, prefix_table, prefix_lens, cu_seq, table, lens, cu_new, *, k_scale=None,
                           v_scale=None, window=None, sinks=0, scale=None, out=None, workspace=None, stream=None):
    """paged_attention() of sequences that share prefixes, each read once for
    its group (lact_paged_prefix_attention): group g is sequences cu_seq[g] ..
    cu_seq[g + 1] - 1 (int32 [groups + 1]), its prefix the first prefix_lens[g]
    (int32 [groups]) positions on pages prefix_table[g] (int32 [groups,
    max_pages]) of the same cache. table and lens of a sequence begin at the
    prefix's end; window and sinks go by the positions from the prefix's
    start. With k_scale and v_scale the cache is one of paged_append_e4m3()."""
    import torch
    if q.dim() != 3 or prefix_table.dim() != 2:
        raise LactError(-1, "q must be [n_new, H, d], prefix_table [groups, max_pages]")
    T, H, _ = q.shape
    dt, i32 = q.dtype, torch.int32
    if (k_scale is None) != (v_scale is None):
        raise LactError(-1, "k_scale and v_scale are given both or not at all")
    if k_scale is None:
        d, _, dev, desc, tail = _paged_args(q, H, k_cache, v_cache, table, lens, cu_new, window, sinks, scale, torch)
        tail = (*tail[:2], None, None, *tail[2:])
    else:
        d, dev, desc, tail = _code_args(q, H, T, dt, k_cache, v_cache, k_scale, v_scale, table, lens, cu_new, window,
                                        sinks, scale, torch)
    groups, width = prefix_table.shape
    prefix = _pack(_pack_prefix, groups, width, _aux(prefix_table, "prefix_table", (groups, width), i32, dev) or 0,
                   _aux(prefix_lens, "prefix_lens", (groups,), i32, dev) or 0, _aux(cu_seq, "cu_seq", (groups + 1,), i32, dev) or 0)
    s = (T, H, d)
    qv = _view_n(q, "q", s, dt, dev)
    o = _new(q, s, stream, torch) if out is None else out
    workspace, wp, nb = _workspace("lact_paged_prefix_attention_workspace_bytes", desc, workspace, q, stream, torch, prefix,
                                   int(k_scale is not None))
    _call("lact_paged_prefix_attention", dev, stream, torch, desc, prefix, qv, *tail, _view_n(o, "o", s, dt, dev), wp, nb)
    return o


def timing_enable(on: bool = True):
    lib().lact_timing_enable(int(on))


def timing_reset():
    lib().lact_timing_reset()


def timing_read(kclass: int):
    n, ms, fl = ctypes.c_int64(0), ctypes.c_double(0), ctypes.c_double(0)
    rc = lib().lact_timing_read(int(kclass), ctypes.byref(n), ctypes.byref(ms), ctypes.byref(fl))
    if rc:
        _raise(rc)
    return int(n.value), float(ms.value), float(fl.value)
