"""ctypes binding of include/moe.h.  Argument marshalling only.

Every function takes torch CUDA tensors (device memory) and forwards their data pointers,
the sizes and torch's current HIP stream to the C entry point of the same name.  There is
no fallback: if libmoe_mi355x.so is missing or a call returns an error code, MoeError is
raised.

A call whose arguments are all as they should be is checked and made by csrc/marshal.cpp, which
takes the host less than half of the time (figures there); any other is left to the checks
here, and all are where that extension was not built for this Python and torch.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
import sys
import warnings

MOE_F32, MOE_BF16 = 0, 1
GATE_SOFTMAX_RENORM, GATE_SIGMOID_RENORM, GATE_SOFTMAX = 0, 1, 2
WS_DISPATCH, WS_EXPERT_FWD, WS_EXPERT_BWD, WS_ROUTER, WS_BLOCK_NORM, WS_MX4_EXPERT_FWD = 0, 1, 2, 3, 4, 5
WS_LAYER_NORM, WS_LINEAR_FWD, WS_LINEAR_BWD = 6, 7, 8
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = 0, 1, 2, 3, 4
ACTIVATIONS = dict(none=ACT_NONE, relu=ACT_RELU, gelu=ACT_GELU, gelu_tanh=ACT_GELU_TANH, silu=ACT_SILU)

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None
_MARSHAL = None

EXPORTS = ("moe_route", "moe_dispatch", "moe_dispatch_static", "moe_expert_fwd", "moe_expert_bwd", "moe_combine",
           "moe_router_fwd", "moe_combine_bwd", "moe_gate_bwd", "moe_router_bwd",
           "moe_block_norm_fwd", "moe_block_norm_bwd", "moe_layer_norm_fwd", "moe_layer_norm_bwd", "moe_linear_fwd", "moe_linear_bwd",
           "moe_mx4_quantize", "moe_mx4_dequantize", "moe_mx4_expert_fwd",
           "moe_profile_enable", "moe_profile_read", "moe_profile_stats", "moe_probe_mfma_bf16", "moe_probe_mfma_fed_bf16",
           "moe_probe_copy", "moe_probe_stream",
           "moe_workspace_bytes", "moe_error_string")
# what csrc/marshal.cpp calls, in its order
_MARSHALLED = ("moe_route", "moe_dispatch", "moe_dispatch_static", "moe_expert_fwd", "moe_expert_bwd", "moe_combine", "moe_router_fwd",
               "moe_combine_bwd", "moe_gate_bwd", "moe_router_bwd", "moe_block_norm_fwd", "moe_block_norm_bwd", "moe_mx4_quantize",
               "moe_mx4_dequantize", "moe_mx4_expert_fwd", "moe_layer_norm_fwd", "moe_layer_norm_bwd", "moe_linear_fwd", "moe_linear_bwd")


class MoeError(RuntimeError):
    pass


def lib_path() -> str:
    return os.path.join(_HERE, "libmoe_mi355x.so")


def load_library():
    """Load the HIP library (built by __graft_entry__.build() / csrc/build.sh)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise MoeError(f"{path} not found: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    lib = ctypes.CDLL(path)
    c_int, c_void_p, c_size_t = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    lib.moe_route.restype = c_int
    lib.moe_route.argtypes = [c_void_p, c_int, c_int, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.moe_dispatch.restype = c_int
    lib.moe_dispatch.argtypes = [c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_int, c_int, c_void_p,
                                 c_void_p, c_void_p, c_int, c_void_p, c_int, c_void_p, c_size_t, c_void_p]
    lib.moe_dispatch_static.restype = c_int
    lib.moe_dispatch_static.argtypes = [c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_int, c_int, c_void_p,
                                        c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_void_p]
    lib.moe_expert_fwd.restype = c_int
    lib.moe_expert_fwd.argtypes = [c_void_p, c_int, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.moe_expert_bwd.restype = c_int
    lib.moe_expert_bwd.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, c_void_p,
                                   c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int,
                                   c_void_p, c_size_t, c_void_p]
    lib.moe_combine.restype = c_int
    lib.moe_combine.argtypes = [c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.moe_router_fwd.restype = c_int
    lib.moe_router_fwd.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.moe_combine_bwd.restype = c_int
    lib.moe_combine_bwd.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p,
                                    c_void_p, c_void_p]
    lib.moe_gate_bwd.restype = c_int
    lib.moe_gate_bwd.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_void_p]
    lib.moe_router_bwd.restype = c_int
    lib.moe_router_bwd.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_int, c_void_p,
                                   c_int, c_void_p, c_size_t, c_void_p]
    c_float = ctypes.c_float
    lib.moe_block_norm_fwd.restype = c_int
    lib.moe_block_norm_fwd.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_float,
                                       c_float, c_float, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.moe_block_norm_bwd.restype = c_int
    lib.moe_block_norm_bwd.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_int, c_int, c_int, c_int, c_float, c_float, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_int, c_void_p, c_size_t, c_void_p]
    lib.moe_mx4_quantize.restype = c_int
    lib.moe_mx4_quantize.argtypes = [c_void_p, c_int, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p]
    lib.moe_mx4_dequantize.restype = c_int
    lib.moe_mx4_dequantize.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_int, c_void_p]
    lib.moe_mx4_expert_fwd.restype = c_int
    lib.moe_mx4_expert_fwd.argtypes = [c_void_p, c_int, c_int, c_int, c_int, c_int] + [c_void_p] * 9 + [c_size_t, c_void_p]
    lib.moe_layer_norm_fwd.restype = c_int
    lib.moe_layer_norm_fwd.argtypes = [c_void_p] * 4 + [c_int] * 4 + [c_float] + [c_void_p] * 5
    lib.moe_layer_norm_bwd.restype = c_int
    lib.moe_layer_norm_bwd.argtypes = [c_void_p] * 6 + [c_int] * 4 + [c_void_p] * 4 + [c_int, c_void_p, c_size_t, c_void_p]
    lib.moe_linear_fwd.restype = c_int
    lib.moe_linear_fwd.argtypes = [c_void_p] + [c_int] * 5 + [c_void_p] * 3 + [c_int] + [c_void_p] * 4 + [c_size_t, c_void_p]
    lib.moe_linear_bwd.restype = c_int
    lib.moe_linear_bwd.argtypes = [c_void_p] * 3 + [c_int] * 5 + [c_void_p] * 2 + [c_int, c_void_p, c_int] + [c_void_p] * 2 + [c_int, c_void_p, c_size_t, c_void_p]
    lib.moe_workspace_bytes.restype = c_size_t
    lib.moe_workspace_bytes.argtypes = [c_int] * 8
    lib.moe_error_string.restype = ctypes.c_char_p
    lib.moe_error_string.argtypes = [c_int]
    _LIB = lib
    return lib


def marshal_path() -> str:
    import torch
    return os.path.join(_HERE, f"_marshal.{sys.implementation.cache_tag}.torch-{torch.__version__}.so")


class _ChecksHere:
    """In the native marshalling's place where it cannot be loaded: takes no call."""

    def __getattr__(self, name):
        return lambda *args: -1


def _marshal():
    """The native marshalling, bound to the library's entry points."""
    global _MARSHAL
    if _MARSHAL is None:
        path, lib = marshal_path(), load_library()      # (torch's libraries come first)
        try:
            loader = importlib.machinery.ExtensionFileLoader("_marshal", path)
            module = importlib.util.module_from_spec(importlib.util.spec_from_file_location("_marshal", path, loader=loader))
            loader.exec_module(module)
            module.bind(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _MARSHALLED))
        except ImportError as e:
            warnings.warn(f"calls take the host longer without their native marshalling, which __graft_entry__.build() builds: {e}", RuntimeWarning)
            module = _ChecksHere()
        _MARSHAL = module
    return _MARSHAL


def _check(rc: int, name: str):
    if rc != 0:
        raise MoeError(f"{name} failed: {load_library().moe_error_string(rc).decode()} (code {rc})")


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dtype_code(t):
    import torch
    if t.dtype == torch.float32:
        return MOE_F32
    if t.dtype == torch.bfloat16:
        return MOE_BF16
    raise MoeError(f"unsupported dtype {t.dtype}")


def _need(t, dtype=None, shape=None, name="tensor"):
    if t is None:
        return
    if not t.is_cuda or not t.is_contiguous():
        raise MoeError(f"{name} must be a contiguous device tensor")
    if dtype is not None and t.dtype != dtype:
        raise MoeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise MoeError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def moe_workspace_bytes(which, dtype, T, k, d, f, e_cnt, cap) -> int:
    return int(load_library().moe_workspace_bytes(which, dtype, T, k, d, f, e_cnt, cap))


def moe_route(logits, k, gate_mode, e_lo, e_cnt, topk_idx, topk_w, counts):
    rc = _marshal().route(logits, k, gate_mode, e_lo, e_cnt, topk_idx, topk_w, counts)
    if rc >= 0:
        return _check(rc, "moe_route")
    import torch
    T, E = logits.shape
    _need(logits, torch.float32, name="logits")
    _need(topk_idx, torch.int32, (T, k), "topk_idx")
    _need(topk_w, torch.float32, (T, k), "topk_w")
    _need(counts, torch.int32, (e_cnt,), "counts")
    _check(load_library().moe_route(_ptr(logits), T, E, k, gate_mode, e_lo, e_cnt, _ptr(topk_idx), _ptr(topk_w),
                                    _ptr(counts), _stream()), "moe_route")


def moe_dispatch(x, k, topk_idx, row_scale, e_lo, e_cnt, offsets, perm, inv, reuse_plan, xp, ws):
    rc = _marshal().dispatch(x, k, topk_idx, row_scale, e_lo, e_cnt, offsets, perm, inv, reuse_plan, xp, ws)
    if rc >= 0:
        return _check(rc, "moe_dispatch")
    import torch
    T, d = x.shape
    cap = xp.shape[0]
    _need(x, name="x"); _need(xp, x.dtype, (cap, d), "xp")
    _need(topk_idx, torch.int32, (T, k), "topk_idx")
    _need(row_scale, torch.float32, (T, k), "row_scale")
    _need(offsets, torch.int32, (e_cnt + 1,), "offsets")
    _need(perm, torch.int32, (cap,), "perm")
    _need(inv, torch.int32, (T, k), "inv")
    _need(ws, name="ws")
    _check(load_library().moe_dispatch(_ptr(x), _dtype_code(x), T, d, k, _ptr(topk_idx), _ptr(row_scale), e_lo, e_cnt,
                                       _ptr(offsets), _ptr(perm), _ptr(inv), int(reuse_plan), _ptr(xp), cap,
                                       _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(), _stream()),
           "moe_dispatch")


def moe_dispatch_static(x, k, topk_idx, row_scale, e_lo, e_cnt, offsets, perm, inv, xp, status=None):
    """moe_dispatch (plan + row move) on the library's built-in plan scratch: no workspace argument."""
    rc = _marshal().dispatch_static(x, k, topk_idx, row_scale, e_lo, e_cnt, offsets, perm, inv, xp, status)
    if rc >= 0:
        return _check(rc, "moe_dispatch_static")
    import torch
    T, d = x.shape
    cap = xp.shape[0]
    _need(x, name="x"); _need(xp, x.dtype, (cap, d), "xp")
    _need(topk_idx, torch.int32, (T, k), "topk_idx")
    _need(row_scale, torch.float32, (T, k), "row_scale")
    _need(offsets, torch.int32, (e_cnt + 1,), "offsets")
    _need(perm, torch.int32, (cap,), "perm")
    _need(inv, torch.int32, (T, k), "inv")
    _need(status, torch.int32, name="status")
    lib = load_library()
    _check(lib.moe_dispatch_static(_ptr(x), _dtype_code(x), T, d, k, _ptr(topk_idx), _ptr(row_scale), e_lo, e_cnt,
                                   _ptr(offsets), _ptr(perm), _ptr(inv), _ptr(xp), cap, _ptr(status), _stream()),
           "moe_dispatch_static")


def moe_expert_fwd(xp, offsets, w1, w3, w2, h1, h3, o, ws, a=None):
    rc = _marshal().expert_fwd(xp, offsets, w1, w3, w2, h1, h3, o, ws, a)
    if rc >= 0:
        return _check(rc, "moe_expert_fwd")
    import torch
    cap, d = xp.shape
    e_cnt, _, f = w1.shape
    _need(xp, name="xp"); _need(o, xp.dtype, (cap, d), "o")
    _need(w1, xp.dtype, (e_cnt, d, f), "w1"); _need(w3, xp.dtype, (e_cnt, d, f), "w3")
    _need(w2, xp.dtype, (e_cnt, f, d), "w2")
    _need(h1, xp.dtype, (cap, f), "h1"); _need(h3, xp.dtype, (cap, f), "h3"); _need(a, xp.dtype, (cap, f), "a")
    _need(offsets, torch.int32, (e_cnt + 1,), "offsets"); _need(ws, name="ws")
    _check(load_library().moe_expert_fwd(_ptr(xp), _dtype_code(xp), cap, d, f, e_cnt, _ptr(offsets), _ptr(w1), _ptr(w3),
                                         _ptr(w2), _ptr(h1), _ptr(h3), _ptr(a), _ptr(o), _ptr(ws),
                                         ws.numel() * ws.element_size(), _stream()), "moe_expert_fwd")


def moe_expert_bwd(xp, h1, h3, d_o, offsets, w1, w3, w2, dxp, dw1, dw3, dw2, accumulate, ws, a=None):
    rc = _marshal().expert_bwd(xp, h1, h3, d_o, offsets, w1, w3, w2, dxp, dw1, dw3, dw2, accumulate, ws, a)
    if rc >= 0:
        return _check(rc, "moe_expert_bwd")
    import torch
    cap, d = xp.shape
    e_cnt, _, f = w1.shape
    dt = xp.dtype
    _need(xp, name="xp"); _need(h1, dt, (cap, f), "h1"); _need(h3, dt, (cap, f), "h3"); _need(a, dt, (cap, f), "a")
    _need(d_o, dt, (cap, d), "d_o"); _need(dxp, dt, (cap, d), "dxp")
    _need(w1, dt, (e_cnt, d, f), "w1"); _need(w3, dt, (e_cnt, d, f), "w3"); _need(w2, dt, (e_cnt, f, d), "w2")
    _need(dw1, dt, (e_cnt, d, f), "dw1"); _need(dw3, dt, (e_cnt, d, f), "dw3"); _need(dw2, dt, (e_cnt, f, d), "dw2")
    _need(offsets, torch.int32, (e_cnt + 1,), "offsets"); _need(ws, name="ws")
    _check(load_library().moe_expert_bwd(_ptr(xp), _ptr(h1), _ptr(h3), _ptr(a), _ptr(d_o), _dtype_code(xp), cap, d, f, e_cnt,
                                         _ptr(offsets), _ptr(w1), _ptr(w3), _ptr(w2), _ptr(dxp), _ptr(dw1), _ptr(dw3),
                                         _ptr(dw2), int(accumulate), _ptr(ws), ws.numel() * ws.element_size(),
                                         _stream()), "moe_expert_bwd")


def moe_combine(o, inv, topk_w, y):
    rc = _marshal().combine(o, inv, topk_w, y)
    if rc >= 0:
        return _check(rc, "moe_combine")
    import torch
    T, k = inv.shape
    d = o.shape[1]
    _need(o, name="o"); _need(y, o.dtype, (T, d), "y")
    _need(inv, torch.int32, name="inv"); _need(topk_w, torch.float32, (T, k), "topk_w")
    _check(load_library().moe_combine(_ptr(o), _dtype_code(o), T, d, k, _ptr(inv), _ptr(topk_w), _ptr(y), _stream()),
           "moe_combine")


def moe_router_fwd(x, wr, logits, ws):
    rc = _marshal().router_fwd(x, wr, logits, ws)
    if rc >= 0:
        return _check(rc, "moe_router_fwd")
    import torch
    T, d = x.shape
    E = wr.shape[1]
    _need(x, name="x"); _need(wr, x.dtype, (d, E), "wr"); _need(logits, torch.float32, (T, E), "logits")
    _need(ws, name="ws")
    _check(load_library().moe_router_fwd(_ptr(x), _ptr(wr), _dtype_code(x), T, d, E, _ptr(logits), _ptr(ws),
                                         ws.numel() * ws.element_size(), _stream()), "moe_router_fwd")


def moe_combine_bwd(dy, o, inv, topk_w, d_o, dgate):
    rc = _marshal().combine_bwd(dy, o, inv, topk_w, d_o, dgate)
    if rc >= 0:
        return _check(rc, "moe_combine_bwd")
    import torch
    T, k = inv.shape
    d = dy.shape[1]
    _need(dy, name="dy"); _need(o, dy.dtype, name="o"); _need(d_o, dy.dtype, tuple(o.shape), "d_o")
    _need(inv, torch.int32, name="inv"); _need(topk_w, torch.float32, (T, k), "topk_w")
    _need(dgate, torch.float32, (T, k), "dgate")
    if o.shape[1] != d or dy.shape[0] != T:
        raise MoeError("dy must be [T,d] and o [rows,d]")
    _check(load_library().moe_combine_bwd(_ptr(dy), _ptr(o), _dtype_code(dy), T, d, k, _ptr(inv), _ptr(topk_w),
                                          _ptr(d_o), _ptr(dgate), _stream()), "moe_combine_bwd")


def moe_gate_bwd(logits, topk_idx, dgate, gate_mode, dlogits):
    rc = _marshal().gate_bwd(logits, topk_idx, dgate, gate_mode, dlogits)
    if rc >= 0:
        return _check(rc, "moe_gate_bwd")
    import torch
    T, E = logits.shape
    k = topk_idx.shape[1]
    _need(logits, torch.float32, name="logits"); _need(topk_idx, torch.int32, (T, k), "topk_idx")
    _need(dgate, torch.float32, (T, k), "dgate"); _need(dlogits, torch.float32, (T, E), "dlogits")
    _check(load_library().moe_gate_bwd(_ptr(logits), _ptr(topk_idx), _ptr(dgate), T, E, k, gate_mode, _ptr(dlogits),
                                       _stream()), "moe_gate_bwd")


def moe_router_bwd(x, wr, dlogits, dwr, dwr_accumulate, dx, dx_accumulate, ws):
    rc = _marshal().router_bwd(x, wr, dlogits, dwr, dwr_accumulate, dx, dx_accumulate, ws)
    if rc >= 0:
        return _check(rc, "moe_router_bwd")
    import torch
    T, d = x.shape
    E = wr.shape[1]
    _need(x, name="x"); _need(wr, x.dtype, (d, E), "wr"); _need(dlogits, torch.float32, (T, E), "dlogits")
    _need(dwr, x.dtype, (d, E), "dwr"); _need(dx, x.dtype, (T, d), "dx"); _need(ws, name="ws")
    _check(load_library().moe_router_bwd(_ptr(x), _ptr(wr), _ptr(dlogits), _dtype_code(x), T, d, E, _ptr(dwr),
                                         int(dwr_accumulate), _ptr(dx), int(dx_accumulate), _ptr(ws),
                                         ws.numel() * ws.element_size(), _stream()), "moe_router_bwd")


def moe_block_norm_fwd(y, gate, w_post, post_norm, h, w_pre, alpha, beta, eps, h_out, n, r_post=None, r_pre=None):
    """y [T,d] or None (the norm in front of a first block), h [T,d]; w_pre and n both or neither."""
    rc = _marshal().block_norm_fwd(y, gate, w_post, post_norm, h, w_pre, alpha, beta, eps, h_out, n, r_post, r_pre)
    if rc >= 0:
        return _check(rc, "moe_block_norm_fwd")
    import torch
    T, d = h.shape
    t = w_pre if y is None else y
    if t is None:
        raise MoeError("without y there must be w_pre and n")
    dt = t.dtype
    _need(h, name="h"); _need(y, dt, (T, d), "y"); _need(gate, torch.float32, (T,), "gate")
    _need(w_post, dt, (d,), "w_post"); _need(w_pre, dt, (d,), "w_pre")
    _need(h_out, h.dtype, (T, d), "h_out"); _need(n, dt, (T, d), "n")
    _need(r_post, torch.float32, (T,), "r_post"); _need(r_pre, torch.float32, (T,), "r_pre")
    _check(load_library().moe_block_norm_fwd(_ptr(y), _ptr(gate), _ptr(w_post), int(post_norm), _ptr(h), _ptr(w_pre), _dtype_code(t),
                                             _dtype_code(h), T, d, alpha, beta, eps, _ptr(h_out), _ptr(n), _ptr(r_post), _ptr(r_pre),
                                             _stream()), "moe_block_norm_fwd")


def moe_block_norm_bwd(y, gate, w_post, post_norm, h_out, w_pre, r_post, r_pre, dh_out, dn, alpha, beta, dh, dy, dgate, dw_post,
                       dw_pre, accumulate, ws):
    """h_out is the saved sum of the forward (h itself where y is None); it may be None where dn is."""
    rc = _marshal().block_norm_bwd(y, gate, w_post, post_norm, h_out, w_pre, r_post, r_pre, dh_out, dn, alpha, beta, dh, dy, dgate, dw_post,
                                   dw_pre, accumulate, ws)
    if rc >= 0:
        return _check(rc, "moe_block_norm_bwd")
    import torch
    res, t = (next((v for v in pair if v is not None), None) for pair in ((h_out, dh_out), (dn, y)))
    if res is None or t is None:
        raise MoeError("there must be h_out or dh_out, and dn or y")
    (T, d), dt, rt = t.shape, t.dtype, res.dtype
    _need(y, dt, (T, d), "y"); _need(gate, torch.float32, (T,), "gate")
    _need(w_post, dt, (d,), "w_post"); _need(w_pre, dt, (d,), "w_pre")
    _need(h_out, rt, (T, d), "h_out"); _need(dh_out, rt, (T, d), "dh_out"); _need(dn, dt, (T, d), "dn")
    _need(r_post, torch.float32, (T,), "r_post"); _need(r_pre, torch.float32, (T,), "r_pre")
    _need(dh, rt, (T, d), "dh"); _need(dy, dt, (T, d), "dy"); _need(dgate, torch.float32, (T,), "dgate")
    _need(dw_post, dt, (d,), "dw_post"); _need(dw_pre, dt, (d,), "dw_pre"); _need(ws, name="ws")
    _check(load_library().moe_block_norm_bwd(_ptr(y), _ptr(gate), _ptr(w_post), int(post_norm), _ptr(h_out), _ptr(w_pre), _ptr(r_post),
                                             _ptr(r_pre), _ptr(dh_out), _ptr(dn), _dtype_code(t), _dtype_code(res), T, d, alpha, beta,
                                             _ptr(dh), _ptr(dy), _ptr(dgate), _ptr(dw_post), _ptr(dw_pre), int(accumulate), _ptr(ws),
                                             ws.numel() * ws.element_size(), _stream()), "moe_block_norm_bwd")


def moe_layer_norm_fwd(y, h, w, b, eps, h_out, n, mean=None, rstd=None):
    """h [T,d], n [T,d]; y [T,d] or None (nothing is added), and then h_out None."""
    rc = _marshal().layer_norm_fwd(y, h, w, b, eps, h_out, n, mean, rstd)
    if rc >= 0:
        return _check(rc, "moe_layer_norm_fwd")
    import torch
    (T, d), dt = h.shape, n.dtype
    _need(h, name="h"); _need(y, dt, (T, d), "y"); _need(w, dt, (d,), "w"); _need(b, dt, (d,), "b")
    _need(h_out, h.dtype, (T, d), "h_out"); _need(n, dt, (T, d), "n")
    _need(mean, torch.float32, (T,), "mean"); _need(rstd, torch.float32, (T,), "rstd")
    _check(load_library().moe_layer_norm_fwd(_ptr(y), _ptr(h), _ptr(w), _ptr(b), _dtype_code(n), _dtype_code(h), T, d, eps, _ptr(h_out), _ptr(n),
                                             _ptr(mean), _ptr(rstd), _stream()), "moe_layer_norm_fwd")


def moe_layer_norm_bwd(h_out, w, mean, rstd, dh_out, dn, dh, dy, dw, db, accumulate, ws):
    """h_out is the saved sum of the forward (h itself where y was None); dh_out None: no gradient from further on.  Outputs may be None."""
    rc = _marshal().layer_norm_bwd(h_out, w, mean, rstd, dh_out, dn, dh, dy, dw, db, accumulate, ws)
    if rc >= 0:
        return _check(rc, "moe_layer_norm_bwd")
    import torch
    (T, d), dt, rt = h_out.shape, dn.dtype, h_out.dtype
    _need(h_out, name="h_out"); _need(w, dt, (d,), "w"); _need(mean, torch.float32, (T,), "mean"); _need(rstd, torch.float32, (T,), "rstd")
    _need(dh_out, rt, (T, d), "dh_out"); _need(dn, dt, (T, d), "dn"); _need(dh, rt, (T, d), "dh"); _need(dy, dt, (T, d), "dy")
    _need(dw, dt, (d,), "dw"); _need(db, dt, (d,), "db"); _need(ws, name="ws")
    _check(load_library().moe_layer_norm_bwd(_ptr(h_out), _ptr(w), _ptr(mean), _ptr(rstd), _ptr(dh_out), _ptr(dn), _dtype_code(dn), _dtype_code(h_out),
                                             T, d, _ptr(dh), _ptr(dy), _ptr(dw), _ptr(db), int(accumulate), _ptr(ws),
                                             ws.numel() * ws.element_size(), _stream()), "moe_layer_norm_bwd")


def _linear_shapes(rows, weights, offsets):
    """(cap, K, N, e_cnt, batch of a weight) of rows [cap,K] and weights [K,N] without offsets, [e_cnt,K,N] with them."""
    if rows.dim() != 2 or weights.dim() != (2 if offsets is None else 3):
        raise MoeError("rows must be a matrix, and weights a matrix without offsets, matrices with them")
    return rows.shape[0], *weights.shape[-2:], 1 if offsets is None else weights.shape[0], tuple(weights.shape[:-2])


def moe_linear_fwd(x, offsets, w, bias, act, residual, z, y, ws):
    """x [cap,K]; offsets None: w [K,N], bias [N]; else w [e_cnt,K,N], bias [e_cnt,N].  act: ACT_*; bias, residual and z may be None."""
    rc = _marshal().linear_fwd(x, offsets, w, bias, act, residual, z, y, ws)
    if rc >= 0:
        return _check(rc, "moe_linear_fwd")
    import torch
    cap, K, N, e_cnt, batch = _linear_shapes(x, w, offsets)
    dt = x.dtype
    _need(x, dt, (cap, K), "x"); _need(w, dt, name="w"); _need(bias, dt, batch + (N,), "bias"); _need(offsets, torch.int32, (e_cnt + 1,), "offsets")
    _need(residual, dt, (cap, N), "residual"); _need(z, dt, (cap, N), "z"); _need(y, dt, (cap, N), "y"); _need(ws, name="ws")
    _check(load_library().moe_linear_fwd(_ptr(x), _dtype_code(x), cap, K, N, e_cnt, _ptr(offsets), _ptr(w), _ptr(bias), int(act), _ptr(residual),
                                         _ptr(z), _ptr(y), _ptr(ws), ws.numel() * ws.element_size(), _stream()), "moe_linear_fwd")


def moe_linear_bwd(x, z, dy, offsets, w, act, dx, dw, db, accumulate, ws, dx_accumulate=False):
    """Shapes as in moe_linear_fwd; z None where act is ACT_NONE; outputs may be None.  The gradient of a residual is dy."""
    rc = _marshal().linear_bwd(x, z, dy, offsets, w, act, dx, dw, db, accumulate, ws, dx_accumulate)
    if rc >= 0:
        return _check(rc, "moe_linear_bwd")
    import torch
    cap, K, N, e_cnt, batch = _linear_shapes(x, w, offsets)
    dt = x.dtype
    _need(x, dt, (cap, K), "x"); _need(w, dt, name="w"); _need(offsets, torch.int32, (e_cnt + 1,), "offsets")
    _need(z, dt, (cap, N), "z"); _need(dy, dt, (cap, N), "dy"); _need(dx, dt, (cap, K), "dx"); _need(dw, dt, batch + (K, N), "dw")
    _need(db, dt, batch + (N,), "db"); _need(ws, name="ws")
    _check(load_library().moe_linear_bwd(_ptr(x), _ptr(z), _ptr(dy), _dtype_code(x), cap, K, N, e_cnt, _ptr(offsets), _ptr(w), int(act), _ptr(dx),
                                         int(dx_accumulate), _ptr(dw), _ptr(db), int(accumulate), _ptr(ws), ws.numel() * ws.element_size(), _stream()), "moe_linear_bwd")


def mx4_shapes(n, K):
    """Shapes (data, scales) of n rows of K elements in microscaled 4 bits, both uint8 (layout: moe.h)."""
    return ((n + 15) // 16, (K + 127) // 128, 4, 16, 16), ((n + 15) // 16, (K + 511) // 512, 4, 16, 4)


def _need_mx4(data, scales, batch, n, K, name):
    import torch
    for t, shape, what in zip((data, scales), mx4_shapes(n, K), ("data", "scales")):
        _need(t, torch.uint8, tuple(batch) + shape, f"{name} {what}")


def moe_mx4_quantize(x, along_rows, data, scales):
    """x [n,K] or [batch,n,K]; along_rows: [K,n] or [batch,K,n].  data, scales: mx4_shapes(n, K), behind the batch."""
    rc = _marshal().mx4_quantize(x, along_rows, data, scales)
    if rc >= 0:
        return _check(rc, "moe_mx4_quantize")
    if x.dim() not in (2, 3):
        raise MoeError("x must be a matrix or a batch of matrices")
    (rows, cols), batch = x.shape[-2:], x.shape[:-2]
    _need(x, name="x")
    _need_mx4(data, scales, batch, *((cols, rows) if along_rows else (rows, cols)), "x's")
    _check(load_library().moe_mx4_quantize(_ptr(x), _dtype_code(x), batch[0] if batch else 1, rows, cols, int(along_rows), _ptr(data),
                                           _ptr(scales), _stream()), "moe_mx4_quantize")


def moe_mx4_dequantize(data, scales, out):
    """out [n,K] or [batch,n,K], the values of data and scales."""
    rc = _marshal().mx4_dequantize(data, scales, out)
    if rc >= 0:
        return _check(rc, "moe_mx4_dequantize")
    if out.dim() not in (2, 3):
        raise MoeError("out must be a matrix or a batch of matrices")
    (n, K), batch = out.shape[-2:], out.shape[:-2]
    _need(out, name="out")
    _need_mx4(data, scales, batch, n, K, "out's")
    _check(load_library().moe_mx4_dequantize(_ptr(data), _ptr(scales), batch[0] if batch else 1, n, K, _ptr(out), _dtype_code(out),
                                             _stream()), "moe_mx4_dequantize")


def moe_mx4_expert_fwd(xp, offsets, w1, s1, w3, s3, w2, s2, o, ws):
    """w1, s1, w3, s3: data and scales of e_cnt matrices with n = f, K = d; w2, s2: n = d, K = f (f is a multiple of 32: w1's tiles say it)."""
    rc = _marshal().mx4_expert_fwd(xp, offsets, w1, s1, w3, s3, w2, s2, o, ws)
    if rc >= 0:
        return _check(rc, "moe_mx4_expert_fwd")
    import torch
    cap, d = xp.shape
    if w1.dim() != 6:
        raise MoeError("w1 must hold the tiles of e_cnt matrices")
    e_cnt, f = w1.shape[0], 16 * w1.shape[1]
    _need(xp, name="xp"); _need(o, xp.dtype, (cap, d), "o")
    _need_mx4(w1, s1, (e_cnt,), f, d, "w1's"); _need_mx4(w3, s3, (e_cnt,), f, d, "w3's"); _need_mx4(w2, s2, (e_cnt,), d, f, "w2's")
    _need(offsets, torch.int32, (e_cnt + 1,), "offsets"); _need(ws, name="ws")
    _check(load_library().moe_mx4_expert_fwd(_ptr(xp), _dtype_code(xp), cap, d, f, e_cnt, _ptr(offsets), _ptr(w1), _ptr(s1), _ptr(w3), _ptr(s3),
                                             _ptr(w2), _ptr(s2), _ptr(o), _ptr(ws), ws.numel() * ws.element_size(), _stream()),
           "moe_mx4_expert_fwd")


KERNEL_IDS = dict(route=0, plan=1, dispatch=2, combine=3, up=4, down=5, da=6, dx=7, wg=8, wgd=9, router_fwd=10,
                  combine_bwd=11, gate_bwd=12, router_dw=13, router_dx=14, wgrad_reduce=15, da_wg=16, dx_wgd=17, norm_fwd=18,
                  norm_bwd=19, norm_sums=20, mx4_quantize=21, mx4_dequantize=22, mx4_rows=23, mx4_up=24, mx4_down=25,
                  layer_norm_fwd=26, layer_norm_bwd=27, layer_norm_sums=28, linear=29, linear_act=30, linear_bias=31, linear_dx=32,
                  linear_dw=33, linear_dx_dw=34)


def moe_profile_enable(on: bool):
    lib = load_library()
    lib.moe_profile_enable.restype = ctypes.c_int
    lib.moe_profile_enable.argtypes = [ctypes.c_int]
    _check(lib.moe_profile_enable(int(on)), "moe_profile_enable")


def moe_profile_read(kernel: str):
    """(total milliseconds, launches) recorded for one kernel family since profiling was enabled."""
    lib = load_library()
    lib.moe_profile_read.restype = ctypes.c_int
    lib.moe_profile_read.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int)]
    ms, n = ctypes.c_double(0), ctypes.c_int(0)
    _check(lib.moe_profile_read(KERNEL_IDS[kernel], ctypes.byref(ms), ctypes.byref(n)), "moe_profile_read")
    return ms.value, n.value


def moe_profile_stats(kernel: str):
    """(shortest, median) launch in milliseconds of one kernel family since profiling was enabled."""
    lib = load_library()
    lib.moe_profile_stats.restype = ctypes.c_int
    lib.moe_profile_stats.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    lo, med = ctypes.c_double(0), ctypes.c_double(0)
    _check(lib.moe_profile_stats(KERNEL_IDS[kernel], ctypes.byref(lo), ctypes.byref(med)), "moe_profile_stats")
    return lo.value, med.value


def moe_probe_mfma_bf16(sink, iters: int, random_operands: bool) -> float:
    """Enqueue the MFMA-only ceiling kernel; returns the FLOP count of the launch."""
    lib = load_library()
    lib.moe_probe_mfma_bf16.restype = ctypes.c_int
    lib.moe_probe_mfma_bf16.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int,
                                        ctypes.POINTER(ctypes.c_double), ctypes.c_void_p]
    flop = ctypes.c_double(0)
    _check(lib.moe_probe_mfma_bf16(_ptr(sink), sink.numel() * sink.element_size(), int(iters), int(random_operands),
                                   ctypes.byref(flop), _stream()), "moe_probe_mfma_bf16")
    return flop.value


def moe_probe_copy(src, dst):
    lib = load_library()
    lib.moe_probe_copy.restype = ctypes.c_int
    lib.moe_probe_copy.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    _check(lib.moe_probe_copy(_ptr(src), _ptr(dst), src.numel() * src.element_size(), _stream()), "moe_probe_copy")


def moe_probe_mfma_fed_bf16(sink, iters: int, feed: int) -> float:
    """Enqueue the MFMA loop whose operands are re-read from LDS (feed 1: 16-byte reads, 2: transposing
    reads); returns the FLOP count of the launch."""
    lib = load_library()
    lib.moe_probe_mfma_fed_bf16.restype = ctypes.c_int
    lib.moe_probe_mfma_fed_bf16.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int,
                                            ctypes.POINTER(ctypes.c_double), ctypes.c_void_p]
    flop = ctypes.c_double(0)
    _check(lib.moe_probe_mfma_fed_bf16(_ptr(sink), sink.numel() * sink.element_size(), int(iters), int(feed),
                                       ctypes.byref(flop), _stream()), "moe_probe_mfma_fed_bf16")
    return flop.value


def moe_probe_stream(src, dst, writes: int, sink=None):
    """Streaming ceiling kernels over src's bytes: writes = -1 read only, 0 fill dst, n >= 1 one read and n writes."""
    lib = load_library()
    lib.moe_probe_stream.restype = ctypes.c_int
    lib.moe_probe_stream.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_void_p,
                                     ctypes.c_void_p]
    nbytes = src.numel() * src.element_size()
    if writes >= 1 and dst.numel() * dst.element_size() < writes * nbytes:
        raise MoeError("dst must hold `writes` copies of src")
    _check(lib.moe_probe_stream(_ptr(src), _ptr(dst), nbytes, int(writes), _ptr(sink), _stream()), "moe_probe_stream")
