"""A residual block of experts of two matrices with biases, with a dense expert that every token passes and layer norms between the blocks, as a model of
that kind stacks them: what one GPU's share of the experts and the dense expert add to the residual stream.

    a = act(xp W1[e] + b1[e])       o = a W2[e] + b2[e]       y = combine(o) + act(x Ws1 + bs1) Ws2 + bs2
    h' = h + y                      x' = layernorm(h') w + b

x is the block's input, the normalised residual stream h; x' is the next block's.  The norm in front of a first block is moe_layer_norm_fwd with
y = None, and its gradient moe_layer_norm_bwd with the stream itself.

training: run_ffn_forward, and run_ffn_backward from the last block to the first: its `dh` and `dx` are the `dh_out` and `dn` of the block before.
serving : run_ffn_forward with buffers without gradients, of as many tokens as these are for, or fewer.
Nothing synchronises with the host between the calls.
"""
from __future__ import annotations

import torch

from . import binding as B
from .layer import torch_dtype


class FfnBlockBuffers:
    """All outputs, saved activations and scratch of one block's step, allocated once.  shared_f: width of the dense expert.  residual: the type of the
    residual stream, the tokens' own or fp32.  Without gradients they serve up to wl.T tokens; a training step takes wl.T."""

    def __init__(self, wl, cap: int, shared_f: int, act: str = "gelu", residual=None, grads: bool = True, device="cuda"):
        dt, T, d, k, f, ec = torch_dtype(wl), wl.T, wl.d, wl.k, wl.f, wl.e_cnt
        code = B.MOE_BF16 if wl.dtype == "bf16" else B.MOE_F32
        new = lambda *shape, dtype=dt: torch.empty(shape, dtype=dtype, device=device)  # noqa: E731
        i32, f32 = torch.int32, torch.float32
        self.act, self.grads = B.ACTIVATIONS[act], grads
        self.logits, self.topk_idx, self.topk_w = new(T, wl.E, dtype=f32), new(T, k, dtype=i32), new(T, k, dtype=f32)
        self.counts, self.offsets, self.perm, self.inv = new(ec, dtype=i32), new(ec + 1, dtype=i32), new(cap, dtype=i32), new(T, k, dtype=i32)
        self.xp, self.a, self.o = new(cap, d), new(cap, f), new(cap, d)
        self.sa, self.y = new(T, shared_f), new(T, d)
        self.h, self.x = new(T, d, dtype=residual or dt), new(T, d)
        self.z = self.sz = self.mean = self.rstd = None
        ws = lambda which, *sizes: B.moe_workspace_bytes(which, code, *sizes)  # noqa: E731
        uses = [ws(B.WS_LINEAR_FWD, 0, 0, K, N, n, rows) for K, N, n, rows in self._products(wl, cap, shared_f)]
        if grads:
            self.z, self.sz = new(cap, f), new(T, shared_f)
            self.mean, self.rstd = new(T, dtype=f32), new(T, dtype=f32)
            self.dh, self.dx = torch.empty_like(self.h), new(T, d)
            self.dy = self.dh if self.h.dtype == dt else new(T, d)
            self.d_o, self.da, self.dxp, self.dsa = new(cap, d), new(cap, f), new(cap, d), new(T, shared_f)
            self.dgate, self.dlogits = new(T, k, dtype=f32), new(T, wl.E, dtype=f32)
            self.dw = dict(wr=new(d, wl.E), w1=new(ec, d, f), b1=new(ec, f), w2=new(ec, f, d), b2=new(ec, d), ws1=new(d, shared_f), bs1=new(shared_f),
                           ws2=new(shared_f, d), bs2=new(d), w=new(d), b=new(d))
            uses += [ws(B.WS_LINEAR_BWD, 0, 0, K, N, n, rows) for K, N, n, rows in self._products(wl, cap, shared_f)]
            uses.append(ws(B.WS_LAYER_NORM, T, 0, d, 0, 0, 0))
        # (what the router's logits take is not monotonic in the tokens: of all numbers of them that may come the largest)
        uses += [ws(B.WS_DISPATCH, T, k, d, f, ec, cap)] + [ws(B.WS_ROUTER, t, k, d, f, wl.E, cap) for t in ((T,) if grads else range(T + 1))]
        self.ws = new(max(uses), dtype=torch.uint8)        # one after the other on a stream: the calls take turns

    def of_tokens(self, T):
        """What the forward writes per token; without gradients T rows of each (refused by the calls where there are fewer)."""
        per_token = self.logits, self.topk_idx, self.topk_w, self.inv, self.sa, self.y, self.h, self.x
        return per_token if self.grads or len(self.y) == T else tuple(t[:T] for t in per_token)

    @staticmethod
    def _products(wl, cap, shared_f):
        return (wl.d, wl.f, wl.e_cnt, cap), (wl.f, wl.d, wl.e_cnt, cap), (wl.d, shared_f, 1, wl.T), (shared_f, wl.d, 1, wl.T)


def run_ffn_forward(wl, w, h, x, buf: FfnBlockBuffers, eps: float = 1e-5):
    """w: "wr", "w1", "b1", "w2", "b2" of the experts, "ws1", "bs1", "ws2", "bs2" of the dense one, "w", "b" of the norm.  -> buf.h, buf.x, of which fewer
    tokens than the buffers are for (without gradients) take the first rows"""
    logits, topk_idx, topk_w, inv, sa, y, h_out, x_out = buf.of_tokens(x.shape[0])
    B.moe_router_fwd(x, w["wr"], logits, buf.ws)
    B.moe_route(logits, wl.k, wl.gate_mode, wl.e_lo, wl.e_cnt, topk_idx, topk_w, buf.counts)
    B.moe_dispatch(x, wl.k, topk_idx, None, wl.e_lo, wl.e_cnt, buf.offsets, buf.perm, inv, False, buf.xp, buf.ws)
    B.moe_linear_fwd(buf.xp, buf.offsets, w["w1"], w["b1"], buf.act, None, buf.z, buf.a, buf.ws)
    B.moe_linear_fwd(buf.a, buf.offsets, w["w2"], w["b2"], B.ACT_NONE, None, None, buf.o, buf.ws)
    B.moe_combine(buf.o, inv, topk_w, y)
    B.moe_linear_fwd(x, None, w["ws1"], w["bs1"], buf.act, None, buf.sz, sa, buf.ws)
    B.moe_linear_fwd(sa, None, w["ws2"], w["bs2"], B.ACT_NONE, y, None, y, buf.ws)      # onto what the experts gave
    B.moe_layer_norm_fwd(y, h, w["w"], w["b"], eps, h_out, x_out, buf.mean, buf.rstd)


def run_ffn_backward(wl, w, x, buf: FfnBlockBuffers, dh_out, dn, accumulate: bool = False):
    """dh_out, dn: the gradients of buf.h (None: nothing behind reads it but the norm) and of buf.x.  -> buf.dh, buf.dx, and buf.dw by w's names"""
    g, act = buf.dw, buf.act
    B.moe_layer_norm_bwd(buf.h, w["w"], buf.mean, buf.rstd, dh_out, dn, buf.dh, None if buf.dy is buf.dh else buf.dy, g["w"], g["b"], accumulate, buf.ws)
    B.moe_combine_bwd(buf.dy, buf.o, buf.inv, buf.topk_w, buf.d_o, buf.dgate)
    B.moe_linear_bwd(buf.a, None, buf.d_o, buf.offsets, w["w2"], B.ACT_NONE, buf.da, g["w2"], g["b2"], accumulate, buf.ws)
    B.moe_linear_bwd(buf.xp, buf.z, buf.da, buf.offsets, w["w1"], act, buf.dxp, g["w1"], g["b1"], accumulate, buf.ws)
    B.moe_combine(buf.dxp, buf.inv, None, buf.dx)
    B.moe_linear_bwd(buf.sa, None, buf.dy, None, w["ws2"], B.ACT_NONE, buf.dsa, g["ws2"], g["bs2"], accumulate, buf.ws)
    B.moe_linear_bwd(x, buf.sz, buf.dsa, None, w["ws1"], act, buf.dx, g["ws1"], g["bs1"], accumulate, buf.ws, True)
    B.moe_gate_bwd(buf.logits, buf.topk_idx, buf.dgate, wl.gate_mode, buf.dlogits)
    B.moe_router_bwd(x, w["wr"], buf.dlogits, g["wr"], accumulate, buf.dx, True, buf.ws)
