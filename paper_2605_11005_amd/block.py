"""A residual block around the expert layer, as a model stacks them: what one GPU's share of the experts adds to the residual stream,
and the norms on either side of it.

    y = experts(x)        h' = h + norm(y) w_post        x' = norm(h') w_pre

x is the block's input, the normalised residual stream h; x' is the next block's.  The norm in front of a first block is
moe_block_norm_fwd with y = None, and its gradient moe_block_norm_bwd with y = None.

training: run_block_forward, and run_block_backward from the last block to the first: its `dh` and `layer.dx` are the `dh_out` and
          `dn` of the block before.
serving : run_block_serve with the experts' weights in microscaled 4 bits (serve_weights).
Nothing synchronises with the host between the calls.
"""
from __future__ import annotations

import torch

from . import binding as B
from .layer import MoeLayerBuffers, mx4_weights, run_backward_router, run_forward_router, torch_dtype


class _Norms:
    """What the norms behind the layer write: the residual stream (bf16 or fp32) and the next block's input."""

    def __init__(self, wl, residual, device):
        self.h = torch.empty((wl.T, wl.d), dtype=residual or torch_dtype(wl), device=device)
        self.x = torch.empty((wl.T, wl.d), dtype=torch_dtype(wl), device=device)


class MoeBlockBuffers(_Norms):
    """All outputs, saved activations and scratch of one block's training step, allocated once."""

    def __init__(self, wl, cap: int, residual=None, device="cuda"):
        super().__init__(wl, residual, device)
        self.layer = MoeLayerBuffers(wl, cap, device=device, router=True)
        self.r_post, self.r_pre = (torch.empty((wl.T,), dtype=torch.float32, device=device) for _ in range(2))
        self.dh, self.dy = torch.empty_like(self.h), torch.empty_like(self.x)
        self.dw_post, self.dw_pre = (torch.empty((wl.d,), dtype=self.x.dtype, device=device) for _ in range(2))
        self.ws = torch.empty(B.moe_workspace_bytes(B.WS_BLOCK_NORM, 0, wl.T, 0, wl.d, 0, 0, 0), dtype=torch.uint8, device=device)


def run_block_forward(wl, w, h, x, buf: MoeBlockBuffers, eps: float = 1e-6):
    """w: "wr", "w1", "w3", "w2", "w_post", "w_pre".  -> buf.h, buf.x"""
    run_forward_router(wl, dict(w, x=x), buf.layer)
    B.moe_block_norm_fwd(buf.layer.y, None, w["w_post"], True, h, w["w_pre"], 1.0, 1.0, eps, buf.h, buf.x, buf.r_post, buf.r_pre)


def run_block_backward(wl, w, x, buf: MoeBlockBuffers, dh_out, dn, accumulate: bool = False):
    """dh_out, dn: the gradients of buf.h (None: nothing behind reads it but the norm) and of buf.x.  -> buf.dh, buf.layer.dx and the weights'"""
    B.moe_block_norm_bwd(buf.layer.y, None, w["w_post"], True, buf.h, w["w_pre"], buf.r_post, buf.r_pre, dh_out, dn, 1.0, 1.0, buf.dh, buf.dy, None,
                         buf.dw_post, buf.dw_pre, accumulate, buf.ws)
    run_backward_router(wl, dict(w, x=x, dy=buf.dy), buf.layer, accumulate)


class MoeServeBuffers(_Norms):
    """What one block keeps for up to T tokens when its experts are in 4 bits."""

    def __init__(self, wl, cap: int, residual=None, device="cuda"):
        super().__init__(wl, residual, device)
        i32 = dict(dtype=torch.int32, device=device)
        self.logits = torch.empty((wl.T, wl.E), dtype=torch.float32, device=device)
        self.topk_idx, self.inv = torch.empty((wl.T, wl.k), **i32), torch.empty((wl.T, wl.k), **i32)
        self.topk_w = torch.empty((wl.T, wl.k), dtype=torch.float32, device=device)
        self.counts, self.offsets, self.perm = torch.empty((wl.e_cnt,), **i32), torch.empty((wl.e_cnt + 1,), **i32), torch.empty((cap,), **i32)
        self.xp, self.o = (torch.empty((cap, wl.d), dtype=torch.bfloat16, device=device) for _ in range(2))
        self.y = torch.empty((wl.T, wl.d), dtype=torch.bfloat16, device=device)
        # (what the router's logits take is not monotonic in the tokens: of all numbers of them the largest)
        ws = lambda which, n, tokens=(wl.T,): torch.empty(  # noqa: E731
            max(B.moe_workspace_bytes(which, B.MOE_BF16, T, wl.k, wl.d, wl.f, n, cap) for T in tokens), dtype=torch.uint8, device=device)
        self.ws_router, self.ws_dispatch = ws(B.WS_ROUTER, wl.E, range(wl.T + 1)), ws(B.WS_DISPATCH, wl.e_cnt)
        self.ws_experts = ws(B.WS_MX4_EXPERT_FWD, wl.e_cnt)

    def of_tokens(self, T):
        """What has a row per token, T rows of each (refused by the calls where there are fewer)."""
        per_token = self.logits, self.topk_idx, self.topk_w, self.inv, self.y, self.h, self.x
        return per_token if len(self.y) == T else tuple(t[:T] for t in per_token)


def serve_weights(w):
    """The block's weights with the experts' in 4 bits: "w1", "w3", "w2" become (data, scales)."""
    return dict(w, **{name: mx4_weights(w[name]) for name in ("w1", "w3", "w2")})


def run_block_serve(wl, w, h, x, buf: MoeServeBuffers, eps: float = 1e-6):
    """w: serve_weights; h, x of as many tokens as the buffers are for, or fewer.  -> the first rows of buf.h, buf.x"""
    logits, topk_idx, topk_w, inv, y, h_out, x_out = buf.of_tokens(x.shape[0])
    B.moe_router_fwd(x, w["wr"], logits, buf.ws_router)
    B.moe_route(logits, wl.k, wl.gate_mode, wl.e_lo, wl.e_cnt, topk_idx, topk_w, buf.counts)
    B.moe_dispatch(x, wl.k, topk_idx, None, wl.e_lo, wl.e_cnt, buf.offsets, buf.perm, inv, False, buf.xp, buf.ws_dispatch)
    B.moe_mx4_expert_fwd(buf.xp, buf.offsets, *w["w1"], *w["w3"], *w["w2"], buf.o, buf.ws_experts)
    B.moe_combine(buf.o, inv, topk_w, y)
    B.moe_block_norm_fwd(y, None, w["w_post"], True, h, w["w_pre"], 1.0, 1.0, eps, h_out, x_out)
