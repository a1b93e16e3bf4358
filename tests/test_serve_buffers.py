"""Buffers for serving have room for every number of tokens up to theirs."""
import pytest

from paper_2605_11005_amd import binding as B
from paper_2605_11005_amd import block as K
from paper_2605_11005_amd import workloads as W


@pytest.mark.parametrize("T,d,E,k", [(0, 256, 64, 4), (1, 256, 64, 4), (4164, 256, 64, 4), (5134, 256, 64, 4), (2500, 2048, 128, 8)])
def test_workspaces_for_fewer_tokens(T, d, E, k):
    wl = W.QWEN.scaled(name="serve-room", T=T, d=d, f=96, E=E, e_lo=0, e_cnt=8, k=k)
    cap = max(T, 1)
    buf = K.MoeServeBuffers(wl, cap, device="cpu")
    for t in range(T + 1):
        for which, n, ws in ((B.WS_ROUTER, E, buf.ws_router), (B.WS_DISPATCH, 8, buf.ws_dispatch), (B.WS_MX4_EXPERT_FWD, 8, buf.ws_experts)):
            assert B.moe_workspace_bytes(which, B.MOE_BF16, t, k, d, wl.f, n, cap) <= ws.numel(), (t, which)
