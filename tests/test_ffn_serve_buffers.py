"""Buffers of the block of two-matrix experts that serve have room for every number of tokens up to theirs."""
import pytest

from paper_2605_11005_amd import binding as B
from paper_2605_11005_amd import ffn_block as F
from paper_2605_11005_amd import workloads as W


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("T,d,E,k", [(0, 256, 64, 4), (1, 256, 64, 4), (4164, 256, 64, 4), (5134, 256, 64, 4), (2500, 2048, 128, 8)])
def test_workspace_for_fewer_tokens(T, d, E, k, dtype):
    wl = W.QWEN.scaled(name="ffn-room", T=T, d=d, f=96, E=E, e_lo=0, e_cnt=8, k=k, dtype=dtype)
    cap, shared, code = max(T, 1), 520, B.MOE_BF16 if dtype == "bf16" else B.MOE_F32
    room = F.FfnBlockBuffers(wl, cap, shared, grads=False, device="cpu").ws.numel()
    for t in range(T + 1):
        for which, *sizes in ((B.WS_ROUTER, t, k, d, 96, E, cap), (B.WS_DISPATCH, t, k, d, 96, 8, cap), (B.WS_LINEAR_FWD, 0, 0, d, shared, 1, t),
                              (B.WS_LINEAR_FWD, 0, 0, shared, d, 1, t), (B.WS_LINEAR_FWD, 0, 0, d, 96, 8, cap), (B.WS_LINEAR_FWD, 0, 0, 96, d, 8, cap)):
            assert B.moe_workspace_bytes(which, code, *sizes) <= room, (t, which)
