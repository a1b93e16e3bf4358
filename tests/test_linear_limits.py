"""What the linear layer and the layer norm refuse before they launch anything, and their workspaces' sizes."""
import ctypes

import pytest
import torch

from paper_2605_11005_amd import binding as B

EINVAL, EUNSUPPORTED, EWORKSPACE = 1, 2, 3
P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4104)
MB = 1 << 40


def fwd(x=P, dtype=B.MOE_BF16, cap=4, K=16, N=8, e_cnt=2, offsets=P, w=P, bias=P, act=0, residual=P, z=P, y=P, ws=P, ws_bytes=MB):
    return B.load_library().moe_linear_fwd(x, dtype, cap, K, N, e_cnt, offsets, w, bias, act, residual, z, y, ws, ws_bytes, None)


def bwd(x=P, z=P, dy=P, dtype=B.MOE_BF16, cap=4, K=16, N=8, e_cnt=2, offsets=P, w=P, act=2, dx=P, dw=P, db=P, accumulate=0, ws=P, ws_bytes=MB,
        dx_accumulate=0):
    return B.load_library().moe_linear_bwd(x, z, dy, dtype, cap, K, N, e_cnt, offsets, w, act, dx, dx_accumulate, dw, db, accumulate, ws, ws_bytes, None)


@pytest.mark.parametrize("call", (fwd, bwd))
@pytest.mark.parametrize("args,code", [
    (dict(dtype=2), EINVAL), (dict(cap=-1), EINVAL), (dict(K=0), EINVAL), (dict(N=-8), EINVAL), (dict(e_cnt=-1), EINVAL), (dict(act=-1), EINVAL),
    (dict(act=5), EINVAL), (dict(offsets=None), EINVAL), (dict(w=None), EINVAL), (dict(x=None), EINVAL), (dict(x=ODD), EINVAL), (dict(w=ODD), EINVAL),
    (dict(z=ODD), EINVAL), (dict(e_cnt=1025), EUNSUPPORTED), (dict(K=12), EUNSUPPORTED), (dict(N=20), EUNSUPPORTED),
    (dict(dtype=B.MOE_F32, K=18), EUNSUPPORTED), (dict(K=(1 << 20) + 8), EUNSUPPORTED), (dict(cap=1 << 30, N=8), EUNSUPPORTED),
    (dict(cap=1 << 22, K=64, N=1 << 14), EUNSUPPORTED), (dict(e_cnt=1024, K=1 << 13, N=1 << 13), EUNSUPPORTED),
    (dict(ws=None), EWORKSPACE), (dict(ws=ODD), EWORKSPACE), (dict(ws_bytes=16), EWORKSPACE)])
def test_linear_refuses(call, args, code):
    assert call(**args) == code


def test_linear_refuses_one_way():
    assert fwd(y=None) == EINVAL and fwd(y=ODD) == EINVAL and fwd(bias=ODD) == EINVAL and fwd(residual=ODD) == EINVAL
    assert bwd(dy=None) == EINVAL and bwd(z=None) == EINVAL and bwd(accumulate=2) == EINVAL and bwd(dx_accumulate=-1) == EINVAL and bwd(dx=ODD) == EINVAL and bwd(dw=ODD) == EINVAL
    # nothing to do: no launch
    assert fwd(cap=0, x=None, y=None) == 0 and fwd(e_cnt=0, w=None) == 0 and bwd(e_cnt=0) == 0


def test_linear_workspaces_grow():
    for dtype in (B.MOE_F32, B.MOE_BF16):
        for which in (B.WS_LINEAR_FWD, B.WS_LINEAR_BWD):
            sizes = [B.moe_workspace_bytes(which, dtype, 0, 0, 64, 128, 4, cap) for cap in (0, 1, 63, 64, 65, 1000, 1 << 20)]
            assert sizes == sorted(sizes) and sizes[0] >= 256
        assert B.moe_workspace_bytes(B.WS_LINEAR_BWD, dtype, 0, 0, 64, 128, 4, 1000) >= 1000 * 128 * (2 if dtype == B.MOE_BF16 else 4)


def norm_fwd(y=P, h=P, w=P, b=P, dtype=B.MOE_BF16, res=B.MOE_F32, T=4, d=64, eps=1e-5, h_out=P, n=P, mean=P, rstd=P):
    return B.load_library().moe_layer_norm_fwd(y, h, w, b, dtype, res, T, d, eps, h_out, n, mean, rstd, None)


def norm_bwd(h=P, w=P, mean=P, rstd=P, dh_out=P, dn=P, dtype=B.MOE_BF16, res=B.MOE_F32, T=4, d=64, dh=P, dy=P, dw=P, db=P, accumulate=0, ws=P,
             ws_bytes=MB):
    return B.load_library().moe_layer_norm_bwd(h, w, mean, rstd, dh_out, dn, dtype, res, T, d, dh, dy, dw, db, accumulate, ws, ws_bytes, None)


@pytest.mark.parametrize("call", (norm_fwd, norm_bwd))
@pytest.mark.parametrize("args,code", [
    (dict(dtype=3), EINVAL), (dict(dtype=B.MOE_F32, res=B.MOE_BF16), EINVAL), (dict(T=-1), EINVAL), (dict(d=0), EINVAL), (dict(h=None), EINVAL),
    (dict(h=ODD), EINVAL), (dict(w=ODD), EINVAL), (dict(d=12), EUNSUPPORTED), (dict(dtype=B.MOE_F32, d=6), EUNSUPPORTED),
    (dict(d=16392), EUNSUPPORTED), (dict(T=0x7FFF0001), EUNSUPPORTED)])
def test_layer_norm_refuses(call, args, code):
    assert call(**args) == code


def test_layer_norm_refuses_one_way():
    inf, nan = float("inf"), float("nan")
    for eps in (0.0, -1e-5, inf, nan):
        assert norm_fwd(eps=eps) == EINVAL
    assert norm_fwd(n=None) == EINVAL and norm_fwd(y=None) == EINVAL and norm_fwd(n=ODD) == EINVAL and norm_fwd(b=ODD) == EINVAL
    assert norm_bwd(dn=None) == EINVAL and norm_bwd(mean=None) == EINVAL and norm_bwd(rstd=None) == EINVAL and norm_bwd(accumulate=-1) == EINVAL
    assert norm_bwd(ws=None) == EWORKSPACE and norm_bwd(ws=ODD) == EWORKSPACE and norm_bwd(ws_bytes=64) == EWORKSPACE
    assert norm_fwd(T=0, y=None, h=None, n=None) == 0


def test_layer_norm_workspace_grows_with_the_rows():
    for d in (8, 512, 1024, 2048, 8192, 16384):
        sizes = [B.moe_workspace_bytes(B.WS_LAYER_NORM, 0, T, 0, d, 0, 0, 0) for T in (0, 1, 5, 511, 512, 513, 2048, 4096, 8191, 8192, 1 << 20)]
        assert sizes == sorted(sizes)


def test_tensors_that_are_not_what_they_should_be():
    """Host tensors, or shapes that do not fit, are named before anything is called."""
    t = torch.zeros((4, 8), dtype=torch.bfloat16)
    with pytest.raises(B.MoeError, match="weights"):
        B.moe_linear_fwd(t, None, torch.zeros((1, 8, 8), dtype=torch.bfloat16), None, 0, None, None, t, t)
    with pytest.raises(B.MoeError, match="weights"):
        B.moe_linear_fwd(t, torch.zeros(2, dtype=torch.int32), t, None, 0, None, None, t, t)
    with pytest.raises(B.MoeError, match="device tensor"):
        B.moe_linear_fwd(t, None, torch.zeros((8, 8), dtype=torch.bfloat16), None, 0, None, None, t, t)
    with pytest.raises(B.MoeError, match="device tensor"):
        B.moe_layer_norm_fwd(None, t, None, None, 1e-5, None, t)
