"""The block norms with NaN and infinities in the sums over rows, and with more rows than one launch holds."""
import numpy as np
import pytest
import torch

from oracle import norm_oracle as N
from paper_2605_11005_amd import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-6
BF16, F32 = torch.bfloat16, torch.float32


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def workspace(T, d):
    return torch.full((B.moe_workspace_bytes(B.WS_BLOCK_NORM, 0, T, 0, d, 0, 0, 0),), 0xFF, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("bits", [0x7FFFFFFF, 0xFFFFFFFF, 0x7FC00000, 0x7F800001, 0x7F800000, 0xFF800000])
def test_sums_over_rows_keep_nan_and_infinities(bits, accumulate):
    """bf16 blocks on an fp32 residual stream, whose NaN may have any payload."""
    T, d = 9, 72
    g = torch.Generator().manual_seed(1)
    r = lambda *s, dtype=BF16: torch.randn(s, generator=g).to(dtype)  # noqa: E731
    y, w_post, w_pre, h, dn, dh_out = r(T, d), r(d), r(d), r(T, d, dtype=F32), r(T, d), r(T, d, dtype=F32)
    value = torch.tensor([bits - (1 << 32) if bits >> 31 else bits], dtype=torch.int32).view(F32)
    h.view(torch.int32)[2, 11] = value.view(torch.int32)[0]
    dh_out.view(torch.int32)[5, 30] = value.view(torch.int32)[0]
    r_pre, ws = torch.ones(T, device="cuda"), workspace(T, d)
    dw_post, dw_pre = torch.ones(d, dtype=BF16, device="cuda"), torch.ones(d, dtype=BF16, device="cuda")
    dh, dy = torch.empty(T, d, device="cuda"), torch.empty(T, d, dtype=BF16, device="cuda")
    B.moe_block_norm_bwd(y.cuda(), None, w_post.cuda(), False, h.cuda(), w_pre.cuda(), None, r_pre, dh_out.cuda(), dn.cuda(), 1.0, 1.0, dh, dy, None,
                         dw_post, dw_pre, accumulate, ws)
    with np.errstate(invalid="ignore"):
        ref, _ = N.bwd(host(y), None, host(w_post), False, host(h), host(w_pre), None, host(r_pre), host(dh_out), host(dn), 1.0, 1.0)
    for name, got in (("dw_pre", dw_pre), ("dw_post", dw_post)):
        got, want = host(got), ref[name]
        assert not np.isfinite(want).all()
        assert np.array_equal(np.isnan(got), np.isnan(want)), (name, got, want)
        inf = np.isinf(want)
        assert np.array_equal(got[inf], want[inf]) and np.isfinite(got[np.isfinite(want)]).all(), name


def test_more_rows_than_a_launch_holds():
    """2^28 rows of one wavefront each are 2^32 work-items."""
    T, d, part = (1 << 28) + 5, 8, 1 << 24
    if torch.cuda.mem_get_info()[0] < 4 * T * d * 2:
        pytest.skip("not enough device memory")
    h, w = torch.empty(T, d, dtype=BF16, device="cuda"), torch.linspace(0.5, 2, d, device="cuda").to(BF16)
    g = torch.Generator(device="cuda").manual_seed(2)
    for lo in range(0, T, part):
        h[lo:lo + part].normal_(generator=g)
    n, r_pre = torch.full_like(h, float("nan")), torch.full((T,), float("nan"), device="cuda")
    B.moe_block_norm_fwd(None, None, None, False, h, w, 1.0, 1.0, EPS, None, n, None, r_pre)
    for lo in range(0, T, part):
        v = h[lo:lo + part].float()
        r = (v.square().mean(1, keepdim=True) + EPS).rsqrt()
        ref = v * r * w.float()
        assert ((r_pre[lo:lo + part] / r[:, 0] - 1).abs() <= 1e-5).all(), lo
        assert ((n[lo:lo + part].float() - ref).abs() <= 2.0 ** -8 * 1.01 * ref.abs() + 1e-30).all(), lo
