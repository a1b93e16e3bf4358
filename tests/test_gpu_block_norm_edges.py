"""The block norms where sizes and values are at their edges: NaN in the sums over rows, rows beyond one launch's, four blocks on a CU.

Bounds, set before the first run.  Column sums: a block adds at most T/256 + 1 rows one after the other, and at most 1024/16 + 16 blocks' sums follow;
each product is a chain of some twenty fp32 operations with 1/rms factors of trees over d: (T/256 + 200) * 2^-24 * sum |terms|."""
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


@pytest.mark.parametrize("dt,rt", [(BF16, BF16), (BF16, F32), (F32, F32)])
def test_rows_of_zeros_with_a_small_eps(dt, rt):
    """1/rms is 1e15 there, and its cube no number of fp32: what it multiplies is zero."""
    T, d, eps = 5, 136, 1e-30
    g = torch.Generator().manual_seed(4)
    r = lambda *s, dtype=dt: torch.randn(s, generator=g).to(dtype).cuda()  # noqa: E731
    y, h, w_post, w_pre, dn, dh_out = r(T, d), r(T, d, dtype=rt), r(d), r(d), r(T, d), r(T, d, dtype=rt)
    y[1] = 0
    y[3], h[3] = 0, 0
    h_out, n, dh, dy = torch.empty_like(h), torch.empty_like(y), torch.empty_like(h), torch.empty_like(y)
    r_post, r_pre, dgate = (torch.empty(T, device="cuda") for _ in range(3))
    dw_post, dw_pre = torch.empty_like(w_post), torch.empty_like(w_pre)
    B.moe_block_norm_fwd(y, None, w_post, True, h, w_pre, 0.5, 1.5, eps, h_out, n, r_post, r_pre)
    B.moe_block_norm_bwd(y, None, w_post, True, h_out, w_pre, r_post, r_pre, dh_out, dn, 0.5, 1.5, dh, dy, dgate, dw_post, dw_pre, False, workspace(T, d))
    ref, mag = N.bwd(host(y), None, host(w_post), True, host(h_out), host(w_pre), host(r_post), host(r_pre), host(dh_out), host(dn), 0.5, 1.5)
    half = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
    for name, got in (("dh", dh), ("dy", dy), ("dgate", dgate), ("dw_post", dw_post), ("dw_pre", dw_pre)):
        assert torch.isfinite(got).all(), name
        over = np.abs(host(got) - ref[name]) - (half[got.dtype] * np.abs(ref[name]) * (1 + 2.0 ** -7) + 200 * 2.0 ** -24 * mag[name])
        assert (over <= 0).all(), (name, float(over.max()))


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


@pytest.mark.parametrize("T,d,dt,rt", [(8200, 1408, BF16, BF16), (8193, 2048, BF16, F32), (8200, 1544, BF16, F32), (8192, 1032, BF16, F32)])
def test_four_blocks_on_a_cu(T, d, dt, rt):
    print(f"case norm {T} {d} {dt} {rt}", flush=True)
    g = torch.Generator().manual_seed(d)
    r = lambda *s, dtype=dt: torch.randn(s, generator=g).to(dtype).cuda()  # noqa: E731
    y, h, w_post, w_pre, dn, dh_out = r(T, d), r(T, d, dtype=rt), r(d), r(d), r(T, d), r(T, d, dtype=rt)
    h_out, n, dh, dy = torch.empty_like(h), torch.empty_like(y), torch.empty_like(h), torch.empty_like(y)
    r_post, r_pre, dgate, gate = (torch.rand(T, generator=g).cuda() for _ in range(4))
    dw_post, dw_pre = torch.empty_like(w_post), torch.empty_like(w_pre)
    B.moe_block_norm_fwd(y, gate, w_post, True, h, w_pre, 0.5, 1.5, EPS, h_out, n, r_post, r_pre)
    B.moe_block_norm_bwd(y, gate, w_post, True, h_out, w_pre, r_post, r_pre, dh_out, dn, 0.5, 1.5, dh, dy, dgate, dw_post, dw_pre, False, workspace(T, d))
    ref, mag = N.bwd(host(y), host(gate), host(w_post), True, host(h_out), host(w_pre), host(r_post), host(r_pre), host(dh_out), host(dn), 0.5, 1.5)
    half = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
    for name, got, steps in (("dh", dh, 100), ("dy", dy, 100), ("dgate", dgate, 100), ("dw_post", dw_post, T / 256 + 200), ("dw_pre", dw_pre, T / 256 + 200)):
        over = np.abs(host(got) - ref[name]) - (half[got.dtype] * np.abs(ref[name]) * (1 + 2.0 ** -7) + steps * 2.0 ** -24 * mag[name])
        assert (over <= 0).all(), (name, float(over.max()))
