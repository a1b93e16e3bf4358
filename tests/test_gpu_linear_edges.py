"""The linear layer where values and sizes are unusual, against float64.  Bounds stand at each test, set before its first run."""
import numpy as np
import pytest
import torch

from oracle import linear_oracle as L
from paper_2605_11005_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def code(dt):
    return B.MOE_BF16 if dt == BF16 else B.MOE_F32


@pytest.mark.parametrize("rows", [3, 200])
def test_gelu_far_below_zero_keeps_its_digits(rows):
    """gelu(z) = z erfc(-z / sqrt 2) / 2 for z down to -12.5, where it is 5e-35: by what fraction it is off, in bf16, besides its rounding.  erfc is off by
    6e-5 (2^-14) of itself; exp2 takes an argument of up to 113 that two products rounded, 113 log(2) 2^-23 = 2^-16.7; the rest is a few 2^-24.  Together
    less than 2^-13.  What is rounded to bf16 is off by 2^-8 of the value."""
    z = torch.cat([-torch.arange(0, 12.5, 0.0625), torch.arange(0, 12.5, 0.0625)]).to(BF16)      # (each of them a bf16 number)
    n = len(z)
    x, w = torch.zeros(rows, 16, dtype=BF16, device="cuda"), torch.zeros(16, n, dtype=BF16, device="cuda")
    y, zz, bias = torch.empty(rows, n, dtype=BF16, device="cuda"), torch.empty(rows, n, dtype=BF16, device="cuda"), z.cuda()
    ws = torch.empty(B.moe_workspace_bytes(B.WS_LINEAR_FWD, B.MOE_BF16, 0, 0, 16, n, 1, rows), dtype=torch.uint8, device="cuda")
    B.moe_linear_fwd(x, None, w, bias, B.ACT_GELU, None, zz, y, ws)
    assert torch.equal(zz, bias.expand(rows, n))
    z, y = z.double().numpy(), y.double().cpu().numpy()
    ref = L.act(z, "gelu")
    off = np.abs(y - ref)
    bad = ~(off <= (2.0 ** -8 + 2.0 ** -13 + 2.0 ** -21) * np.abs(ref))
    assert not bad.any(), (z[bad.any(0)], (off / np.maximum(np.abs(ref), 1e-300)).max())


def fp32_products(x, w, dy):
    rows, K, N = *x.shape, w.shape[1]
    new = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    y, dx, dw = new(rows, N), new(rows, K), new(K, N)
    ws = torch.empty(max(B.moe_workspace_bytes(which, B.MOE_F32, 0, 0, K, N, 1, rows) for which in (B.WS_LINEAR_FWD, B.WS_LINEAR_BWD)), dtype=torch.uint8,
                     device="cuda")
    B.moe_linear_fwd(x, None, w, None, B.ACT_NONE, None, None, y, ws)
    B.moe_linear_bwd(x, None, dy, None, w, B.ACT_NONE, dx, dw, None, False, ws)
    return y, dx, dw


def test_fp32_infinities_do_not_show_in_the_other_tile_of_a_pair():
    """4200 rows of 136 to 2060 take tiles of 128 columns, two of 64 beside each other.  What an infinite weight or gradient makes infinite is formed again
    from the operands: all other outputs keep their bits."""
    g = torch.Generator().manual_seed(2)
    r = lambda *s: (torch.rand(s, generator=g) + 0.5).cuda()  # noqa: E731
    x, w, dy = r(4200, 136), r(136, 2060), r(4200, 2060)
    y, dx, dw = fp32_products(x, w, dy)
    infinite = w.clone()
    infinite[5, 3] = float("inf")             # column 3 of y, column 5 of dx
    y2, dx2, _ = fp32_products(x, infinite, dy)
    others = lambda t, at: torch.cat([t[:, :at], t[:, at + 1:]], 1)  # noqa: E731
    assert torch.isposinf(y2[:, 3]).all() and torch.equal(others(y, 3), others(y2, 3))
    assert torch.isposinf(dx2[:, 5]).all() and torch.equal(others(dx, 5), others(dx2, 5))
    infinite = dy.clone()
    infinite[7, 100] = float("inf")           # column 100 of dw, row 7 of dx
    _, dx3, dw3 = fp32_products(x, w, infinite)
    assert torch.isposinf(dw3[:, 100]).all() and torch.equal(others(dw, 100), others(dw3, 100))
    assert torch.isposinf(dx3[7]).all() and torch.equal(dx[:7], dx3[:7]) and torch.equal(dx[8:], dx3[8:])
