"""Microscaled 4-bit calls of more workgroups than one launch holds."""
import pytest
import torch

from oracle import mx4_oracle as M
from paper_2605_11005_amd import binding as B

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def need(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes * 2 ** 30:
        pytest.skip("not enough device memory")


def same(parts, whole, part):
    """whole is `part` again and again"""
    for lo in range(0, len(whole), parts):
        if not torch.equal(whole[lo:lo + parts], part[:len(whole) - lo]):
            return False
    return True


# ---- more workgroups of 256 threads than one launch holds (2^24)
def test_weights_beyond_one_launch():
    n, K, part, batch = 8, 32, 1 << 20, (1 << 22) + 77          # four workgroups each
    need(12)
    g = torch.Generator(device="cuda").manual_seed(1)
    x1 = torch.randn(part, K, n, generator=g, device="cuda").to(BF16)
    q1, s1 = (torch.empty((part,) + shape, dtype=torch.uint8, device="cuda") for shape in B.mx4_shapes(n, K))
    B.moe_mx4_quantize(x1, True, q1, s1)
    x = torch.cat([x1] * (batch // part) + [x1[:batch % part]])
    q, s = (torch.full((batch,) + shape, 0xA5, dtype=torch.uint8, device="cuda") for shape in B.mx4_shapes(n, K))
    B.moe_mx4_quantize(x, True, q, s)
    assert same(part, q, q1) and same(part, s, s1)


def test_values_beyond_one_launch():
    n, K, part, batch = 1, 32, 1 << 20, (1 << 24) + 77          # a workgroup each
    need(28)
    g = torch.Generator(device="cuda").manual_seed(2)
    x1 = torch.randn(part, n, K, generator=g, device="cuda").to(BF16)
    q1, s1 = (torch.empty((part,) + shape, dtype=torch.uint8, device="cuda") for shape in B.mx4_shapes(n, K))
    B.moe_mx4_quantize(x1, False, q1, s1)
    v1 = torch.empty_like(x1)
    B.moe_mx4_dequantize(q1, s1, v1)
    assert (v1[:100, 0].double().cpu().numpy() == M.values(*M.quantize(x1[:100, 0].double().cpu().numpy()))).all()
    q, s = (torch.cat([t] * (batch // part) + [t[:batch % part]]) for t in (q1, s1))
    v = torch.full((batch, n, K), float("nan"), dtype=BF16, device="cuda")
    B.moe_mx4_dequantize(q, s, v)
    assert same(part, v, v1)


def test_rows_beyond_one_launch():
    n, K, part, batch = 1, 32, 1 << 20, (1 << 26) + 77          # a workgroup for four
    need(100)
    g = torch.Generator(device="cuda").manual_seed(3)
    x1 = torch.randn(part, n, K, generator=g, device="cuda").to(BF16)
    q1, s1 = (torch.empty((part,) + shape, dtype=torch.uint8, device="cuda") for shape in B.mx4_shapes(n, K))
    B.moe_mx4_quantize(x1, False, q1, s1)
    x = torch.cat([x1] * (batch // part) + [x1[:batch % part]])
    q, s = (torch.full((batch,) + shape, 0xA5, dtype=torch.uint8, device="cuda") for shape in B.mx4_shapes(n, K))
    B.moe_mx4_quantize(x, False, q, s)
    assert same(part, q, q1) and same(part, s, s1)
