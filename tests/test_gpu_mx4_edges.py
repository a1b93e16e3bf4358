"""Microscaled 4-bit calls of more workgroups than one launch holds."""
import pytest
import torch

from oracle import mx4_oracle as M
from paper_2605_11005_amd import binding as B
from paper_2605_11005_amd import layer as L

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


def test_experts_of_more_tiles_than_one_launch():
    d, f, part, cap = 32, 32, 1 << 20, (1 << 28) + 160          # a workgroup for 16 rows
    need(90)
    g = torch.Generator(device="cuda").manual_seed(4)
    w = [t for shape in ((d, f), (d, f), (f, d)) for t in L.mx4_weights(torch.randn(2, *shape, generator=g, device="cuda").to(BF16))]
    x1 = torch.randn(part, d, generator=g, device="cuda").to(BF16)
    o1 = torch.empty_like(x1)
    ws = torch.empty(B.moe_workspace_bytes(B.WS_MX4_EXPERT_FWD, B.MOE_BF16, 0, 0, d, f, 2, cap), dtype=torch.uint8, device="cuda")
    offsets = lambda first, last: torch.tensor([0, first, last], dtype=torch.int32, device="cuda")  # noqa: E731
    B.moe_mx4_expert_fwd(x1, offsets(part, part), *w, o1, ws)
    x = torch.cat([x1] * (cap // part) + [x1[:cap % part]])
    o = torch.full_like(x, float("nan"))
    B.moe_mx4_expert_fwd(x, offsets(cap - 60, cap - 3), *w, o, ws)
    assert same(part, o[:cap - 60], o1) and torch.isnan(o[cap - 3:]).all()
    last = torch.empty_like(o[:57])
    B.moe_mx4_expert_fwd(x[cap - 60:cap - 3], offsets(0, 57), *w, last, ws)
    assert torch.equal(o[cap - 60:cap - 3], last)
