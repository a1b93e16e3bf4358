"""Microscaled 4-bit calls at the edges of their sizes, and experts beside other experts: whatever those get, a row's results are the same bits."""
import numpy as np
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


# ---- experts beside other experts
def weights(E, d, f, seed, order_shows=False):
    """order_shows: what the first third of a contraction adds the second takes back, and the last adds 2^-16 of it: the order of the sums, and
    where they are rounded, decides the results."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    raw = [torch.randn(E, *shape, generator=g, device="cuda").mul(shape[0] ** -0.5).to(BF16) for shape in ((d, f), (d, f), (f, d))]
    if order_shows:
        for w in raw:
            third = 32 * (w.shape[1] // 96)
            w[:, third:2 * third] = -w[:, :third]
            w[:, 2 * third:] *= 2.0 ** -16
        for w in raw[:2]:
            third = 32 * (f // 96)
            w[:, :, third:2 * third] = w[:, :, :third]
    return raw, [L.mx4_weights(w) for w in raw]


def forward(x, rows, q, cap=None):
    """o of the rows (expert after expert) with the experts' weights q, out of buffers of `cap` rows."""
    R, (cap, d), e = sum(rows), (cap or max(sum(rows), 1), x.shape[1]), len(rows)
    f = 16 * q[0][0].shape[1]
    xp = torch.full((cap, d), float("nan"), dtype=BF16, device="cuda")
    xp[:R] = x
    off = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32, device="cuda")
    o = torch.full_like(xp, float("nan"))
    ws = torch.full((B.moe_workspace_bytes(B.WS_MX4_EXPERT_FWD, B.MOE_BF16, 0, 0, d, f, e, cap),), 0xFF, dtype=torch.uint8, device="cuda")
    B.moe_mx4_expert_fwd(xp, off, *q[0], *q[1], *q[2], o, ws)
    assert torch.isnan(o[R:]).all()
    return o[:R]


def tokens(n, d, seed, order_shows=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, d, generator=g, device="cuda").mul(torch.exp(0.5 * torch.randn(d, generator=g, device="cuda"))).to(BF16)
    if order_shows:
        third = 32 * (d // 96)
        x[:, third:2 * third] = x[:, :third]
    return x


OTHERS = {"alone": [0] * 31, "one": [1] + [0] * 30, "three": [0, 5, 0, 2, 0, 1] + [0] * 25, "seven": [3] * 7 + [0] * 24, "fifteen": [2, 0] * 15 + [1],
          "all": [4] * 31, "more": [30] * 31, "large": [0] * 30 + [600], "mixed": [33, 1, 0] * 10 + [300], "larger": [700] * 4 + [20] * 27}


@pytest.mark.parametrize("d,f", [(4096, 1536), (7168, 2048), (2880, 1440), (768, 3328)])
@pytest.mark.parametrize("mine", [1, 16, 20, 45, 300])
def test_rows_of_other_experts_do_not_enter(mine, d, f):
    print(f"case mx4 beside others {mine} {d} {f}", flush=True)
    _, q = weights(32, d, f, d + f, order_shows=True)
    x = tokens(mine, d, mine, order_shows=True)
    want = {}
    for name, others in OTHERS.items():
        rest = tokens(sum(others), d, 9)
        # among the first, and among the last
        o = forward(torch.cat([x, rest]), [mine] + others, q)[:mine]
        assert torch.isfinite(o).all()
        last = forward(torch.cat([rest, x]), others + [mine], [tuple(t.roll(-1, 0) for t in w) for w in q])[sum(others):]
        wide = forward(torch.cat([x, rest]), [mine] + others, q, cap=mine + sum(others) + 900)[:mine]
        want[name] = o, last, wide
    differ = {(name, i): (o != want["alone"][0]).sum().item() for name, all_ in want.items() for i, o in enumerate(all_)}
    assert not any(differ.values()), {k: v for k, v in differ.items() if v}


def exact(x, raw, e):
    """Oracle of one expert, and what it may be off by."""
    host = lambda t: t.double().cpu().numpy()  # noqa: E731
    v = [M.values(*M.quantize(host(w[e]).T))[None] for w in raw]
    d = x.shape[1]
    return M.expert_fwd(host(x), np.array([0, len(x)]), *v, h_err=(d / 128 + 16) * 2.0 ** -23)


def check(o, x, rows, raw, experts):
    """Bound as for a few experts at a time: half a unit of bf16, the fp32 sums, activations near a halfway value."""
    off = np.concatenate([[0], np.cumsum(rows)])
    for e in experts:
        ref, slack = exact(x[off[e]:off[e + 1]], raw, e)
        got = o[off[e]:off[e + 1]].double().cpu().numpy()
        assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + slack + 1e-5 * np.abs(ref).max()).all(), e
        assert np.linalg.norm(got - ref) <= 6e-3 * np.linalg.norm(ref), e


def fits_the_cache(d, f):
    """Experts whose weights in 4 bits fit 256 MB: with more, weights are loaded with the hint that they are used once."""
    return (256 << 20) * 32 // (51 * d * f)


MANY = {
    # every expert a stream of few rows
    "few": ([1, 2, 3] * 24, [0, 41, 71]),
    "up to 32": ([32, 17, 5, 1] * 18, [0, 1, 70]),
    # large experts among the first 64 and behind them, few of them
    "large behind 64": ([3] * 66 + [300, 40, 257, 33, 128, 1], [5, 66, 69, 71]),
    # so many streams that the workgroups with a large tile take some too
    "both": ([31] * 64 + [300] * 4 + [20] * 4, [0, 64, 67, 70]),
    # every large tile's weights are read once
    "one tile each": ([33, 64, 65, 128, 129, 256] * 12, [0, 33, 68, 71]),
    # and several times
    "several tiles each": ([300, 513] * 36, [0, 71]),
}


@pytest.mark.parametrize("name", MANY)
def test_more_experts_than_the_cache_holds(name):
    d, f = 2048, 1408
    rows, looked_at = MANY[name]
    E = len(rows)
    assert E > fits_the_cache(d, f)
    print(f"case mx4 many experts {name}", flush=True)
    raw, q = weights(E, d, f, 7)
    x = tokens(sum(rows), d, 8)
    o = forward(x, rows, q, cap=sum(rows) + 5)
    off = np.concatenate([[0], np.cumsum(rows)])
    for e in range(0, E, 6):                    # six at a time, as the cache holds them
        part = forward(x[off[e]:off[e + 6]], rows[e:e + 6], [tuple(t[e:e + 6] for t in w) for w in q])
        assert torch.equal(part, o[off[e]:off[e + 6]]), e
    check(o, x, rows, raw, looked_at)


@pytest.mark.parametrize("rows", [[1] * 32, [1] * 28 + [4]])
def test_few_rows_in_all_of_more_experts_than_the_cache_holds(rows):
    d, f = 4096, 1536
    E = len(rows)
    assert E > fits_the_cache(d, f) and sum(rows) <= 32
    raw, q = weights(E, d, f, 9)
    x = tokens(sum(rows), d, 10)
    o = forward(x, rows, q)
    assert torch.equal(forward(x, rows, q, cap=200), o)
    check(o, x, rows, raw, [0, E - 1])
