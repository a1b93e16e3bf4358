"""Microscaled 4-bit numbers against the oracle, through the binding: codes, scales and values equal bit for bit; the experts' forward within a
bound that is set before the first run: half a unit of bf16, the fp32 sums' error, and what the activations that lie within the
products' error of a halfway value can do (oracle.mx4_oracle.expert_fwd)."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as M
from paper_2605_11005_amd import binding as B
from paper_2605_11005_amd import layer as L

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def poisoned(shape):
    return torch.full(tuple(shape), 0xA5, dtype=torch.uint8, device="cuda")


def wild(n, K, dt, seed):
    """Magnitudes over the whole range of exponents, a chunk's within a few binades of each other; zeros, halfway values."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, K, generator=g) * torch.exp2(torch.randint(-130, 120, (n, K // 32), generator=g).float()).repeat_interleave(32, 1)
    x[torch.rand(n, K, generator=g) < 0.1] = 0
    if n > 2:
        x[0, :32] = torch.tensor([0.25, .75, 1.25, 1.75, 2.5, 3.5, 5, 7, -5, .2, 0, -.1, -.25, -.75, 6, -6] + [4.] * 16)
        x[1] = 0
        x[2, -32:] = 1e-45
    return x.to(dt)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("n,K", [(1, 32), (3, 64), (16, 512), (17, 544), (40, 1120), (200, 160), (257, 2880)])
@pytest.mark.parametrize("along_rows", [False, True])
def test_codes_scales_and_values(n, K, dt, along_rows):
    if along_rows:
        n = -(-n // 8) * 8
    print(f"case mx4 {n} {K} {dt} {along_rows}", flush=True)
    x = wild(n, K, dt, n + K)
    codes, scales = M.quantize(x.double().numpy())
    want = M.tiles(codes, scales)
    q, s = (poisoned(shape) for shape in B.mx4_shapes(n, K))
    B.moe_mx4_quantize((x.t().contiguous() if along_rows else x).cuda(), along_rows, q, s)
    assert (s.cpu().numpy() == want[1]).all() and (q.cpu().numpy() == want[0]).all()
    for out_dt in (BF16, F32):
        v = torch.full((n, K), float("nan"), dtype=out_dt, device="cuda")
        B.moe_mx4_dequantize(q, s, v)
        assert (v.double().cpu().numpy() == M.values(codes, scales)).all()


def test_batches_equal_their_matrices():
    x = torch.stack([wild(264, 96, BF16, i).t() for i in range(3)]).contiguous().cuda()
    q, s = (poisoned((3,) + shape) for shape in B.mx4_shapes(264, 96))
    B.moe_mx4_quantize(x, True, q, s)
    v = torch.empty(3, 264, 96, dtype=F32, device="cuda")
    B.moe_mx4_dequantize(q, s, v)
    for i in range(3):
        q1, s1 = (poisoned(shape) for shape in B.mx4_shapes(264, 96))
        B.moe_mx4_quantize(x[i].t().contiguous(), False, q1, s1)
        assert torch.equal(q[i], q1) and torch.equal(s[i], s1)
        assert (v[i].double().cpu().numpy() == M.values(*M.quantize(x[i].t().double().cpu().numpy()))).all()
    empty = torch.empty(0, 64, dtype=BF16, device="cuda")
    B.moe_mx4_quantize(empty, False, *(poisoned(shape) for shape in B.mx4_shapes(0, 64)))


@pytest.mark.parametrize("along_rows", [False, True])
def test_infinities_and_nan_spoil_their_chunk_only(along_rows):
    x = torch.randn(24, 192).to(BF16)
    x[3, 40], x[9, 130], x[9, 131] = float("nan"), float("inf"), float("-inf")
    q, s = (poisoned(shape) for shape in B.mx4_shapes(24, 192))
    B.moe_mx4_quantize((x.t().contiguous() if along_rows else x).cuda(), along_rows, q, s)
    v = torch.empty(24, 192, dtype=BF16, device="cuda")
    B.moe_mx4_dequantize(q, s, v)
    want = M.values(*M.quantize(x.double().numpy()))
    assert np.isnan(want).sum() == 64 and np.array_equal(v.double().cpu().numpy(), want, equal_nan=True)


# ---- experts
def make(rows, d, f, seed=0, cap=None):
    g = torch.Generator().manual_seed(seed)
    e = len(rows)
    R = sum(rows)
    off = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32)
    cap = R if cap is None else cap
    xp = (torch.randn(cap, d, generator=g) * torch.exp(0.5 * torch.randn(d, generator=g))).to(BF16)
    w = [torch.randn(e, *shape, generator=g).mul(shape[0] ** -0.5).to(BF16) for shape in ((d, f), (d, f), (f, d))]
    return xp, off, w


def run(xp, off, w, poison=True):
    q = [L.mx4_weights(t.cuda()) for t in w]
    (cap, d), f, e = xp.shape, w[0].shape[2], w[0].shape[0]
    ws = torch.full((B.moe_workspace_bytes(B.WS_MX4_EXPERT_FWD, B.MOE_BF16, 0, 0, d, f, e, cap),), 0xFF if poison else 0, dtype=torch.uint8, device="cuda")
    o = torch.full((cap, d), float("nan"), dtype=BF16, device="cuda")
    B.moe_mx4_expert_fwd(xp.cuda(), off.cuda(), *q[0], *q[1], *q[2], o, ws)
    torch.cuda.synchronize()
    return o, q, ws


def check(xp, off, w, o):
    R, (d, f) = int(off[-1]), w[0].shape[1:]
    v = [np.stack([M.values(*M.quantize(m.double().numpy().T)) for m in t]) for t in w]
    # fp32 sums of K exact products: K/128 + 8 roundings of partial sums no larger than the terms' magnitudes together
    ref, slack = M.expert_fwd(xp[:R].double().numpy(), off.numpy(), *v, h_err=(d / 128 + 16) * 2.0 ** -23)
    got = o.double().cpu().numpy()
    assert np.isnan(got[R:]).all(), "rows past R are left untouched"
    got = got[:R]
    assert np.isfinite(got).all()
    over = np.abs(got - ref) - (2.0 ** -8 * np.abs(ref) + slack + 1e-5 * np.abs(ref).max())
    assert (over <= 0).all(), float(over.max())
    # the slack is an exception: nearly everything is as near as bf16 allows
    assert (np.linalg.norm(got - ref) <= 6e-3 * np.linalg.norm(ref)), np.linalg.norm(got - ref) / np.linalg.norm(ref)


@pytest.mark.parametrize("rows,d,f", [([1], 32, 32), ([0, 1, 0], 512, 64), ([3, 0, 16, 17], 160, 96), ([33, 1, 64], 544, 288), ([5, 130], 1056, 544),
                                      ([0, 0, 2, 300, 15, 31], 256, 1024), ([257, 512, 40], 640, 384), ([1] * 70 + [9], 128, 128),
                                      ([2] * 3, 4224, 160), ([700], 2880, 128)])
def test_experts(rows, d, f):
    print(f"case mx4 experts {rows} {d} {f}", flush=True)
    xp, off, w = make(rows, d, f, seed=d + f, cap=sum(rows) + 3)
    o, _, _ = run(xp, off, w)
    check(xp, off, w, o)


def test_experts_without_rows():
    xp, off, w = make([0, 0], 64, 64, cap=5)
    o, _, _ = run(xp, off, w)
    assert torch.isnan(o).all()
    xp, off, w = make([0, 0], 64, 64, cap=0)
    run(xp, off, w)


def test_capacity_and_old_contents_do_not_enter():
    rows, d, f = [20, 0, 70, 400], 768, 320
    xp, off, w = make(rows, d, f, seed=5, cap=2000)
    R = sum(rows)
    o, _, _ = run(xp, off, w)
    check(xp, off, w, o)
    again, _, _ = run(xp, off, w, poison=False)
    assert torch.equal(o[:R], again[:R])
    check(xp[:R], off, w, run(xp[:R].contiguous(), off, w)[0])


def test_a_row_of_nan_keeps_to_itself():
    rows, d, f = [18, 300], 256, 256
    xp, off, w = make(rows, d, f, seed=6)
    clean, _, _ = run(xp, off, w)
    xp[4, 10], xp[100, 200] = float("nan"), float("inf")
    o, _, _ = run(xp, off, w)
    bad = torch.zeros(sum(rows), dtype=torch.bool, device="cuda")
    bad[[4, 100]] = True
    assert torch.isnan(o[bad]).all() and torch.equal(o[~bad], clean[~bad])


def test_in_a_graph():
    xp, off, w = make([7, 0, 90, 33], 512, 384, seed=7)
    o, q, ws = run(xp, off, w)
    want = o.clone()
    x, offsets = xp.cuda(), off.cuda()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        B.moe_mx4_expert_fwd(x, offsets, *q[0], *q[1], *q[2], o, ws)
    for _ in range(3):
        o.fill_(float("nan"))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)


def test_refusals():
    x = torch.zeros(4, 64, dtype=BF16, device="cuda")
    q, s = (poisoned(shape) for shape in B.mx4_shapes(4, 64))
    B.moe_mx4_quantize(x, False, q, s)
    for args in ((x[:, :48].contiguous(), False, q, s), (x.half(), False, q, s), (x, False, q[:0], s), (x, False, q, s.int()), (x.t(), False, q, s),
                 (x[0], False, q, s), (x, 2, q, s), (x.cpu(), False, q, s), (torch.zeros(64, 4, dtype=BF16, device="cuda"), True, q, s)):
        with pytest.raises(B.MoeError):
            B.moe_mx4_quantize(*args)
    for args in ((q, s, x[:, :32].contiguous().half()), (q, s[:, :0], x), (q.int(), s, x)):
        with pytest.raises(B.MoeError):
            B.moe_mx4_dequantize(*args)
    xp, off, w = make([3, 4], 64, 96)
    o, (a, b, c), ws = run(xp, off, w)
    x, offsets = xp.cuda(), off.cuda()
    for args in ((x.float(), offsets, *a, *b, *c, o.float(), ws), (x, offsets[:2], *a, *b, *c, o, ws), (x, offsets, *a, *b, *a, o, ws),
                 (x, offsets, *a, *b, *c, o, ws[:256]), (x, offsets, *a, *b, *c, o[:3], ws), (x, offsets, a[1], a[0], *b, *c, o, ws)):
        with pytest.raises(B.MoeError):
            B.moe_mx4_expert_fwd(*args)


@pytest.mark.parametrize("d,f", [(640, 1152), (736, 1216), (832, 1408), (512, 1536)])
def test_workgroups_with_several_tiles(d, f):
    """The same experts a few at a time, as many as every workgroup has one tile of: the last stages of a contraction (of 128: 5, 6, 7, 4; 9, 10,
    11, 12) and the first of the next tile's in one ring of loads."""
    print(f"case mx4 several tiles {d} {f}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(d)
    E, rows, part = 32, 768, 8
    xp = torch.randn(E * rows, d, generator=g, device="cuda").mul(torch.exp(torch.randn(E * rows, 1, generator=g, device="cuda"))).to(BF16)
    off = rows * torch.arange(E + 1, dtype=torch.int32, device="cuda")
    q = []
    for shape in ((d, f), (d, f), (f, d)):
        w = torch.randn(E, *shape, generator=g, device="cuda") * torch.exp2(torch.randint(-4, 5, (E, shape[0] // 32, shape[1]), generator=g, device="cuda")
                                                                            ).repeat_interleave(32, 1) * shape[0] ** -0.5
        q.append(L.mx4_weights(w.to(BF16)))
    ws = torch.empty(B.moe_workspace_bytes(B.WS_MX4_EXPERT_FWD, B.MOE_BF16, 0, 0, d, f, E, E * rows), dtype=torch.uint8, device="cuda")
    o, ref = torch.empty_like(xp), torch.empty_like(xp)
    B.moe_mx4_expert_fwd(xp, off, *q[0], *q[1], *q[2], o, ws)
    for e in range(0, E, part):
        r = slice(e * rows, (e + part) * rows)
        args = [t[e:e + part] for w in q for t in w]
        B.moe_mx4_expert_fwd(xp[r], off[:part + 1], *args, ref[r], ws)
    differ = (o != ref).any(1).sum().item()
    assert differ == 0, f"{differ} of {E * rows} rows"


@pytest.mark.parametrize("rows,d,f", [([1], 4096, 1536), ([1, 0, 4, 11, 16], 544, 288), ([0, 3, 0, 2], 96, 544), ([1] * 32, 1152, 96), ([17, 15], 640, 416),
                                      ([32], 2080, 800), ([1] * 20 + [0] * 100 + [3] * 4, 160, 64)])
def test_few_rows_in_all(rows, d, f):
    """At most 32 rows: quantised inside the first product.  The same numbers as with a larger capacity, to the bit where no expert has more than
    a tile of rows."""
    print(f"case mx4 few rows {rows} {d} {f}", flush=True)
    xp, off, w = make(rows, d, f, seed=d + f)
    R = sum(rows)
    o, _, _ = run(xp, off, w)
    check(xp, off, w, o)
    larger, _, _ = run(torch.cat([xp, torch.full((64, d), float("nan"), dtype=BF16)]), off, w)
    check(xp, off, w, larger[:R])
    if max(rows) <= 16:
        assert torch.equal(o, larger[:R])
    # a row of NaN keeps to itself; what the workspace held does not enter
    xp[R // 2, d - 1] = float("nan")
    bad, _, _ = run(xp, off, w, poison=False)
    others = torch.arange(R) != R // 2
    assert torch.isnan(bad[R // 2]).all() and torch.equal(bad[others], o[others])
