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


SLACK = [([3, 0, 9], 136, 264), ([20, 0, 40, 1], 4104, 136), ([300, 5, 0, 100], 136, 264), ([40, 300, 0, 7], 72, 4104), ([1500, 0, 900, 3, 700], 200, 520)]


@pytest.mark.parametrize("rows,K,N,dt", [(*c, dt) for c in SLACK for dt in (BF16, F32)] + [([7000, 1, 0, 1202], 4096, 4104, BF16)], ids=str)
def test_rows_past_the_last_expert_may_be_no_numbers(rows, K, N, dt):
    """What lies there takes no part: the same bits, and nothing written there."""
    print(f"case linear {rows} {K} {N} {dt}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)  # noqa: E731
    R, E = sum(rows), len(rows)
    cap, off = R + 70, torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32, device="cuda")
    x, z, dy, residual, w, bias = r(cap, K), r(cap, N), r(cap, N), r(cap, N), r(E, K, N) * K ** -0.5, r(E, N)
    seen = []
    for fill in (0.0, float("nan"), float("inf")):
        for t in (x, z, dy, residual):
            t[R:] = fill
        y, zz, dx, dw, db = (torch.full_like(t, 7.0) for t in (dy, dy, x, w, bias))
        ws = [torch.full((B.moe_workspace_bytes(which, code(dt), 0, 0, K, N, E, cap),), 0xFF, dtype=torch.uint8, device="cuda")
              for which in (B.WS_LINEAR_FWD, B.WS_LINEAR_BWD)]
        B.moe_linear_fwd(x, off, w, bias, B.ACT_GELU, residual, zz, y, ws[0])
        B.moe_linear_bwd(x, z, dy, off, w, B.ACT_GELU, dx, dw, db, False, ws[1])
        for t in (y, zz, dx):
            assert (t[R:] == 7.0).all()
        for t in (y, zz, dx, dw, db):
            assert torch.isfinite(t).all()
        seen.append((y, zz, dx, dw, db))
    for other in seen[1:]:
        assert all(torch.equal(a, b) for a, b in zip(seen[0], other))


def products_of(x, w, dy, z, act, at):
    """Rows `at` of y and dx, in float64; and dw and db of all rows, in pieces of them."""
    y = L_act(x[at].double() @ w.double(), act)
    slope = lambda t: torch.autograd.grad(L_act(t.requires_grad_(), act).sum(), t)[0]  # noqa: E731
    dz = lambda s: dy[s].double() * slope(z[s].double())  # noqa: E731
    dw, db = torch.zeros_like(w, dtype=torch.float64), torch.zeros(w.shape[1], dtype=torch.float64, device="cuda")
    for a in range(0, len(x), 65536):
        g = dz(slice(a, a + 65536))
        dw += x[a:a + 65536].double().T @ g
        db += g.sum(0)
    return y, dz(at) @ w.double().T, dw, db


def L_act(z, act):
    return z if act == B.ACT_NONE else z * torch.sigmoid(z)


@pytest.mark.parametrize("dt,rows,K,N", [(BF16, 1_100_000, 64, 2056), (F32, 560_000, 64, 4100), (BF16, 300_000, 7200, 64)], ids=str)
@pytest.mark.parametrize("grouped", [False, True])
def test_more_elements_than_32_bits_count(dt, rows, K, N, grouped):
    """2^31 elements and more of an input and an output, rows behind them among others.  Root mean squares, whose bounds are those of the rounding: 2^-8 and
    another for dz in bf16; sums over a million rows in fp32 lose 2^-24 sqrt(rows / 2) = 2^-14.5 of theirs by chance, and by a bias of as many roundings as
    a part or a row tile of them has, at most 1.1e6 / 64 * 2^-24 = 2^-10: 2^-9."""
    print(f"case linear {rows} {K} {N} {dt} {grouped}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(rows)
    new = lambda *s: torch.empty(s, dtype=dt, device="cuda").normal_(generator=g)  # noqa: E731
    x, dy, z = new(rows, K), new(rows, N), new(rows, N)
    w = (torch.randn(K, N, generator=g, device="cuda") * K ** -0.5).to(dt)
    y, dx, dw, db = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w[0])
    off = torch.tensor([0, 0, rows], dtype=torch.int32, device="cuda") if grouped else None
    weights = torch.stack([torch.full_like(w, float("nan")), w]) if grouped else w
    dws, dbs = (torch.stack([dw, dw]), torch.stack([db, db])) if grouped else (dw, db)
    ws = torch.empty(max(B.moe_workspace_bytes(which, code(dt), 0, 0, K, N, 2 if grouped else 1, rows) for which in (B.WS_LINEAR_FWD, B.WS_LINEAR_BWD)),
                     dtype=torch.uint8, device="cuda")
    B.moe_linear_fwd(x, off, weights, None, B.ACT_SILU, None, None, y, ws)
    B.moe_linear_bwd(x, z, dy, off, weights, B.ACT_SILU, dx, dws, dbs, False, ws)
    if grouped:
        assert not dws[0].any() and not dbs[0].any()
        dw, db = dws[1], dbs[1]
    middle = (1 << 31) // max(K, N)
    at = torch.cat([torch.arange(a, b, device="cuda") for a, b in ((0, 300), (middle - 200, middle + 200), (rows - 300, rows))])
    for name, got, ref in zip(("y", "dx", "dw", "db"), (y[at], dx[at], dw, db), products_of(x, w, dy, z, B.ACT_SILU, at)):
        half = 2.0 ** -8 if dt == BF16 else 2.0 ** -20
        off_by = (got.double() - ref).norm() / ref.norm()
        assert off_by <= (1.25 * half if name in ("y", "dx") else half + 2.0 ** -9), (name, float(off_by))


def test_more_weights_than_32_bits_count():
    """40 matrices of 7168 to 8200, 2.35e9 elements: the last one's products."""
    E, K, N, rows = 40, 7168, 8200, 120
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.empty(E, K, N, dtype=BF16, device="cuda").normal_(generator=g)
    off = torch.arange(0, 3 * E + 1, 3, dtype=torch.int32, device="cuda")
    x, dy = (torch.randn(rows, n, generator=g, device="cuda").to(BF16) for n in (K, N))
    y, dx, dw, db = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w), torch.empty(E, N, dtype=BF16, device="cuda")
    ws = torch.empty(max(B.moe_workspace_bytes(which, B.MOE_BF16, 0, 0, K, N, E, rows) for which in (B.WS_LINEAR_FWD, B.WS_LINEAR_BWD)), dtype=torch.uint8, device="cuda")
    B.moe_linear_fwd(x, off, w, None, B.ACT_NONE, None, None, y, ws)
    B.moe_linear_bwd(x, None, dy, off, w, B.ACT_NONE, dx, dw, db, False, ws)
    for e in (0, 36, 37, 39):
        a, b, c = x[3 * e:3 * e + 3].double(), w[e].double(), dy[3 * e:3 * e + 3].double()
        for name, got, ref in (("y", y[3 * e:3 * e + 3], a @ b), ("dx", dx[3 * e:3 * e + 3], c @ b.T), ("dw", dw[e], a.T @ c), ("db", db[e], c.sum(0))):
            assert (got.double() - ref).norm() <= 2.0 ** -8 * ref.norm(), (name, e)


@pytest.mark.parametrize("rows", [4096, [7000, 1, 0, 1202]], ids=str)
def test_largest_tiles_again_and_replayed(rows):
    """The 256x256 tiles, drawn by whoever is free: the same bits in eager calls, and in a graph replayed between them."""
    dense = isinstance(rows, int)
    counts = [rows] if dense else rows
    R, E, K, N = sum(counts), len(counts), 4088, 4088
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)  # noqa: E731
    lead = () if dense else (E,)
    off = None if dense else torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda")
    x, dy, w, bias = r(R, K), r(R, N), r(*lead, K, N) * K ** -0.5, r(*lead, N)

    def outputs():
        return [torch.full_like(t, float("nan")) for t in (dy, dy, x, w, bias)]

    def spaces():
        return [torch.empty(B.moe_workspace_bytes(which, B.MOE_BF16, 0, 0, K, N, E, R), dtype=torch.uint8, device="cuda") for which in (B.WS_LINEAR_FWD, B.WS_LINEAR_BWD)]

    def step(out, ws):
        z, y, dx, dw, db = out
        B.moe_linear_fwd(x, off, w, bias, B.ACT_GELU, None, z, y, ws[0])
        B.moe_linear_bwd(x, z, dy, off, w, B.ACT_GELU, dx, dw, db, False, ws[1])

    eager, captured, ws_e, ws_c = outputs(), outputs(), spaces(), spaces()
    step(eager, ws_e)
    first = [t.clone() for t in eager]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(captured, ws_c)
    for i in range(4):
        if i:
            x.neg_()
        step(eager, ws_e)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, captured)), i
        assert i % 2 or all(torch.equal(a, b) for a, b in zip(eager, first)), i
