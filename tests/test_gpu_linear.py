"""The linear layer, grouped by expert and dense, against the float64 oracle, through the binding.

Bounds, set before the first run.  A bf16 store is off by at most 2^-8 of the value, an fp32 one by 2^-24.  Products of bf16 operands are exact
in fp32, those of fp32 operands off by 2^-24; a sum over K terms rounds at most once per term, to 24 bits and at worst towards zero: with m
the sum of the terms' sizes it is off by (K + 4) 2^-23 m.  Activations: bf16 takes erfc from a formula that is off by 1.5e-7 and the hardware's
exp2 and reciprocal, fp32 the library's functions; both get (1 + |z|) 2^-21 beside the slope (at most 1.13) times z's error.  dz in bf16 is
rounded once more before the products, unless the activation is none or relu, which leave dy's bits or zeros."""
import numpy as np
import pytest
import torch

from oracle import linear_oracle as L
from paper_2605_11005_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
HALF_ULP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


def host(t):
    return t.detach().double().cpu().numpy()


def within(got, ref, tol, name):
    got = host(got)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.unravel_index(bad.argmax(), bad.shape), got[bad][:4], ref[bad][:4])


class Case:
    """rows: an int for a dense layer, a list of each expert's rows for a grouped one.  slack: rows of the buffers past the last expert's."""

    def __init__(self, rows, K, N, act="none", dt=BF16, bias=True, residual=True, save=True, slack=3, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g).to(dt).cuda()  # noqa: E731
        self.dense, self.act, self.dt, self.save = isinstance(rows, int), act, dt, save
        counts = [rows] if self.dense else rows
        self.ref_off = np.concatenate([[0], np.cumsum(counts)])
        self.R, self.K, self.N, E = int(self.ref_off[-1]), K, N, len(counts)
        self.cap = self.R if self.dense else self.R + slack
        self.off = None if self.dense else torch.tensor(self.ref_off, dtype=torch.int32).cuda()
        lead = () if self.dense else (E,)
        self.E, self.lead = E, lead
        self.x, self.w = r(self.cap, K), (torch.randn(*lead, K, N, generator=g) * K ** -0.5).to(dt).cuda()
        self.bias = r(*lead, N) if bias else None
        self.residual = r(self.cap, N) if residual else None
        self.dy = r(self.cap, N)

    def nan(self, *shape):
        return torch.full(shape, float("nan"), dtype=self.dt, device="cuda")

    def ws(self, which):
        n = B.moe_workspace_bytes(which, B.MOE_BF16 if self.dt == BF16 else B.MOE_F32, 0, 0, self.K, self.N, self.E, self.cap)
        return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")

    def forward(self):
        self.z = self.nan(self.cap, self.N) if self.save else None
        self.y = self.nan(self.cap, self.N)
        B.moe_linear_fwd(self.x, self.off, self.w, self.bias, B.ACTIVATIONS[self.act], self.residual, self.z, self.y, self.ws(B.WS_LINEAR_FWD))

    def weights(self):
        return host(self.w).reshape(self.E, self.K, self.N)

    def check_forward(self):
        R = self.R
        bias = None if self.bias is None else host(self.bias).reshape(self.E, self.N)
        ref = L.fwd(host(self.x[:R]), self.ref_off, self.weights(), bias, self.act, None if self.residual is None else host(self.residual[:R]))
        half, err = HALF_ULP[self.dt], (self.K + 4) * 2.0 ** -23 * ref["mag"]
        if self.z is not None:
            within(self.z[:R], ref["z"], err + half * (np.abs(ref["z"]) + err), "z")
        err = 1.13 * err + (0 if self.act == "none" else (1 + np.abs(ref["z"])) * 2.0 ** -21) + 2.0 ** -23 * np.abs(ref["y"])
        within(self.y[:R], ref["y"], err + half * (np.abs(ref["y"]) + err), "y")
        for t in (self.y, self.z):
            assert t is None or torch.isnan(t[R:]).all(), "rows past the last expert's"

    def backward(self, accumulate=False, want=("dx", "dw", "db")):
        out = {"dx": self.nan(self.cap, self.K), "dw": self.nan(*self.lead, self.K, self.N), "db": self.nan(*self.lead, self.N)}
        if accumulate:
            for name in ("dx", "dw", "db"):
                out[name][:self.R if name == "dx" else None].fill_(1.0)
        self.dx, self.dw, self.db = (out[n] if n in want else None for n in ("dx", "dw", "db"))
        B.moe_linear_bwd(self.x, self.z if self.act != "none" else None, self.dy, self.off, self.w, B.ACTIVATIONS[self.act], self.dx, self.dw, self.db,
                         accumulate, self.ws(B.WS_LINEAR_BWD), accumulate)

    def check_backward(self, accumulate=False):
        R = self.R
        z = np.zeros((R, self.N)) if self.z is None else host(self.z[:R])
        ref, mag = L.bwd(host(self.x[:R]), z, host(self.dy[:R]), self.ref_off, self.weights(), self.act)
        half, exact = HALF_ULP[self.dt], self.act in ("none", "relu")
        dz_err = np.zeros_like(z) if exact else (1 + np.abs(z)) * 2.0 ** -20 * np.abs(host(self.dy[:R]))     # |slope| has |z| in it
        rounded = dz_err + (0 if exact or self.dt == F32 else half * (np.abs(ref["dz"]) + dz_err))
        add = 1.0 if accumulate else 0.0
        weights = self.weights()
        for e, at in L.segments(self.ref_off):
            w, x, n = np.abs(weights[e]), np.abs(host(self.x[at])), at.stop - at.start
            pick = (lambda t: t) if self.dense else (lambda t: t[e])
            if self.dx is not None:
                err = rounded[at] @ w.T + (self.N + 4) * 2.0 ** -23 * mag["dx"][at] + 2.0 ** -23 * add
                r = ref["dx"][at] + add
                within(self.dx[at], r, err + half * (np.abs(r) + err), f"dx {e}")
            if self.dw is not None:
                err = x.T @ rounded[at] + (n + 40) * 2.0 ** -23 * mag["dw"][e] + 2.0 ** -23 * add
                r = ref["dw"][e] + add
                within(pick(self.dw), r, err + half * (np.abs(r) + err), f"dw {e}")
            if self.db is not None:
                err = dz_err[at].sum(axis=0) + (n + 4) * 2.0 ** -23 * mag["db"][e] + 2.0 ** -23 * add
                r = ref["db"][e] + add
                within(pick(self.db), r, err + half * (np.abs(r) + err), f"db {e}")
        if self.dx is not None:
            assert torch.isnan(self.dx[R:]).all(), "rows past the last expert's"

    def check_both(self, accumulate=False):
        self.forward()
        self.check_forward()
        self.backward(accumulate)
        self.check_backward(accumulate)


@pytest.mark.parametrize("dt", (BF16, F32))
@pytest.mark.parametrize("K,N", [(8, 8), (16, 264), (64, 64), (72, 40), (96, 72), (520, 136), (264, 776)])
@pytest.mark.parametrize("rows", [0, 1, 2, 17, 64, 130, 257, [0], [1, 0, 2], [5, 0, 0, 33, 1, 64], [129, 300, 0, 7]], ids=str)
def test_sizes(rows, K, N, dt):
    print(f"case linear {rows} {K} {N} {dt}", flush=True)
    c = Case(rows, K, N, "gelu" if K % 64 else "silu", dt, seed=K + N)
    c.check_both()


@pytest.mark.parametrize("K,N", [(4, 4), (12, 100), (100, 68)])
def test_fp32_widths(K, N):
    Case([3, 70, 0], K, N, "gelu_tanh", F32).check_both()


@pytest.mark.parametrize("dt", (BF16, F32))
@pytest.mark.parametrize("act", list(B.ACTIVATIONS))
def test_options(act, dt):
    for rows in (37, [20, 0, 150, 64]):
        for opts in (dict(), dict(bias=False), dict(residual=False), dict(bias=False, residual=False, save=False)):
            print(f"case linear {act} {rows} {opts} {dt}", flush=True)
            c = Case(rows, 88, 136, act, dt, seed=len(act), **opts)
            c.forward()
            c.check_forward()
            if c.save or act == "none":
                for accumulate, want in ((False, ("dx", "dw", "db")), (True, ("dx", "dw", "db")), (True, ("dw", "db")), (False, ("dx",)), (True, ("dx",)),
                                         (True, ("dw",)), (False, ("db",)), (False, ())):
                    c.backward(accumulate, want)
                    c.check_backward(accumulate)


@pytest.mark.parametrize("rows,K,N", [(3000, 264, 2056), (2900, 136, 4104), ([1500, 700, 0, 900, 5], 200, 2056), ([2500], 1032, 1544)], ids=str)
def test_many_tiles(rows, K, N):
    """Several rounds of the large tiles, with what is left of rows, columns and contraction."""
    print(f"case linear {rows} {K} {N}", flush=True)
    Case(rows, K, N, "gelu_tanh", seed=N).check_both()


@pytest.mark.parametrize("rows", [4096, [1030, 1000, 0, 1026, 1040]], ids=str)
def test_a_whole_round_of_the_largest_tiles(rows):
    """About 256 tiles of 256x256 in each product, one per CU, with a contraction that ends inside a k-tile."""
    print(f"case linear {rows} 4088 4088", flush=True)
    c = Case(rows, 4088, 4088, "silu", residual=isinstance(rows, int), seed=9)
    c.check_both(accumulate=isinstance(rows, list))


@pytest.mark.parametrize("dt,K,N", [(BF16, 4104, 136), (BF16, 136, 4104), (BF16, 7176, 2056), (F32, 2052, 68), (F32, 68, 2052)])
@pytest.mark.parametrize("rows", [1, 33, 200, [3, 0, 40, 1], [130, 0, 70, 1, 5]], ids=str)
def test_long_contractions(rows, dt, K, N):
    """Few tiles, whose contractions are cut in parts."""
    print(f"case linear {rows} {K} {N} {dt}", flush=True)
    Case(rows, K, N, "gelu", dt, seed=K).check_both(accumulate=rows in (33, [130, 0, 70, 1, 5]))


@pytest.mark.parametrize("dt", (BF16, F32))
@pytest.mark.parametrize("rows", [[3000, 0, 511, 512, 1024, 1], [0, 0, 5000, 255, 256, 700, 1023], [40] * 20 + [6000]], ids=str)
def test_weight_gradients_of_experts_that_differ(rows, dt):
    """Some experts' rows are cut in parts in a launch where others' are not."""
    print(f"case linear {rows} {dt}", flush=True)
    for accumulate in (False, True):
        Case(rows, 136, 72, "gelu", dt, seed=11).check_both(accumulate)


@pytest.mark.parametrize("dt,N", [(BF16, 4104), (F32, 2052)])
@pytest.mark.parametrize("rows", [8300, [5000, 3, 0, 3300]], ids=str)
def test_gradients_of_large_activations(rows, dt, N):
    """dy and z beyond half of the Infinity Cache."""
    print(f"case linear {rows} 16 {N} {dt}", flush=True)
    Case(rows, 16, N, "gelu", dt, residual=False, seed=7).check_both()


@pytest.mark.parametrize("dt", (BF16, F32))
@pytest.mark.parametrize("rows", [20000, [18000, 12, 0, 300]], ids=str)
def test_weight_gradient_of_many_rows(rows, dt):
    """One heavy expert, whose gradient is summed in pieces."""
    c = Case(rows, 72, 136, "silu", dt, seed=5)
    c.check_both(accumulate=True)


@pytest.mark.parametrize("dt", (BF16, F32))
@pytest.mark.parametrize("rows", [31, 32, 33, 63, 65, 127, 128, 129, 1023, 1024, 1025, [32] * 3, [97, 0, 0], [64, 1, 128], [500, 24, 501]], ids=str)
def test_row_counts_around_the_kernels_limits(rows, dt):
    print(f"case linear {rows} {dt}", flush=True)
    Case(rows, 264, 200, "gelu", dt, slack=0, seed=3).check_both(accumulate=True)


@pytest.mark.parametrize("dt", (BF16, F32))
@pytest.mark.parametrize("rows,K,N", [([i % 3 for i in range(1024)], 16, 24), ([0] * 700 + [150] + [0] * 323, 72, 136), ([(7 * i) % 41 for i in range(130)], 40, 72)],
                         ids=["1024 experts", "one of 1024", "130 experts"])
def test_many_experts(rows, K, N, dt):
    print(f"case linear {len(rows)} experts {dt}", flush=True)
    Case(rows, K, N, "silu", dt, seed=len(rows)).check_both()


@pytest.mark.parametrize("rows,K,N", [(4, 8200, 16392), (100, 8200, 16392), (50, 16392, 8200), ([3, 0, 40, 1, 2], 4104, 6664), ([100, 0, 128, 1, 60], 4104, 6664)],
                         ids=str)
def test_weights_beyond_the_infinity_cache(rows, K, N):
    """The bounds of the other tests, in float64 on the device."""
    print(f"case linear {rows} {K} {N}", flush=True)
    c = Case(rows, 8, 8, "none", slack=0)
    g = torch.Generator(device="cuda").manual_seed(K)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)  # noqa: E731
    c.K, c.N = K, N
    c.x, c.w, c.bias, c.residual, c.dy = r(c.cap, K), r(*c.lead, K, N), r(*c.lead, N), r(c.cap, N), r(c.cap, N)
    c.forward()
    c.backward()
    for e, at in L.segments(c.ref_off):
        pick = (lambda t: t) if c.dense else (lambda t: t[e])
        w, x, dy = pick(c.w).double(), c.x[at].double(), c.dy[at].double()
        for name, got, ref, mag, terms in (
                ("y", c.y[at], x @ w + pick(c.bias).double() + c.residual[at].double(),
                 x.abs() @ w.abs() + pick(c.bias).double().abs() + c.residual[at].double().abs(), K + 5),
                ("dx", c.dx[at], dy @ w.T, dy.abs() @ w.T.abs(), N + 4),
                ("dw", pick(c.dw), x.T @ dy, x.T.abs() @ dy.abs(), at.stop - at.start + 40),
                ("db", pick(c.db), dy.sum(0), dy.abs().sum(0), at.stop - at.start + 4)):
            err = terms * 2.0 ** -23 * mag
            assert ((got.double() - ref).abs() <= err + 2.0 ** -8 * (ref.abs() + err)).all(), (name, e)


@pytest.mark.parametrize("rows,K,N", [(2100, 1032, 2012), (7000, 260, 1220), ([1800, 0, 1300, 900, 40], 516, 1092), ([5, 700, 0, 30, 200, 1, 64, 90], 260, 388)], ids=str)
def test_fp32_of_many_tiles(rows, K, N):
    """Pairs of tiles beside each other whose second one is narrow or missing, and experts whose rows differ, tiles in chunks."""
    print(f"case linear {rows} {K} {N} fp32", flush=True)
    Case(rows, K, N, "gelu_tanh", F32, seed=N).check_both(accumulate=isinstance(rows, list))


def test_fp32_infinities_in_pairs_of_tiles():
    """Sums that are no numbers are formed again from the operands: in both tiles of a pair, and in no others."""
    c = Case(2100, 520, 2060, "none", F32, residual=False, bias=False)
    c.x.abs_().add_(0.5)
    c.w.abs_().add_(0.01)
    for col in (3, 70, 2047, 2059):
        c.w[519, col] = float("inf")
    c.w[0, 130] = 2.0 ** 100
    c.forward()
    y = host(c.y)
    assert (y[:, [3, 70, 2047, 2059]] == np.inf).all()
    rest = np.delete(y, (3, 70, 2047, 2059), axis=1)
    assert np.isfinite(rest).all()
    ref = host(c.x) @ np.delete(host(c.w), (3, 70, 2047, 2059), axis=1)
    assert (np.abs(rest - ref) <= (520 + 4) * 2.0 ** -23 * ref).all()               # (all terms positive: their sum is their sizes')


@pytest.mark.parametrize("dt", (BF16, F32))
@pytest.mark.parametrize("K", (64, 72))
def test_infinities_and_nan_stay_where_they_belong(K, dt):
    """An infinity in a weight, also in the last row of the contraction, makes its column infinite and no NaN, rows of x with one spoil themselves only."""
    c = Case([40, 9], K, 136, "none", dt, residual=False)
    c.x.abs_().add_(0.5)
    c.w[0, K - 1, 3] = float("inf")
    c.w[0, 0, 5] = float("-inf")
    c.x[41, 7] = float("nan")
    c.x[43, K - 1] = float("inf")
    c.w[1].abs_().add_(0.01)
    c.forward()
    y = host(c.y[:c.R])
    assert (y[:40, 3] == np.inf).all() and (y[:40, 5] == -np.inf).all()
    rest = np.delete(y[:40], (3, 5), axis=1)
    assert np.isfinite(rest).all()
    assert np.isnan(y[41]).all() and (y[43] == np.inf).all()
    assert np.isfinite(y[[40, 42, 44, 45, 46, 47, 48]]).all()
    c.dy[2, 135] = float("inf")
    c.dy[3, 0] = float("nan")
    c.w.fill_(1.0)
    c.x.fill_(1.0)
    c.backward()
    assert (host(c.dx[2]) == np.inf).all() and np.isnan(host(c.dx[3])).all() and np.isfinite(host(c.dx[4:c.R])).all()
    assert (host(c.dw[0, :, 135]) == np.inf).all() and np.isnan(host(c.dw[0, :, 0])).all() and np.isfinite(host(c.dw[0, :, 1:135])).all()
    assert np.isfinite(host(c.dw[1])).all() and host(c.db[0, 135]) == np.inf and np.isnan(host(c.db[0, 0]))


def test_extreme_pre_activations():
    """Activations where exp leaves fp32's range."""
    for dt in (BF16, F32):
        z = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 30.0, -30.0, 90.0, -90.0, 1e4, -1e4, 1e30, -1e30, 6.0, -6.0, -12.0, 0.5]).to(dt).cuda()
        w = torch.zeros(16, 16, dtype=dt, device="cuda")
        x = torch.zeros(2, 16, dtype=dt, device="cuda")
        for act in B.ACTIVATIONS:
            y, zz = torch.empty(2, 16, dtype=dt, device="cuda"), torch.empty(2, 16, dtype=dt, device="cuda")
            ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
            B.moe_linear_fwd(x, None, w, z, B.ACTIVATIONS[act], None, zz, y, ws)
            ref = L.act(host(z), act)
            with np.errstate(over="ignore"):
                tol = HALF_ULP[dt] * np.abs(ref) + 2.0 ** -21 * np.minimum(1 + np.abs(ref), 1e30)
            assert np.array_equal(host(zz), np.stack([host(z)] * 2))
            within(y, np.stack([ref] * 2), np.stack([tol] * 2), act)
            dx, db = torch.empty_like(x), torch.empty_like(z)
            ws = torch.empty(B.moe_workspace_bytes(B.WS_LINEAR_BWD, B.MOE_BF16 if dt == BF16 else B.MOE_F32, 0, 0, 16, 16, 1, 2), dtype=torch.uint8, device="cuda")
            B.moe_linear_bwd(x, zz, torch.ones_like(y), None, w, B.ACTIVATIONS[act], dx, None, db, False, ws)
            with np.errstate(over="ignore", invalid="ignore"):
                slope = 2 * np.nan_to_num(L.slope(host(z), act), nan=0.0)
                slope[np.abs(host(z)) >= 1e4] = 2.0 * (host(z)[np.abs(host(z)) >= 1e4] > 0) if act != "none" else 2.0
            within(db, slope, HALF_ULP[dt] * np.abs(slope) + 2.0 ** -15, act)       # z (1 - s) of z = 30 .. 90 in fp32: 90 2^-24, twice


def test_residual_in_place():
    c = Case([70, 200], 264, 520, "relu")
    c.forward()
    in_place = c.residual.clone()
    B.moe_linear_fwd(c.x, c.off, c.w, c.bias, B.ACT_RELU, in_place, None, in_place, c.ws(B.WS_LINEAR_FWD))
    assert torch.equal(in_place[:c.R], c.y[:c.R]) and torch.equal(in_place[c.R:], c.residual[c.R:])


@pytest.mark.parametrize("dt", (BF16, F32))
def test_bits_are_the_same_again(dt):
    for rows in (1, 40, [3000, 5, 0, 200]):
        c = Case(rows, 264, 520, "gelu", dt)
        c.forward()
        c.backward()
        first = [t.clone() for t in (c.z, c.y, c.dx, c.dw, c.db)]
        for _ in range(3):
            c.forward()
            c.backward()
            for a, b in zip(first, (c.z, c.y, c.dx, c.dw, c.db)):
                assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


def test_gradient_against_differences():
    """sum(dy y) moves by the gradients' product with a step, to second order in it."""
    for act in ("gelu", "gelu_tanh", "silu"):
        c = Case([5, 9], 24, 32, act, F32, residual=False, slack=0)
        c.forward()
        c.backward()
        loss = lambda x, w, b: (host(c.dy) * L.fwd(x, c.ref_off, w, b, act, None)["y"]).sum()  # noqa: E731
        rng, base = np.random.default_rng(3), [host(c.x), c.weights(), host(c.bias)]
        for i, grad in enumerate((c.dx, c.dw, c.db)):
            step = rng.standard_normal(base[i].shape) * 1e-5
            up, down = list(base), list(base)
            up[i], down[i] = base[i] + step, base[i] - step
            want, got = (loss(*up) - loss(*down)) / 2, (host(grad) * step).sum()
            assert abs(got - want) <= 1e-5 * np.abs(host(grad) * step).sum(), (act, i)


def test_captured_and_replayed():
    """One stream's graph over both calls, replayed between eager work that uses the same weights."""
    for rows in (4, 300, [100, 0, 30, 260]):
        c = Case(rows, 136, 264, "gelu")
        c.forward()
        c.backward()
        ws_f, ws_b = c.ws(B.WS_LINEAR_FWD), c.ws(B.WS_LINEAR_BWD)
        outs = [torch.empty_like(t) for t in (c.z, c.y, c.dx, c.dw, c.db)]
        act = B.ACTIVATIONS[c.act]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            B.moe_linear_fwd(c.x, c.off, c.w, c.bias, act, c.residual, outs[0], outs[1], ws_f)
            B.moe_linear_bwd(c.x, outs[0], c.dy, c.off, c.w, act, *outs[2:], False, ws_b)
        for i in range(4):
            c.x.mul_(-1.0 if i % 2 else 1.0)
            c.forward()
            c.backward()
            torch.cuda.synchronize()
            for t in outs:
                t.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            for want, got in zip((c.z, c.y, c.dx, c.dw, c.db), outs):
                n = c.R if want.shape[0] == c.cap else want.shape[0]
                assert torch.equal(want[:n], got[:n])


def test_on_another_stream():
    c = Case([100, 0, 30], 136, 264, "gelu")
    c.forward()
    want = c.y.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.forward()
    s.synchronize()
    assert torch.equal(want[:c.R], c.y[:c.R])


def test_two_calls_at_once():
    """Two streams, each with its own workspace, in the kernels for few rows, for tiles and for the largest."""
    for rows, K, N in ((8, 520, 1032), (300, 264, 520), ([300, 0, 100], 136, 264), (4096, 2056, 4088)):
        print(f"case linear {rows} {K} {N}", flush=True)
        cases = [Case(rows, K, N, "gelu", seed=i) for i in range(2)]
        first = []
        for c in cases:
            c.forward()
            c.backward()
            first.append([t.clone() for t in (c.z, c.y, c.dx, c.dw, c.db)])
        torch.cuda.synchronize()
        spaces = [(c.ws(B.WS_LINEAR_FWD), c.ws(B.WS_LINEAR_BWD)) for c in cases]
        outs = [[torch.full_like(t, float("nan")) for t in f] for f in first]
        streams = [torch.cuda.Stream() for _ in cases]
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for _ in range(4):
            for c, s, (fws, bws), (z, y, dx, dw, db) in zip(cases, streams, spaces, outs):
                with torch.cuda.stream(s):
                    B.moe_linear_fwd(c.x, c.off, c.w, c.bias, B.ACT_GELU, c.residual, z, y, fws)
                    B.moe_linear_bwd(c.x, z, c.dy, c.off, c.w, B.ACT_GELU, dx, dw, db, False, bws)
        torch.cuda.synchronize()
        for want, got in zip(first, outs):
            for a, b in zip(want, got):
                assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


def test_the_marshalling_makes_the_calls(monkeypatch):
    class Counting:
        def __init__(self, native):
            self.native, self.calls = native, 0

        def __getattr__(self, name):
            def call(*args):
                rc = getattr(self.native, name)(*args)
                self.calls += rc >= 0
                return rc
            return call

    class NotTaken:
        def __getattr__(self, name):
            return lambda *args: -1

    for rows in (30, [20, 0, 9]):
        for dt in (BF16, F32):
            results = []
            native = Counting(B._marshal())
            for m in (native, NotTaken()):
                monkeypatch.setattr(B, "_MARSHAL", m)
                c = Case(rows, 72, 136, "silu", dt)
                c.forward()
                c.backward()
                results.append([c.z, c.y, c.dx, c.dw, c.db])
            monkeypatch.undo()
            if not isinstance(native.native, B._ChecksHere):
                assert native.calls == 2
            for a, b in zip(*results):
                assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


def test_arguments_that_do_not_fit_are_named():
    c = Case([20, 9], 72, 136, "silu")
    c.forward()
    ws = c.ws(B.WS_LINEAR_BWD)
    good = dict(x=c.x, offsets=c.off, w=c.w, bias=c.bias, act=B.ACT_SILU, residual=c.residual, z=c.z, y=c.y, ws=ws)
    for bad in (dict(bias=c.bias[0]), dict(offsets=c.off[:2]), dict(offsets=c.off.long()), dict(residual=c.residual[:-1]), dict(y=c.y.float()),
                dict(x=c.x[:, ::2]), dict(w=c.w.transpose(1, 2)), dict(ws=ws.cpu()), dict(act=7), dict(z=c.z[:, :64])):
        with pytest.raises(B.MoeError):
            B.moe_linear_fwd(**dict(good, **bad))
    with pytest.raises(B.MoeError):
        B.moe_linear_bwd(c.x, None, c.dy, c.off, c.w, B.ACT_SILU, None, None, None, False, ws)
    torch.cuda.synchronize()
