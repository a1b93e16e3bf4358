"""The layer norm between two blocks against the float64 oracle, through the binding.

Bounds, set before the first run.  A bf16 store is off by at most 2^-8 of the value, an fp32 one by 2^-24.  Before it a value is a short chain of
fp32 operations on terms whose magnitudes add up to m (oracle's mag), with a mean and a 1/deviation whose sums run over d elements in chains
of at most 64 and trees: 100 * 2^-24 * m covers both.  The mean is off by up to that of the row's sizes, and xh by as much over the deviation,
so a row's terms get the size of |h'| + |mean| in place of their difference.  Column sums over T rows: chains of at most T/512 + 1 rows in a
block and 512/16 + 16 blocks behind it, each product off by the former: (T/512 + 160) * 2^-24 * sum |terms|."""
import numpy as np
import pytest
import torch

from oracle import layer_norm_oracle as N
from paper_2605_11005_amd import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-5
BF16, F32 = torch.bfloat16, torch.float32
HALF_ULP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
TYPES = [(BF16, BF16), (BF16, F32), (F32, F32)]


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def close(got, ref, mag, dtype, steps=100, name=""):
    got = host(got)
    assert np.isfinite(got).all(), name
    over = np.abs(got - ref) - (HALF_ULP[dtype] * np.abs(ref) * (1 + 2.0 ** -7) + steps * 2.0 ** -24 * mag)
    assert (over <= 0).all(), (name, float(over.max()), np.unravel_index(over.argmax(), over.shape))


class Case:
    def __init__(self, T, d, dt=BF16, rt=BF16, y=True, w=True, b=True, through=True, shift=0.5, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, dtype: torch.randn(s, generator=g).to(dtype).cuda()  # noqa: E731
        self.T, self.d, self.dt, self.rt = T, d, dt, rt
        self.y, self.h = r(T, d, dtype=dt) if y else None, (shift + torch.randn((T, d), generator=g)).to(rt).cuda()
        self.w, self.b = (1 + r(d, dtype=F32) / 4).to(dt) if w else None, r(d, dtype=dt) if b else None
        self.dn, self.dh_out = r(T, d, dtype=dt), r(T, d, dtype=rt) if through else None

    def nan(self, *shape, dtype):
        return torch.full(shape, float("nan"), dtype=dtype, device="cuda")

    def forward(self, h_out="new", n="new"):
        T, d = self.T, self.d
        self.h_out = (self.nan(T, d, dtype=self.rt) if h_out == "new" else h_out) if self.y is not None else None
        self.n = self.nan(T, d, dtype=self.dt) if n == "new" else n
        self.mean, self.rstd = self.nan(T, dtype=F32), self.nan(T, dtype=F32)
        B.moe_layer_norm_fwd(self.y, self.h, self.w, self.b, EPS, self.h_out, self.n, self.mean, self.rstd)

    def check_forward(self):
        ref = N.fwd(host(self.y), host(self.h), host(self.w), host(self.b), EPS)
        size = np.abs(host(self.h)) + (0 if self.y is None else np.abs(host(self.y)))
        if self.y is not None:
            close(self.h_out, ref["h_out"], size, self.rt, name="h_out")
        close(self.mean, ref["mean"], size.mean(axis=1) if self.d else size[:, 0], F32, name="mean")
        # the variance is off by 100 * 2^-24 of itself and by the mean's error squared
        assert (np.abs(host(self.rstd) / ref["rstd"] - 1) <= 100 * 2.0 ** -24).all(), "rstd"
        w, b = (1.0 if self.w is None else np.abs(host(self.w))), (0.0 if self.b is None else np.abs(host(self.b)))
        close(self.n, ref["n"], (size + size.mean(axis=1, keepdims=True)) * ref["rstd"][:, None] * w + b, self.dt, name="n")

    def backward(self, accumulate=False, want=("dh", "dy", "dw", "db")):
        T, d = self.T, self.d
        self.saved = self.h if self.y is None else self.h_out
        ws = torch.full((B.moe_workspace_bytes(B.WS_LAYER_NORM, 0, T, 0, d, 0, 0, 0),), 0xFF, dtype=torch.uint8, device="cuda")
        out = {"dh": self.nan(T, d, dtype=self.rt), "dy": self.nan(T, d, dtype=self.dt), "dw": self.nan(d, dtype=self.dt), "db": self.nan(d, dtype=self.dt)}
        if accumulate:
            out["dw"].fill_(1.0)
            out["db"].fill_(1.0)
        self.out = {name: t for name, t in out.items() if name in want}
        B.moe_layer_norm_bwd(self.saved, self.w, self.mean, self.rstd, self.dh_out, self.dn, self.out.get("dh"), self.out.get("dy"), self.out.get("dw"),
                             self.out.get("db"), accumulate, ws)

    def check_backward(self, accumulate=False):
        ref, mag = N.bwd(host(self.saved), host(self.w), host(self.mean), host(self.rstd), host(self.dh_out), host(self.dn))
        for name, got in self.out.items():
            sums = name in ("dw", "db")
            add = 1.0 if accumulate and sums else 0.0
            close(got, ref[name] + add, mag[name] + add, self.rt if name == "dh" else self.dt, self.T / 512 + 160 if sums else 100, name)


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("T,d", [(0, 64), (1, 8), (1, 7168), (3, 520), (5, 16384), (65, 2880), (600, 512), (1030, 1032), (2, 9000), (4200, 64), (9000, 1536)])
def test_sizes(T, d, dt, rt):
    print(f"case layer norm {T} {d} {dt} {rt}", flush=True)
    c = Case(T, d, dt, rt, seed=T + d)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("opts", [dict(y=False), dict(w=False), dict(b=False), dict(w=False, b=False), dict(through=False), dict(y=False, through=False)])
def test_options(opts, dt, rt):
    print(f"case layer norm {opts} {dt} {rt}", flush=True)
    for T, d in ((37, 264), (700, 1408), (3, 12000)):       # (more rows than blocks walk at once)
        c = Case(T, d, dt, rt, seed=d, **opts)
        c.forward()
        c.check_forward()
        for accumulate, want in ((False, ("dh", "dy", "dw", "db")), (True, ("dw",)), (True, ("dh", "db")), (False, ("dy",)), (False, ())):
            c.backward(accumulate, want)
            c.check_backward(accumulate)


@pytest.mark.parametrize("d", (64, 520, 4096, 9000))
def test_large_means_keep_their_digits(d):
    """A row of mean 2^12 and deviation 1: squares taken before the mean would lose 24 of their 24 bits.  The values are whole 2^-8ths, so that the
    mean is all that rounds, by d / 64 + 70 steps of 2^-24 of 2^12 at most; the deviation then by that squared."""
    g = torch.Generator().manual_seed(d)
    h = (4096 + torch.round(torch.randn((7, d), generator=g) * 256) / 256).cuda()
    n, mean, rstd = torch.empty_like(h), torch.empty(7, device="cuda"), torch.empty(7, device="cuda")
    B.moe_layer_norm_fwd(None, h, None, None, EPS, None, n, mean, rstd)
    ref = N.fwd(None, host(h), None, None, EPS)
    off = (d / 64 + 70) * 2.0 ** -24 * 4096
    assert (np.abs(host(mean) - ref["mean"]) <= off).all()
    assert (np.abs(host(rstd) / ref["rstd"] - 1) <= off * off + 100 * 2.0 ** -24).all()
    assert (np.abs(host(n) - ref["n"]) <= (off + 2.0 ** -12) * ref["rstd"][:, None] + np.abs(ref["n"]) * (off * off + 100 * 2.0 ** -24)).all()


def test_constant_rows_and_rows_that_are_no_numbers():
    h = torch.full((5, 256), 3.0, device="cuda")
    h[1, 7] = float("inf")
    h[2, 255] = float("nan")
    h[4] = 0
    n, mean, rstd = torch.empty_like(h), torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    b = torch.ones(256, device="cuda")
    B.moe_layer_norm_fwd(None, h, None, b, EPS, None, n, mean, rstd)
    assert (n[[0, 3, 4]] == 1).all() and torch.isnan(n[2]).all() and not torch.isfinite(n[1]).all()
    assert (mean[[0, 3]] == 3).all() and mean[4] == 0 and (rstd[[0, 3, 4]] - EPS ** -0.5).abs().max() < 1e-4 * EPS ** -0.5
    dh, ws = torch.empty_like(h), torch.empty(B.moe_workspace_bytes(B.WS_LAYER_NORM, 0, 5, 0, 256, 0, 0, 0), dtype=torch.uint8, device="cuda")
    B.moe_layer_norm_bwd(h, None, mean, rstd, None, torch.randn_like(h), dh, None, None, None, False, ws)
    assert torch.isfinite(dh[[0, 3, 4]]).all() and not torch.isfinite(dh[[1, 2]]).all()


def test_in_place():
    for dt, rt in TYPES:
        c = Case(70, 520, dt, rt)
        c.forward()
        c.backward()
        h, y = c.h.clone(), c.y.clone()
        B.moe_layer_norm_fwd(y, h, c.w, c.b, EPS, h, y)
        assert torch.equal(h, c.h_out) and torch.equal(y, c.n)
        dh, dn = c.dh_out.clone(), c.dn.clone()
        ws = torch.empty(B.moe_workspace_bytes(B.WS_LAYER_NORM, 0, 70, 0, 520, 0, 0, 0), dtype=torch.uint8, device="cuda")
        B.moe_layer_norm_bwd(c.h_out, c.w, c.mean, c.rstd, dh, dn, dh, dn, None, None, False, ws)
        assert torch.equal(dh, c.out["dh"]) and torch.equal(dn, c.out["dy"])


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("T,d", [(2, 16384), (70, 520), (500, 4096), (1024, 1032), (1400, 264)])
def test_in_place_beside_the_column_sums(T, d, dt, rt):
    """dy over dn and dh over dh_out where dw and db are formed too."""
    c = Case(T, d, dt, rt, seed=T)
    c.forward()
    c.backward()
    ws = torch.empty(B.moe_workspace_bytes(B.WS_LAYER_NORM, 0, T, 0, d, 0, 0, 0), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        dh, dn = c.dh_out.clone(), c.dn.clone()
        dw, db = (torch.full_like(c.w, float("nan")) for _ in range(2))
        B.moe_layer_norm_bwd(c.h_out, c.w, c.mean, c.rstd, dh, dn, dh, dn, dw, db, False, ws)
        c.out = {"dh": dh, "dy": dn, "dw": dw, "db": db}       # (the sums may take rows in other groups than out of place: held to the oracle)
        c.check_backward()


@pytest.mark.parametrize("T,d", [(T, d) for T in (511, 512, 513, 1023, 1024, 1025) for d in (264, 3080)] + [(699, 4096), (700, 4096), (2100, 1032), (140000, 8), (65000, 64)])
def test_one_launch_and_two(T, d):
    """Around the row counts that one launch takes."""
    for dt, rt in TYPES:
        c = Case(T, d, dt, rt, seed=T)
        c.forward()
        c.check_forward()
        for accumulate, want in ((True, ("dh", "dy", "dw", "db")), (False, ("dw",)), (False, ("dy",))):
            c.backward(accumulate, want)
            c.check_backward(accumulate)


@pytest.mark.parametrize("dt,rt,T,d", [(BF16, BF16, 66000, 1032), (BF16, BF16, 16500, 4104), (BF16, F32, 33000, 2056), (BF16, F32, 9000, 9000),
                                       (F32, F32, 66000, 520), (F32, F32, 20000, 2052), (F32, F32, 4200, 16384), (BF16, BF16, 131000, 520)])
def test_tensors_beyond_the_infinity_cache(dt, rt, T, d):
    """The same bounds, in float64 on the device."""
    print(f"case layer norm {T} {d} {dt} {rt}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(d)
    r = lambda *s, dtype: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    y, h, dn, dh_out, w, b = r(T, d, dtype=dt), r(T, d, dtype=rt), r(T, d, dtype=dt), r(T, d, dtype=rt), r(d, dtype=dt), r(d, dtype=dt)
    h_out, n, mean, rstd = torch.empty_like(h), torch.empty_like(y), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    B.moe_layer_norm_fwd(y, h, w, b, EPS, h_out, n, mean, rstd)
    dh, dy, dw, db = torch.empty_like(h), torch.empty_like(y), torch.empty_like(w), torch.empty_like(b)
    ws = torch.empty(B.moe_workspace_bytes(B.WS_LAYER_NORM, 0, T, 0, d, 0, 0, 0), dtype=torch.uint8, device="cuda")
    B.moe_layer_norm_bwd(h_out, w, mean, rstd, dh_out, dn, dh, dy, dw, db, False, ws)

    def held(got, ref, mag, steps=100):
        half = HALF_ULP[got.dtype]
        assert ((got.double() - ref).abs() <= half * (1 + 2.0 ** -7) * ref.abs() + steps * 2.0 ** -24 * mag).all()

    W, Bb, sums, mags = w.double(), b.double(), torch.zeros(2, d, dtype=torch.float64, device="cuda"), torch.zeros(2, d, dtype=torch.float64, device="cuda")
    for at in torch.arange(T).split(8192):
        at = slice(int(at[0]), int(at[-1]) + 1)
        x, size = y[at].double() + h[at].double(), y[at].double().abs() + h[at].double().abs()
        m = x.mean(1, keepdim=True)
        rs = ((x - m).square().mean(1, keepdim=True) + EPS).rsqrt()
        held(h_out[at], x, size)
        held(mean[at], m[:, 0], size.mean(1))
        held(rstd[at], rs[:, 0], rs[:, 0])
        held(n[at], (x - m) * rs * W + Bb, (size + size.mean(1, keepdim=True)) * rs * W.abs() + Bb.abs())
        m, rs, dN, through = mean[at, None].double(), rstd[at, None].double(), dn[at].double(), dh_out[at].double()
        x, size = (h_out[at].double() - m) * rs, (h_out[at].double().abs() + m.abs()) * rs
        t = W * dN
        want = through + rs * (t - t.mean(1, keepdim=True) - x * (t * x).mean(1, keepdim=True))
        mag = through.abs() + rs * (t.abs() + t.abs().mean(1, keepdim=True) + size * (t.abs() * size).mean(1, keepdim=True))
        held(dh[at], want, mag)
        held(dy[at], want, mag)
        sums += torch.stack([(dN * x).sum(0), dN.sum(0)])
        mags += torch.stack([(dN.abs() * size).sum(0), dN.abs().sum(0)])
    held(dw, sums[0], mags[0], T / 512 + 160)
    held(db, sums[1], mags[1], T / 512 + 160)


def test_gradient_against_differences():
    c = Case(4, 24, F32, F32)
    c.forward()
    c.backward()
    base = dict(y=host(c.y), w=host(c.w), b=host(c.b))

    def loss(y, w, b):
        out = N.fwd(y, host(c.h), w, b, EPS)
        return (out["n"] * host(c.dn)).sum() + (out["h_out"] * host(c.dh_out)).sum()

    rng = np.random.default_rng(1)
    for name, grad in (("y", c.out["dy"]), ("w", c.out["dw"]), ("b", c.out["db"])):
        step = rng.standard_normal(base[name].shape) * 1e-5
        want = (loss(**dict(base, **{name: base[name] + step})) - loss(**dict(base, **{name: base[name] - step}))) / 2
        assert abs((host(grad) * step).sum() - want) <= 2e-5 * np.abs(host(grad) * step).sum(), name


@pytest.mark.parametrize("T,d", [(5, 64), (300, 1408), (20, 12000)])
def test_captured_and_replayed(T, d):
    c = Case(T, d, BF16, F32)
    c.forward()
    c.backward()
    n, mean, rstd, h_out = (torch.empty_like(t) for t in (c.n, c.mean, c.rstd, c.h_out))
    outs = {k: torch.empty_like(v) for k, v in c.out.items()}
    ws = torch.empty(B.moe_workspace_bytes(B.WS_LAYER_NORM, 0, T, 0, d, 0, 0, 0), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.moe_layer_norm_fwd(c.y, c.h, c.w, c.b, EPS, h_out, n, mean, rstd)
        B.moe_layer_norm_bwd(h_out, c.w, mean, rstd, c.dh_out, c.dn, outs["dh"], outs["dy"], outs["dw"], outs["db"], False, ws)
    for _ in range(4):
        c.h.neg_()
        c.forward()
        c.backward()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip([c.n, c.mean, c.rstd, c.h_out] + list(c.out.values()), [n, mean, rstd, h_out] + list(outs.values())):
            assert torch.equal(a, b)


def test_the_marshalling_makes_the_calls(monkeypatch):
    class NotTaken:
        def __getattr__(self, name):
            return lambda *args: -1

    for dt, rt in TYPES:
        for opts in (dict(), dict(y=False, w=False, b=False, through=False)):
            results = []
            for m in (B._marshal(), NotTaken()):
                monkeypatch.setattr(B, "_MARSHAL", m)
                c = Case(21, 192, dt, rt, **opts)
                c.forward()
                c.backward(True)
                results.append([c.n, c.mean, c.rstd] + list(c.out.values()))
            monkeypatch.undo()
            for a, b in zip(*results):
                assert torch.equal(a, b)
