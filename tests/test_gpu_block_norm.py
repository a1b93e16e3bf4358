"""The norms between two blocks against the float64 oracle, through the binding.

Bounds, set before the first run.  A bf16 store is off by at most 2^-8 of the value, an fp32 one by 2^-24.  Before it a value is a short chain of
fp32 operations on terms whose magnitudes add up to m (oracle's mag), with 1/rms factors whose sums run over d elements in chains of at
most 64 and trees: 100 * 2^-24 * m covers both.  Column sums over T rows: chains of at most T/512 + 1 rows in a block and 512/16 + 16 blocks
behind it, each product off by the former: (T/512 + 160) * 2^-24 * sum |terms|."""
import numpy as np
import pytest
import torch

from oracle import norm_oracle as N
from paper_2605_11005_amd import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-6
BF16, F32 = torch.bfloat16, torch.float32
HALF_ULP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


class Case:
    def __init__(self, T, d, dt=BF16, rt=BF16, post_norm=True, w_post=True, gate=True, alpha=0.5, beta=1.5, y=True, w_pre=True, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, dtype: torch.randn(s, generator=g).to(dtype).cuda()  # noqa: E731
        self.T, self.d, self.dt, self.rt, self.post_norm, self.alpha, self.beta = T, d, dt, rt, post_norm and y, alpha, beta
        self.y, self.h = r(T, d, dtype=dt) if y else None, r(T, d, dtype=rt)
        self.gate = torch.rand(T, generator=g).cuda() if gate and y else None
        self.w_post = (1 + r(d, dtype=F32) / 4).to(dt) if w_post and y else None
        self.w_pre = (1 + r(d, dtype=F32) / 4).to(dt) if w_pre else None
        self.dn, self.dh_out = r(T, d, dtype=dt) if w_pre else None, r(T, d, dtype=rt)

    def nan(self, *shape, dtype):
        return torch.full(shape, float("nan"), dtype=dtype, device="cuda")

    def forward(self, h_out="new", n="new"):
        T, d = self.T, self.d
        self.h_out = (self.nan(T, d, dtype=self.rt) if h_out == "new" else h_out) if self.y is not None else None
        self.n = (self.nan(T, d, dtype=self.dt) if n == "new" else n) if self.w_pre is not None else None
        self.r_post = self.nan(T, dtype=F32) if self.post_norm else None
        self.r_pre = self.nan(T, dtype=F32) if self.w_pre is not None else None
        B.moe_block_norm_fwd(self.y, self.gate, self.w_post, self.post_norm, self.h, self.w_pre, self.alpha, self.beta, EPS, self.h_out, self.n,
                             self.r_post, self.r_pre)

    def backward(self, accumulate=False, dh_out=True):
        T, d, y = self.T, self.d, self.y is not None
        self.saved = self.h_out if y else self.h
        self.ws = torch.full((B.moe_workspace_bytes(B.WS_BLOCK_NORM, 0, T, 0, d, 0, 0, 0),), 0xFF, dtype=torch.uint8, device="cuda")
        self.dh, self.dy = self.nan(T, d, dtype=self.rt), self.nan(T, d, dtype=self.dt) if y else None
        self.dgate = self.nan(T, dtype=F32) if y else None
        fill = (lambda: torch.ones(d, dtype=self.dt, device="cuda")) if accumulate else (lambda: self.nan(d, dtype=self.dt))
        self.dw_post, self.dw_pre = fill() if y else None, fill() if self.w_pre is not None else None
        B.moe_block_norm_bwd(self.y, self.gate, self.w_post, self.post_norm, self.saved, self.w_pre, self.r_post, self.r_pre,
                             self.dh_out if dh_out else None, self.dn, self.alpha, self.beta, self.dh, self.dy, self.dgate, self.dw_post,
                             self.dw_pre, accumulate, self.ws)

    def check_forward(self):
        ref = N.fwd(host(self.y), host(self.gate), host(self.w_post), self.post_norm, host(self.h), host(self.w_pre), self.alpha, self.beta, EPS)
        mag = np.abs(host(self.h))
        if self.y is not None:
            part = N.fwd(host(self.y), host(self.gate), host(self.w_post), self.post_norm, 0 * host(self.h), None, 1.0, self.beta, EPS)["h_out"]
            mag = abs(self.alpha) * mag + np.abs(part)
            close(self.h_out, ref["h_out"], mag, self.rt)
        for name in ("r_post", "r_pre"):
            if getattr(self, name) is not None:
                assert (np.abs(host(getattr(self, name)) / ref[name] - 1) <= 100 * 2.0 ** -24).all(), name
        if self.w_pre is not None:
            close(self.n, ref["n"], mag * ref["r_pre"][:, None] * np.abs(host(self.w_pre)), self.dt)

    def check_backward(self, accumulate=False, dh_out=True):
        ref, mag = N.bwd(host(self.y), host(self.gate), host(self.w_post), self.post_norm, host(self.saved), host(self.w_pre), host(self.r_post),
                         host(self.r_pre), host(self.dh_out) if dh_out else None, host(self.dn), self.alpha, self.beta)
        for name, value in ref.items():
            sums = name.startswith("dw")
            add = 1.0 if accumulate and sums else 0.0
            close(getattr(self, name), value + add, mag[name] + add, F32 if name == "dgate" else self.rt if name == "dh" else self.dt,
                  self.T / 512 + 160 if sums else 100, name)


def close(got, ref, mag, dtype, steps=100, name=""):
    got = host(got)
    assert np.isfinite(got).all(), name
    over = np.abs(got - ref) - (HALF_ULP[dtype] * np.abs(ref) * (1 + 2.0 ** -7) + steps * 2.0 ** -24 * mag)
    assert (over <= 0).all(), (name, float(over.max()), np.unravel_index(over.argmax(), over.shape))


TYPES = [(BF16, BF16), (BF16, F32), (F32, F32)]


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("T,d", [(0, 64), (1, 8), (1, 7168), (3, 520), (5, 16384), (65, 2880), (600, 512), (1030, 1032), (2, 9000)])
def test_sizes(T, d, dt, rt):
    print(f"case norm {T} {d} {dt} {rt}", flush=True)
    c = Case(T, d, dt, rt, seed=T + d)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("opts", [dict(post_norm=False), dict(w_post=False), dict(gate=False), dict(post_norm=False, w_post=False, gate=False),
                                  dict(y=False), dict(w_pre=False), dict(w_pre=False, post_norm=False), dict(alpha=1.0, beta=1.0)])
def test_options(opts, dt, rt):
    print(f"case norm {opts} {dt} {rt}", flush=True)
    for T, d in ((37, 264), (700, 1408)):       # (more rows than blocks walk at once)
        c = Case(T, d, dt, rt, seed=d, **opts)
        c.forward()
        c.check_forward()
        for accumulate, dh_out in ((False, True), (True, c.dn is None)):
            c.backward(accumulate, dh_out)
            c.check_backward(accumulate, dh_out)


def test_gradient_against_differences():
    c = Case(4, 24, F32, F32, alpha=0.75, beta=0.5)
    c.forward()
    c.backward()

    def loss(**change):
        a = dict(y=host(c.y), gate=host(c.gate), w_post=host(c.w_post), h=host(c.h), w_pre=host(c.w_pre))
        out = N.fwd(**{**a, **change}, post_norm=True, alpha=c.alpha, beta=c.beta, eps=EPS)
        return (out["n"] * host(c.dn)).sum() + (out["h_out"] * host(c.dh_out)).sum()

    for name, of in (("dh", "h"), ("dy", "y"), ("dgate", "gate"), ("dw_post", "w_post"), ("dw_pre", "w_pre")):
        base, got = host(getattr(c, of)), host(getattr(c, name))
        for at in list(np.ndindex(base.shape))[::7]:
            step = np.zeros_like(base)
            step[at] = 1e-5
            # central differences are off by about 1e-9 here, the fp32 gradient by 1e-5 at most
            assert abs((loss(**{of: base + step}) - loss(**{of: base - step})) / 2e-5 - got[at]) < 2e-5 * max(1, abs(got).max()), (name, at)


def test_in_place_and_optional_outputs():
    for dt, rt in TYPES:
        c = Case(33, 1040, dt, rt, seed=4)
        c.forward()
        ref = c.h_out.clone(), c.n.clone()
        h, y = c.h.clone(), c.y.clone()
        B.moe_block_norm_fwd(y, c.gate, c.w_post, True, h, c.w_pre, c.alpha, c.beta, EPS, h, y)             # h_out is h, n is y
        assert torch.equal(h, ref[0]) and torch.equal(y, ref[1])
        n = torch.empty_like(c.n)
        B.moe_block_norm_fwd(c.y, c.gate, c.w_post, True, c.h, c.w_pre, c.alpha, c.beta, EPS, None, n)      # h' is not stored
        assert torch.equal(n, ref[1])
        c.backward()
        want = [t.clone() for t in (c.dh, c.dy, c.dgate, c.dw_post, c.dw_pre)]
        dh_out, dn = c.dh_out.clone(), c.dn.clone()
        B.moe_block_norm_bwd(c.y, c.gate, c.w_post, True, c.h_out, c.w_pre, c.r_post, c.r_pre, dh_out, dn, c.alpha, c.beta, dh_out, dn, None,
                             None, None, False, c.ws)
        assert torch.equal(dh_out, want[0]) and torch.equal(dn, want[1])
        c.backward()                                                        # bit-reproducible
        assert all(torch.equal(a, b) for a, b in zip(want, (c.dh, c.dy, c.dgate, c.dw_post, c.dw_pre)))


def test_rows_of_zeros_and_of_nan_keep_to_themselves():
    c = Case(6, 776, F32, F32, gate=False)
    c.y[1], c.h[1] = 0, 0
    c.y[3, 5] = float("nan")
    c.h[4, 7] = float("inf")
    c.forward()
    n = host(c.n)
    assert not n[1].any() and np.isnan(n[3]).all() and not np.isfinite(n[4]).all()
    rows = [0, 1, 2, 5]
    ref = N.fwd(host(c.y[rows]), None, host(c.w_post), True, host(c.h[rows]), host(c.w_pre), c.alpha, c.beta, EPS)
    assert np.abs(n[rows] - ref["n"]).max() < 1e-5


def test_on_another_stream_and_in_a_graph():
    c = Case(300, 2048, BF16, F32, seed=9)
    c.forward()
    c.backward()
    names = ("h_out", "n", "dh", "dy", "dgate", "dw_post", "dw_pre")
    want = [getattr(c, n).clone() for n in names]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()

    def calls():
        B.moe_block_norm_fwd(c.y, c.gate, c.w_post, True, c.h, c.w_pre, c.alpha, c.beta, EPS, c.h_out, c.n, c.r_post, c.r_pre)
        B.moe_block_norm_bwd(c.y, c.gate, c.w_post, True, c.h_out, c.w_pre, c.r_post, c.r_pre, c.dh_out, c.dn, c.alpha, c.beta, c.dh, c.dy, c.dgate,
                             c.dw_post, c.dw_pre, False, c.ws)

    with torch.cuda.graph(graph, stream=side):
        calls()
    for _ in range(3):
        for n in names:
            getattr(c, n).fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(getattr(c, n), w) for n, w in zip(names, want))


@pytest.mark.parametrize("fault", ["strides", "dtype", "shape", "residual", "width", "wide", "eps", "n", "h_out", "flag", "host"])
def test_refusals(fault):
    c = Case(4, 64)
    c.h_out, c.n = torch.empty_like(c.h), torch.empty_like(c.y)
    a = dict(y=c.y, gate=c.gate, w_post=c.w_post, post_norm=True, h=c.h, w_pre=c.w_pre, alpha=1.0, beta=1.0, eps=EPS, h_out=c.h_out, n=c.n)
    B.moe_block_norm_fwd(**a)
    narrow = lambda k: {n: t[:, :k].contiguous() if t.dim() == 2 else t[:k].contiguous() if n != "gate" else t  # noqa: E731
                        for n, t in a.items() if isinstance(t, torch.Tensor)}
    wide = dict(y=torch.zeros(1, 16392, dtype=BF16, device="cuda"))
    a.update({"strides": dict(h=torch.zeros(64, 4, dtype=BF16, device="cuda").t()), "dtype": dict(n=c.n.float()), "shape": dict(gate=c.gate[:3]),
              "residual": dict(h=c.h.half(), h_out=c.h_out.half()), "width": narrow(60),
              "wide": dict(y=wide["y"], h=wide["y"], h_out=wide["y"], n=wide["y"], gate=None, w_post=None, w_pre=wide["y"][0]), "eps": dict(eps=0.0),
              "n": dict(n=None), "h_out": dict(y=None), "flag": dict(post_norm=2), "host": dict(w_pre=c.w_pre.cpu())}[fault])
    with pytest.raises(B.MoeError):
        B.moe_block_norm_fwd(**a)


def test_backward_refusals():
    c = Case(4, 64)
    c.forward()
    c.backward()
    a = dict(y=c.y, gate=c.gate, w_post=c.w_post, post_norm=True, h_out=c.h_out, w_pre=c.w_pre, r_post=c.r_post, r_pre=c.r_pre, dh_out=c.dh_out, dn=c.dn,
             alpha=1.0, beta=1.0, dh=c.dh, dy=c.dy, dgate=c.dgate, dw_post=c.dw_post, dw_pre=c.dw_pre, accumulate=False, ws=c.ws)
    B.moe_block_norm_bwd(**a)
    for change in (dict(r_pre=None), dict(r_post=None), dict(dy=None), dict(dn=None, dh_out=None), dict(w_pre=None), dict(ws=c.ws[:256]),
                   dict(y=None, dy=None), dict(dh=c.dh.float()), dict(accumulate=2), dict(dw_pre=c.dw_pre[:32])):
        with pytest.raises(B.MoeError):
            B.moe_block_norm_bwd(**{**a, **change})


@pytest.mark.parametrize("dt,rt", TYPES)
@pytest.mark.parametrize("T,d", [(530, 8200), (300, 16384), (2100, 1024), (700, 264), (8200, 520), (600, 4104)])
def test_blocks_that_walk_several_rows(T, d, dt, rt):
    """Column sums over a block's rows and wavefronts, and over blocks with a row more than others: every layout of rows in blocks."""
    print(f"case norm {T} {d} {dt} {rt}", flush=True)
    c = Case(T, d, dt, rt, seed=T + d)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
