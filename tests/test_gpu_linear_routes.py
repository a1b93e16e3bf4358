"""The linear layer's kernels by the route that a call takes to them, against float64 on the device: the 256x256 tiles with every option, each gradient alone,
several rounds of the chip and weight gradients in pieces; few rows whose contraction is cut, with every option; the gradient of the bias alone.

Bounds, set before the first run.  Elementwise, as in test_gpu_linear.py: a bf16 store is off by at most 2^-8 of the value, an fp32 one by 2^-24; a sum over K terms by
(K + 4) 2^-23 of the sum of the terms' sizes; activations by (1 + |z|) 2^-21; dz in bf16 is rounded by 2^-8 once more.  That is a worst case and grows with
K, so a second bound holds for the root mean square over every block of 64 x 64 outputs.  Rounding to bf16 is off by a uniform part of at most 2^-8 of the value:
2^-8 / sqrt(3) of the block's root mean square.  Gradients behind an activation have two such roundings, 0.82 * 2^-8 together.  A sum's roundings, one per eight terms
or fewer times, all towards zero at worst, give up to K / 8 * 2^-23, 0.25 * 2^-8 for the largest K here (16400).  1.25 * 2^-8 leaves a tenth for chance: a block of
one row and 64 columns has 64 values of it, whose mean square of a uniform number is 1/3 +- 0.04.  What the bound is for, 32 of K terms left out, is off by
sqrt(32 / K), 0.04 for that K: eight times as much.  fp32: (K + 16) 2^-23 of the block's root mean square, 16 for the activation's slope."""
import math

import pytest
import torch

from paper_2605_11005_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
BLOCK = 64


def act_of(z, name):
    if name == "relu":
        return torch.relu(z)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def slope_of(z, name):
    z = z.clone().requires_grad_()
    return torch.autograd.grad(act_of(z, name).sum(), z)[0]


def near(got, ref, err, K, name, dt=BF16):
    """got within a rounding of ref, which itself may be off by err; and by blocks."""
    half = 2.0 ** -8 if dt == BF16 else 2.0 ** -24
    got = got.double()
    off = (got - ref).abs()
    assert not torch.isnan(off).any(), (name, "not a number")
    assert (off <= err + half * (ref.abs() + err)).all(), (name, "elementwise", float(off.max()))
    if got.dim() == 1:
        return
    squares = lambda t: torch.nn.functional.avg_pool2d((t * t)[None], BLOCK, ceil_mode=True, count_include_pad=False)[0]  # noqa: E731
    bound = 1.25 * 2.0 ** -8 if dt == BF16 else (K + 16) * 2.0 ** -23
    rms = (squares(off) / squares(ref)).sqrt()
    assert (rms <= bound).all(), (name, "blocks", float(rms.max()), bound)


class Layer:
    """rows: an int for a dense layer, a list of each expert's rows for a grouped one."""

    def __init__(self, rows, K, N, act="none", dt=BF16, bias=True, residual=True, save=True, seed=0):
        print(f"case linear {rows} {K} {N} {act} {dt} bias={bias} residual={residual} z={save}", flush=True)
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)  # noqa: E731
        self.dense, self.act, self.dt, self.save, self.K, self.N = isinstance(rows, int), act, dt, save, K, N
        counts = [rows] if self.dense else rows
        at = [0]
        for n in counts:
            at.append(at[-1] + n)
        self.segments, self.R, self.E = [slice(a, b) for a, b in zip(at, at[1:])], at[-1], len(counts)
        self.cap = self.R + (0 if self.dense else 5)
        self.off = None if self.dense else torch.tensor(at, dtype=torch.int32, device="cuda")
        self.lead = () if self.dense else (self.E,)
        self.x, self.dy = r(self.cap, K), r(self.cap, N)
        self.w = (torch.randn((*self.lead, K, N), generator=g, device="cuda") * K ** -0.5).to(dt)
        self.bias = r(*self.lead, N) if bias else None
        self.residual = r(self.cap, N) if residual else None
        self.noise = r

    def workspace(self, which):
        n = B.moe_workspace_bytes(which, B.MOE_BF16 if self.dt == BF16 else B.MOE_F32, 0, 0, self.K, self.N, self.E, self.cap)
        return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")

    def nan(self, *shape):
        return torch.full(shape, float("nan"), dtype=self.dt, device="cuda")

    @staticmethod
    def drew_tickets(ws):
        """The 256x256 tiles are drawn from counters at the workspace's beginning, which nothing else touches."""
        return bool((ws[:32].view(torch.int32) >= 0).all())

    def of(self, t, e):
        return None if t is None else t.double() if self.dense else t[e].double()

    def forward(self, in_place=False):
        """-> whether it took the 256x256 tiles"""
        self.z = self.nan(self.cap, self.N) if self.save else None
        self.y = self.residual.clone() if in_place else self.nan(self.cap, self.N)
        ws = self.workspace(B.WS_LINEAR_FWD)
        B.moe_linear_fwd(self.x, self.off, self.w, self.bias, B.ACTIVATIONS[self.act], self.y if in_place else self.residual, self.z, self.y, ws)
        for e, at in enumerate(self.segments):
            if at.start == at.stop:
                continue
            x, w, b = self.x[at].double(), self.of(self.w, e), self.of(self.bias, e)
            z, err = x @ w, x.abs() @ w.abs()
            if b is not None:
                z, err = z + b, err + b.abs()
            err *= (self.K + 4) * 2.0 ** -23
            if self.z is not None:
                near(self.z[at], z, err, self.K, f"z {e}", self.dt)
            y = act_of(z, self.act)
            if self.residual is not None:
                y = y + self.residual[at].double()
            err = 1.13 * err + 2.0 ** -23 * y.abs() + (0 if self.act == "none" else (1 + z.abs()) * 2.0 ** -21)
            near(self.y[at], y, err, self.K, f"y {e}", self.dt)
        if not self.dense:
            past = self.y[self.R:]
            assert torch.equal(past, self.residual[self.R:]) if in_place else torch.isnan(past).all(), "rows past the last expert's"
        return self.drew_tickets(ws)

    def backward(self, want=("dx", "dw", "db"), accumulate=False, z=None):
        """at a given z, else the forward's; accumulate: onto numbers of dy's size.  -> whether it took the 256x256 tiles"""
        z = self.z if z is None else z
        through = self.act != "none"
        shapes = dict(dx=(self.cap, self.K), dw=(*self.lead, self.K, self.N), db=(*self.lead, self.N))
        old = {n: self.noise(*shapes[n]) if accumulate else self.nan(*shapes[n]) for n in want}
        out = {n: t.clone() for n, t in old.items()}
        ws = self.workspace(B.WS_LINEAR_BWD)
        B.moe_linear_bwd(self.x, z if through else None, self.dy, self.off, self.w, B.ACTIVATIONS[self.act], out.get("dx"), out.get("dw"), out.get("db"),
                         accumulate, ws, accumulate)
        half = 2.0 ** -8 if self.dt == BF16 else 2.0 ** -24
        for e, at in enumerate(self.segments):
            x, w, dz, n = self.x[at].double(), self.of(self.w, e), self.dy[at].double(), at.stop - at.start
            dz_err = torch.zeros_like(dz)
            if through and n:
                zd = z[at].double()
                dz_err = (1 + zd.abs()) * 2.0 ** -20 * dz.abs() if self.act != "relu" else dz_err
                dz = dz * slope_of(zd, self.act)
            rounded = dz_err + (half * (dz.abs() + dz_err) if through and self.dt == BF16 else 0)
            parts = dict(dx=lambda: (dz @ w.T, rounded @ w.abs().T + (self.N + 4) * 2.0 ** -23 * (dz.abs() @ w.abs().T), self.N),
                         dw=lambda: (x.T @ dz, x.abs().T @ rounded + (n + 40) * 2.0 ** -23 * (x.abs().T @ dz.abs()), n),
                         db=lambda: (dz.sum(0), dz_err.sum(0) + (n + 4) * 2.0 ** -23 * dz.abs().sum(0), n))
            for name in want:
                ref, err, terms = parts[name]()
                got, was = ((out[name][at], old[name][at]) if name == "dx" else (out[name], old[name]) if self.dense else (out[name][e], old[name][e]))
                if n == 0:
                    assert name == "dx" or torch.equal(got, was if accumulate else torch.zeros_like(got)), (name, e, "without rows")
                    continue
                if accumulate:
                    ref, err = ref + was.double(), err + 2.0 ** -23 * (ref + was.double()).abs()
                near(got, ref, err, terms, f"{name} {e}", self.dt)
        if "dx" in want and not self.dense:
            assert torch.equal(out["dx"][self.R:].isnan(), old["dx"][self.R:].isnan()) and torch.equal(out["dx"][self.R:].nan_to_num(), old["dx"][self.R:].nan_to_num())
        return self.drew_tickets(ws)


@pytest.mark.parametrize("act,bias,residual,save", [("gelu", False, True, True), ("relu", True, False, False), ("none", True, False, True), ("gelu_tanh", False, False, True),
                                                    ("silu", True, True, False), ("none", False, False, False)])
def test_largest_tiles_forward(act, bias, residual, save):
    """One matrix of 4088 by 4088 (the contraction ends inside a k-tile), 4096 rows."""
    assert Layer(4096, 4088, 4088, act, bias=bias, residual=residual, save=save).forward()


@pytest.mark.parametrize("act,save", [("gelu", True), ("none", False)])
def test_largest_tiles_onto_the_residual(act, save):
    assert Layer(4096, 4088, 4088, act, save=save).forward(in_place=True)


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("want", [("dx", "dw", "db"), ("dx", "dw"), ("dx",), ("dw",), ("dw", "db")], ids="-".join)
@pytest.mark.parametrize("accumulate", [False, True])
def test_largest_tiles_gradients(act, want, accumulate):
    c = Layer(4096, 4088, 4088, act, residual=False)
    assert c.backward(want, accumulate, c.noise(c.cap, c.N))


@pytest.mark.parametrize("rows", [[2050, 2051, 2049, 2053], [7000, 1, 0, 1202], [0, 300, 7603, 300], [3, 2, 8190, 8]], ids=str)
def test_largest_tiles_of_experts(rows):
    """Four experts of 4096 to 4104, alike and unlike in rows: several rounds, and weight gradients of a heavy expert in pieces."""
    c = Layer(rows, 4096, 4104, "gelu_tanh")
    assert c.forward() and c.backward()
    assert c.backward(("dx", "dw"), True)
    c.bias, c.residual, c.save, c.act = None, None, False, "silu"
    assert c.forward()


def test_largest_tiles_in_many_rounds():
    """16380 rows of 14328 to 2040: fourteen rounds of dx's tiles, so that dx and dW are two launches."""
    c = Layer(16380, 14328, 2040, "gelu", residual=False)
    assert c.forward() and c.backward()
    c.act = "none"
    assert c.backward(("dx", "dw"), True)


@pytest.mark.parametrize("dt", (BF16, F32))
@pytest.mark.parametrize("rows", [1, 5, 17, [3, 0, 7, 1], [20, 0, 40, 1]], ids=str)
@pytest.mark.parametrize("bias,residual,save", [(False, True, True), (True, False, False), (False, False, False), (True, True, True)])
def test_few_rows_of_long_contractions(rows, dt, bias, residual, save):
    """4104 inputs (2052 in fp32) whose contraction is cut and whose parts a second launch adds up, to 136 outputs."""
    K, N = (4104, 136) if dt == BF16 else (2052, 132)
    for act in ("none", "gelu"):
        c = Layer(rows, K, N, act, dt, bias, residual, save)
        assert not c.forward()
        if residual:
            c.forward(in_place=True)
        c.backward(z=c.noise(c.cap, N))
        c.backward(("db",), True, c.noise(c.cap, N))


@pytest.mark.parametrize("dt", (BF16, F32))
@pytest.mark.parametrize("rows", [100, 1500, [70, 0, 300, 5]], ids=str)
def test_onto_the_residual(rows, dt):
    for K, N in ((264, 520), (4104, 136)):
        for act in ("none", "silu"):
            Layer(rows, K, N, act, dt).forward(in_place=True)


@pytest.mark.parametrize("dt", (BF16, F32))
@pytest.mark.parametrize("rows", [600, 641, 3000, 9000, [1500, 0, 900, 3, 700]], ids=str)
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_gradient_of_the_bias_alone(rows, act, dt):
    for N in (264, 1032):
        for accumulate in (False, True):
            c = Layer(rows, 72, N, act, dt)
            c.backward(("db",), accumulate, c.noise(c.cap, N))


@pytest.mark.parametrize("rows,K,N,dt", [(4, 8200, 16392, BF16), (100, 16392, 8200, BF16), (700, 16392, 1032, BF16), ([3, 0, 40, 1, 2], 16392, 1032, BF16),
                                         ([700, 30, 0, 2000], 8200, 1032, BF16), (16384, 264, 520, BF16), (300, 8196, 516, F32), ([40, 0, 500], 4100, 260, F32),
                                         (9000, 260, 516, F32)], ids=str)
def test_long_contractions_by_blocks(rows, K, N, dt):
    """A step of the contraction left out would pass the worst case's bound here, and not the blocks'."""
    c = Layer(rows, K, N, "none", dt)
    c.forward()
    c.backward()
