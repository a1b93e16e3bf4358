"""Pins of the linear layer's and the layer norm's oracles: torch's own functions and autograd in float64, and closed forms."""
import numpy as np
import pytest
import torch

from oracle import layer_norm_oracle as LN
from oracle import linear_oracle as L

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
F = torch.nn.functional
LIBRARY = dict(none=lambda z: z, relu=F.relu, gelu=F.gelu, gelu_tanh=lambda z: F.gelu(z, approximate="tanh"), silu=F.silu)


def rand(rng, *shape):
    return rng.standard_normal(shape)


@pytest.mark.parametrize("act", ACTS)
def test_linear_is_torchs(act):
    rng = np.random.default_rng(1)
    offsets, K, N = [0, 3, 3, 8, 9], 5, 7
    x, w, b, res, dy = rand(rng, 9, K), rand(rng, 4, K, N), rand(rng, 4, N), rand(rng, 9, N), rand(rng, 9, N)
    t = lambda a: torch.tensor(a, requires_grad=True)  # noqa: E731
    tx, tw, tb, tr = t(x), t(w), t(b), t(res)
    ty = torch.cat([LIBRARY[act](tx[at] @ tw[e] + tb[e]) for e, at in L.segments(offsets)]) + tr
    fw = L.fwd(x, offsets, w, b, act, res)
    assert np.allclose(fw["y"], ty.detach().numpy(), rtol=1e-12, atol=1e-12)
    ty.backward(torch.tensor(dy))
    bw, _ = L.bwd(x, fw["z"], dy, offsets, w, act)
    for name, got in (("dx", tx.grad), ("dw", tw.grad), ("db", tb.grad)):
        assert np.allclose(bw[name], got.numpy(), rtol=1e-11, atol=1e-12), name
    assert np.array_equal(tr.grad.numpy(), dy)
    assert not bw["dw"][1].any() and not bw["db"][1].any()          # an expert without rows


def test_activations_at_known_points():
    z = np.array([0.0, 1.0, -1.0])
    assert np.allclose(L.act(z, "gelu"), [0, 0.8413447460685429, -0.15865525393145707], atol=1e-15)
    assert np.allclose(L.act(z, "silu"), [0, 0.7310585786300049, -0.2689414213699951], atol=1e-15)
    assert list(L.act(z, "relu")) == [0, 1, 0] and list(L.slope(z, "relu")) == [0, 1, 0]
    for name in ACTS:                                               # central differences, away from relu's corner
        p, step = np.array([-3.3, -0.7, 0.2, 1.9]), 1e-6
        assert np.allclose((L.act(p + step, name) - L.act(p - step, name)) / (2 * step), L.slope(p, name), atol=1e-8), name


@pytest.mark.parametrize("through", (False, True))
def test_layer_norm_is_torchs(through):
    rng = np.random.default_rng(2)
    T, d, eps = 6, 11, 1e-5
    y, h, w, b, dn, dh_out = rand(rng, T, d), 3 + rand(rng, T, d), rand(rng, d), rand(rng, d), rand(rng, T, d), rand(rng, T, d)
    t = lambda a: torch.tensor(a, requires_grad=True)  # noqa: E731
    ty, th, tw, tb = t(y), t(h), t(w), t(b)
    ts = th + ty
    tn = F.layer_norm(ts, (d,), tw, tb, eps)
    fw = LN.fwd(y, h, w, b, eps)
    assert np.allclose(fw["n"], tn.detach().numpy(), rtol=1e-12, atol=1e-12)
    ((tn * torch.tensor(dn)).sum() + ((ts * torch.tensor(dh_out)).sum() if through else 0)).backward()
    bw, _ = LN.bwd(fw["h_out"], w, fw["mean"], fw["rstd"], dh_out if through else None, dn)
    for name, got in (("dh", th.grad), ("dy", ty.grad), ("dw", tw.grad), ("db", tb.grad)):
        assert np.allclose(bw[name], got.numpy(), rtol=1e-10, atol=1e-11), name


def test_layer_norm_of_a_constant_row():
    fw = LN.fwd(None, np.full((1, 8), 7.0), None, None, 1e-5)
    assert not fw["n"].any() and fw["mean"][0] == 7 and np.isclose(fw["rstd"][0], 1e-5 ** -0.5)
    bw, _ = LN.bwd(fw["h_out"], None, fw["mean"], fw["rstd"], None, np.arange(8.0)[None])
    assert np.isclose(bw["dh"].sum(), 0.0, atol=1e-9)               # the gradient has no mean
