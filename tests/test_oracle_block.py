"""Pins of the oracles of the norms between blocks and of microscaled 4-bit numbers: closed forms, hand-worked numbers, differences and
another library's differentiation."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as M
from oracle import norm_oracle as N

CASES = [(True, True, True, 1.0, 1.0), (True, False, False, 0.5, 2.0), (False, True, True, 1.0, 0.25), (False, False, False, -1.5, 1.0)]


def _inputs(post_norm, weighted, gated, T=5, d=12, seed=0):
    g = np.random.default_rng(seed)
    y, h = g.standard_normal((T, d)), g.standard_normal((T, d))
    return dict(y=y, gate=g.random(T) if gated else None, w_post=1 + g.standard_normal(d) / 3 if weighted else None, post_norm=post_norm, h=h,
                w_pre=1 + g.standard_normal(d) / 3)


def test_norm_closed_forms():
    # a row of equal elements c has rms |c|: its norm is sign(c)
    h = np.array([[3.0] * 8, [-0.25] * 8])
    out = N.fwd(None, None, None, False, h, np.arange(8.0), 1.0, 1.0, 0.0)
    assert np.allclose(out["n"], np.sign(h) * np.arange(8.0)) and np.allclose(out["r_pre"], [1 / 3, 4])
    # a norm with unit weights has mean square 1 whatever its input's scale
    y = np.random.default_rng(1).standard_normal((3, 64)) * np.array([[1e-3], [1.0], [1e3]])
    out = N.fwd(y, None, None, True, np.zeros((3, 64)), np.ones(64), 1.0, 1.0, 0.0)
    assert np.allclose((out["h_out"] ** 2).mean(axis=1), 1) and np.allclose(out["h_out"], out["n"])


@pytest.mark.parametrize("case", CASES)
def test_norm_gradient_against_differences_and_torch(case):
    post_norm, weighted, gated, alpha, beta = case
    i = _inputs(post_norm, weighted, gated)
    g = np.random.default_rng(2)
    dn, dh_out = g.standard_normal(i["h"].shape), g.standard_normal(i["h"].shape)
    eps = 1e-3
    fw = N.fwd(**i, alpha=alpha, beta=beta, eps=eps)
    got, mag = N.bwd(i["y"], i["gate"], i["w_post"], post_norm, fw["h_out"], i["w_pre"], fw["r_post"], fw["r_pre"], dh_out, dn, alpha, beta)

    def loss(**change):
        out = N.fwd(**{**i, **change}, alpha=alpha, beta=beta, eps=eps)
        return (out["n"] * dn).sum() + (out["h_out"] * dh_out).sum()

    for name, of in (("dh", "h"), ("dy", "y"), ("dgate", "gate"), ("dw_post", "w_post"), ("dw_pre", "w_pre")):
        if i[of] is None:
            continue
        for at in list(np.ndindex(i[of].shape))[::5]:
            plus, minus = i[of].copy(), i[of].copy()
            plus[at] += 1e-5
            minus[at] -= 1e-5
            assert abs((loss(**{of: plus}) - loss(**{of: minus})) / 2e-5 - got[name][at]) < 1e-7, (name, at)
        assert (np.abs(got[name]) <= mag[name] * (1 + 1e-12)).all()
    # torch's differentiation of the same formula
    t = {n: torch.tensor(i[n], requires_grad=True) for n in ("y", "gate", "w_post", "h", "w_pre") if i[n] is not None}
    u = t["y"] * torch.rsqrt(t["y"].square().mean(1, keepdim=True) + eps) if post_norm else t["y"]
    u = u * t["w_post"] if weighted else u
    u = u * t["gate"][:, None] if gated else u
    h = alpha * t["h"] + beta * u
    n = h * torch.rsqrt(h.square().mean(1, keepdim=True) + eps) * t["w_pre"]
    ((n * torch.tensor(dn)).sum() + (h * torch.tensor(dh_out)).sum()).backward()
    for name, of in (("dh", "h"), ("dy", "y"), ("dgate", "gate"), ("dw_post", "w_post"), ("dw_pre", "w_pre")):
        if of in t:
            assert np.allclose(t[of].grad.numpy(), got[name], rtol=1e-10, atol=1e-12), name


def test_mx4_hand_worked_chunk():
    x = np.zeros((1, 32))
    # the largest magnitude 7 lies in [4, 8): scale 1.  Halfway values go to the even code; what is past 6 saturates.
    x[0, :14] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7, -5, 0.2, 0, -0.1, -0.26, 5.01]
    codes, scales = M.quantize(x)
    assert scales.tolist() == [[127]]
    assert M.values(codes, scales)[0, :14].tolist() == [0, 1, 1, 2, 2, 4, 4, 6, -4, 0, 0, 0, -0.5, 6]
    assert codes[0, 11] == 8                                    # a negative number that rounds to zero keeps its sign
    codes, scales = M.quantize(x * 2.0 ** -9)
    assert scales.tolist() == [[118]] and M.values(codes, scales)[0, 7] == 6 * 2.0 ** -9


def test_mx4_edges_of_the_range():
    x = np.zeros((4, 32))
    x[1, 3], x[2, 3], x[3, 3] = np.inf, 2.0 ** -149, 3e38
    codes, scales = M.quantize(x)
    assert scales[:, 0].tolist() == [0, 255, 0, 127 + 127 - 2] and not codes[:3].any()
    v = M.values(codes, scales)
    assert not v[0].any() and np.isnan(v[1]).all() and not v[2].any() and v[3, 3] == 6 * 2.0 ** 125     # (3e38 = 7.05 * 2^125)


@pytest.mark.parametrize("n,K", [(1, 32), (17, 160), (33, 1056)])
def test_mx4_is_the_nearest_value_and_layout_inverts(n, K):
    x = np.random.default_rng(n).standard_normal((n, K)) * 3
    codes, scales = M.quantize(x)
    v = M.values(codes, scales)
    s = np.exp2(scales.astype(float) - 127).repeat(32, axis=1)
    assert (np.abs(v - x) <= np.where(np.abs(x) < 2 * s, 0.25, np.where(np.abs(x) < 4 * s, 0.5, 1.0)) * s * np.where(np.abs(x) > 6 * s, 2, 1)).all()
    data, sc = M.tiles(codes, scales)
    i, k = n - 1, K - 1
    assert data[i // 16, k // 128, k % 128 // 32, i % 16, k % 32 // 2] >> 4 == codes[i, k]
    assert sc[i // 16, k // 512, k % 128 // 32, i % 16, k % 512 // 128] == scales[i, k // 32]
    back = np.zeros_like(codes)
    for r in range(n):
        row = data[r // 16, :, :, r % 16].reshape(-1)
        back[r, 0::2], back[r, 1::2] = (row & 15)[:K // 2], (row >> 4)[:K // 2]
    assert (back == codes).all()


def test_mx4_experts_equal_a_dense_formula_on_exact_values():
    g = np.random.default_rng(3)
    e, f, d = 3, 64, 32
    w1, w3, w2 = (g.choice([-1.0, -0.5, 0.5, 1.0], size=s) for s in ((e, f, d), (e, f, d), (e, d, f)))
    xp = g.choice([-2.0, -1.0, 0.0, 1.0, 4.0], size=(5, d))
    o, slack = M.expert_fwd(xp, [0, 2, 2, 5], w1, w3, w2)
    for row, x in enumerate(xp):
        i = 0 if row < 2 else 2
        h1, h3 = w1[i] @ x, w3[i] @ x
        a = M.values(*M.quantize((h1 / (1 + np.exp(-h1)) * h3)[None]))[0]
        assert np.allclose(o[row], w2[i] @ a, rtol=1e-12)
    assert (slack >= 0).all()
    # a planted mistake in the oracle's operands is seen
    assert not np.allclose(M.expert_fwd(xp, [0, 2, 2, 5], w3, w1, w2)[0], o)
