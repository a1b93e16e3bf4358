"""Oracle of the linear layer, grouped by expert or dense (numpy, float64): the definition and its gradient."""
import math

import numpy as np

_erfc = np.vectorize(math.erfc, otypes=[np.float64])
_S = math.sqrt(2.0 / math.pi)


def act(z, name):
    if name == "relu":
        return np.where(z < 0, 0.0, z)
    if name == "silu":
        return z / (1.0 + np.exp(-z))
    if name == "gelu":
        return 0.5 * z * _erfc(-z / math.sqrt(2.0))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + np.tanh(_S * (z + 0.044715 * z ** 3)))
    return z


def slope(z, name):
    if name == "relu":
        return np.where(z > 0, 1.0, 0.0)
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        return 0.5 * _erfc(-z / math.sqrt(2.0)) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if name == "gelu_tanh":
        t = np.tanh(_S * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * _S * (1.0 + 3 * 0.044715 * z * z)
    return np.ones_like(z)


def segments(offsets):
    return [(e, slice(int(offsets[e]), int(offsets[e + 1]))) for e in range(len(offsets) - 1)]


def fwd(x, offsets, w, bias, name, residual):
    """x [R,K], w [E,K,N], bias [E,N] or None, residual [R,N] or None -> z, y and mag, the sum of a z's terms' sizes."""
    R, N = x.shape[0], w.shape[2]
    z, mag = np.zeros((R, N)), np.zeros((R, N))
    for e, at in segments(offsets):
        z[at], mag[at] = x[at] @ w[e], np.abs(x[at]) @ np.abs(w[e])
        if bias is not None:
            z[at] += bias[e]
            mag[at] += np.abs(bias[e])
    y = act(z, name)
    return {"z": z, "y": y if residual is None else y + residual, "mag": mag}


def bwd(x, z, dy, offsets, w, name):
    """-> dz, dx, dw, db and the sums of their terms' sizes."""
    dz = dy if name == "none" else dy * slope(z, name)
    out = {"dz": dz, "dx": np.zeros_like(x), "dw": np.zeros(w.shape), "db": np.zeros((w.shape[0], w.shape[2]))}
    mag = {k: np.zeros_like(v) for k, v in out.items()}
    for e, at in segments(offsets):
        for o, f in ((out, lambda a: a), (mag, np.abs)):
            g = f(dz[at])
            o["dx"][at] = g @ f(w[e]).T
            o["dw"][e] = f(x[at]).T @ g
            o["db"][e] = g.sum(axis=0)
    return out, mag
