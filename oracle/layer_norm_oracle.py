"""Oracle of the layer norm between two blocks (numpy, float64): the definition and its gradient, term by term."""
import numpy as np


def fwd(y, h, w, b, eps):
    """h' = h + y, n = layernorm(h') w + b; None in the place of y, w, b as in the library."""
    h = np.asarray(h, np.float64) if y is None else np.asarray(h, np.float64) + np.asarray(y, np.float64)
    mean = h.mean(axis=1)
    centred = h - mean[:, None]
    rstd = 1.0 / np.sqrt((centred * centred).mean(axis=1) + eps)
    n = centred * rstd[:, None] * (1.0 if w is None else np.asarray(w, np.float64)) + (0.0 if b is None else np.asarray(b, np.float64))
    return {"h_out": h, "mean": mean, "rstd": rstd, "n": n}


def bwd(h_out, w, mean, rstd, dh_out, dn):
    """Gradients at the saved sum, mean and 1/deviation.  mag: the size of the terms that meet in each output, for error bounds."""
    h, mean, r, dn = (np.asarray(a, np.float64) for a in (h_out, mean[:, None], rstd[:, None], dn))
    xh = (h - mean) * r
    size = (np.abs(h) + np.abs(mean)) * r
    t = dn if w is None else dn * np.asarray(w, np.float64)
    dh = r * (t - t.mean(axis=1, keepdims=True) - xh * (t * xh).mean(axis=1, keepdims=True))
    m = r * (np.abs(t) + np.abs(t).mean(axis=1, keepdims=True) + size * (np.abs(t) * size).mean(axis=1, keepdims=True))
    if dh_out is not None:
        dh, m = dh + np.asarray(dh_out, np.float64), m + np.abs(np.asarray(dh_out, np.float64))
    out = {"dh": dh, "dy": dh, "dw": (dn * xh).sum(axis=0), "db": dn.sum(axis=0)}
    return out, {"dh": m, "dy": m, "dw": (np.abs(dn) * size).sum(axis=0), "db": np.abs(dn).sum(axis=0)}
