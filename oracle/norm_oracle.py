"""Oracle of the norms between two blocks (numpy, float64): the definition and its gradient, term by term."""
import numpy as np


def _rms(x, eps):
    return 1.0 / np.sqrt((x * x).mean(axis=1) + eps)


def fwd(y, gate, w_post, post_norm, h, w_pre, alpha, beta, eps):
    """h' = alpha h + beta gate u, n = norm(h') w_pre; None in the place of y, gate, w_post, w_pre as in the library."""
    out = {"r_post": None, "n": None, "r_pre": None}
    h = np.asarray(h, np.float64)
    if y is not None:
        u = np.asarray(y, np.float64)
        if post_norm:
            out["r_post"] = _rms(u, eps)
            u = u * out["r_post"][:, None]
        u = u * (1.0 if w_post is None else np.asarray(w_post, np.float64))
        h = alpha * h + beta * (1.0 if gate is None else np.asarray(gate, np.float64)[:, None]) * u
    out["h_out"] = h
    if w_pre is not None:
        out["r_pre"] = _rms(h, eps)
        out["n"] = h * out["r_pre"][:, None] * np.asarray(w_pre, np.float64)
    return out


def bwd(y, gate, w_post, post_norm, h_out, w_pre, r_post, r_pre, dh_out, dn, alpha, beta):
    """Gradients at the saved sum and 1/rms.  mag: the size of the terms that meet in each output, for error bounds."""
    f = lambda a: None if a is None else np.asarray(a, np.float64)  # noqa: E731
    y, gate, w_post, h, w_pre, r_post, r_pre, dh_out, dn = map(f, (y, gate, w_post, h_out, w_pre, r_post, r_pre, dh_out, dn))
    shape = dn.shape if dn is not None else dh_out.shape
    T, d = shape
    gh, mag = (np.zeros(shape), np.zeros(shape)) if dh_out is None else (dh_out.copy(), np.abs(dh_out))
    out, m = {}, {}
    if dn is not None:
        r, t = r_pre[:, None], dn * w_pre
        gh = gh + r * t - h * r ** 3 * (t * h).mean(axis=1, keepdims=True)
        mag = mag + np.abs(r * t) + np.abs(h) * r ** 3 * np.abs(t * h).mean(axis=1, keepdims=True)
        out["dw_pre"], m["dw_pre"] = (dn * h * r).sum(axis=0), np.abs(dn * h * r).sum(axis=0)
    out["dh"], m["dh"] = (gh, mag) if y is None else (alpha * gh, abs(alpha) * mag)
    if y is not None:
        g = np.ones(T) if gate is None else gate
        w = np.ones(d) if w_post is None else w_post
        norm = y * r_post[:, None] if post_norm else y
        out["dgate"], m["dgate"] = beta * (gh * norm * w).sum(axis=1), abs(beta) * (mag * np.abs(norm * w)).sum(axis=1)
        du, mu = beta * g[:, None] * gh, np.abs(beta * g)[:, None] * mag
        out["dw_post"], m["dw_post"] = (du * norm).sum(axis=0), (mu * np.abs(norm)).sum(axis=0)
        du, mu = du * w, mu * np.abs(w)
        if post_norm:
            r = r_post[:, None]
            mu = r * mu + np.abs(y) * r ** 3 * (mu * np.abs(y)).mean(axis=1, keepdims=True)
            du = r * du - y * r ** 3 * (du * y).mean(axis=1, keepdims=True)
        out["dy"], m["dy"] = du, mu
    return out, m
