"""Oracle of microscaled 4-bit numbers (numpy): the rounding by comparing distances, the layout by its index formula, the experts'
forward in float64."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """x [n, K] -> codes [n, K] (0..15) and scale bytes [n, K/32].  A chunk with an infinity or NaN: byte 255, codes 0."""
    x = np.asarray(x, np.float64)
    n, K = x.shape
    b = x.reshape(n, K // 32, 32)
    bad = ~np.isfinite(b).all(axis=2)
    b = np.where(bad[:, :, None], 0.0, b)
    top = np.abs(b).max(axis=2)
    _, e = np.frexp(top)                                    # top = m 2^e, m in [1/2, 1)
    exponent = np.where(top > 0, np.maximum(e - 1 - 2, -127), -127)
    v = np.abs(b) / np.exp2(exponent.astype(np.float64))[:, :, None]
    dist = np.abs(v[..., None] - GRID)
    nearest = dist.min(axis=-1, keepdims=True)
    tied = dist == nearest
    even = tied & (np.arange(8) % 2 == 0)
    code = np.where(even.any(axis=-1), even.argmax(axis=-1), tied.argmax(axis=-1))
    code = code + 8 * np.signbit(b)
    code[bad] = 0
    return code.reshape(n, K).astype(np.uint8), np.where(bad, 255, exponent + 127).astype(np.uint8)


def values(codes, scales):
    n, K = codes.shape
    v = np.where(codes >= 8, -1.0, 1.0) * GRID[codes & 7]
    s = np.exp2(scales.astype(np.float64) - 127)
    s[scales == 255] = np.nan
    return (v.reshape(n, K // 32, 32) * s[:, :, None]).reshape(n, K)


def tiles(codes, scales):
    """The library's layout: data [n/16][K/128][4][16][16], scales [n/16][K/512][4][16][4]."""
    n, K = codes.shape
    data = np.zeros((-(-n // 16), -(-K // 128), 4, 16, 16), np.uint8)
    sc = np.zeros((-(-n // 16), -(-K // 512), 4, 16, 4), np.uint8)
    i, k = np.meshgrid(np.arange(n), np.arange(K), indexing="ij")
    for odd in (0, 1):
        at = k % 2 == odd
        a, b = i[at], k[at]
        data[a // 16, b // 128, b % 128 // 32, a % 16, b % 32 // 2] |= codes[at] << (4 * odd)
    i, c = np.meshgrid(np.arange(n), np.arange(K // 32), indexing="ij")
    sc[i // 16, c // 16, c % 4, i % 16, c % 16 // 4] = scales
    return data, sc


def expert_fwd(xp, offsets, w1, w3, w2, h_err=0.0):
    """o [R, d] from the values of the 4-bit weights w1, w3 [e, f, d], w2 [e, d, f].  Also a bound [R, d] on what o can change by if every product
    h1, h3 is off by up to h_err times the sum of its terms' magnitudes: an activation that close to a halfway value, or a chunk's largest one that
    close to a power of two, may be rounded to its other neighbour."""
    R, d = int(offsets[-1]), w2.shape[1]
    o, slack = np.zeros((R, d)), np.zeros((R, d))
    for e in range(len(offsets) - 1):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if hi == lo:
            continue
        x = values(*quantize(xp[lo:hi]))
        h1, h3 = x @ w1[e].T, x @ w3[e].T
        s = 1.0 / (1.0 + np.exp(-h1))
        a = h1 * s * h3
        codes, scales = quantize(a)
        aq = values(codes, scales)
        o[lo:hi] = aq @ w2[e].T
        m1, m3 = np.abs(x) @ np.abs(w1[e]).T, np.abs(x) @ np.abs(w3[e]).T
        # |silu'| <= 1.1; the logistic function of the kernel is off by a few units in the last place
        da = h_err * (1.1 * m1 * np.abs(h3) + np.abs(h1 * s) * m3) + 2.0 ** -21 * np.abs(a)
        up, down = values(*quantize_as(a + da, scales)), values(*quantize_as(a - da, scales))
        moved = np.maximum(np.abs(up - aq), np.abs(down - aq))
        b = np.abs(a).reshape(hi - lo, -1, 32)
        top, at = b.max(axis=2), b.argmax(axis=2)
        dtop = np.take_along_axis(da.reshape(b.shape), at[:, :, None], axis=2)[:, :, 0]
        p = np.exp2(np.floor(np.log2(np.maximum(top, 1e-300))))
        edge = (top - dtop < p) | (top + dtop >= 2 * p)             # the chunk's scale may be the other one: off by up to half an element each
        moved = np.maximum(moved.reshape(b.shape), np.where(edge[:, :, None], np.maximum(b, 0.0) * 0.5 + p[:, :, None] / 4, 0.0)).reshape(a.shape)
        slack[lo:hi] = moved @ np.abs(w2[e]).T
    return o, slack


def quantize_as(x, scales):
    """As quantize, with the scales given."""
    n, K = x.shape
    v = np.abs(x).reshape(n, K // 32, 32) / np.exp2(scales.astype(np.float64) - 127)[:, :, None]
    code = np.abs(v[..., None] - GRID).argmin(axis=-1) + 8 * np.signbit(x.reshape(v.shape))
    return code.reshape(n, K).astype(np.uint8), scales
