"""Products grouped by expert, products with bias, activation and residual, and layer norm, for timing: what a block of experts of two
matrices with biases, a dense expert beside them and layer norms in front of both calls beside router, dispatch and combine.

A case's "op" is one of

  norm_fwd     h' = h + y and n = layernorm(h') w + b
  norm_bwd     its gradient in h (and y) and in both weights, from the saved h', mean and 1/deviation
  product_fwd  y = act(x W + b) + residual, and z = x W + b where training keeps it
  product_bwd  its gradient in x, W and b, from the saved x and z

A product with "experts" > 0 is grouped: rows of x lie expert after expert, each with a matrix and a bias of its own, as many rows each as a
routing left it.  Sizes are those of workloads.py's configurations or generic.
"""
import math

import torch

own = False

EPS = 1e-5
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


# --------------------------------------------------------------------------------------------------------- cases
def _norm(op, T, d, dtype="bf16", residual="bf16", add=True, through=True):
    # add: a block's output y is added to h first.  through: h' has a gradient of its own from further on.
    return dict(op=op, T=T, d=d, dtype=dtype, residual=residual, add=add, through=through)


def _dense(op, T, K, N, act="none", dtype="bf16", bias=True, residual=False, train=False):
    return dict(op=op, experts=0, T=T, K=K, N=N, act=act, dtype=dtype, bias=bias, residual=residual, train=train)


def _grouped(op, T, K, N, E, experts, k, zipf, act="none", dtype="bf16", bias=True, train=False):
    return dict(op=op, experts=experts, E=E, k=k, zipf=zipf, T=T, K=K, N=N, act=act, dtype=dtype, bias=bias, residual=False, train=train)


def listed():
    cases = {
        # one decode step of a small batch in front of a block: latency counts
        "norm-fwd-decode-t4": _norm("norm_fwd", 4, 4096),
        # a training step's tokens with the residual stream in fp32
        "norm-fwd-t32768": _norm("norm_fwd", 32768, 7168, residual="f32"),
        # one odd prompt's gradient at a hidden size that is no power of two
        "norm-bwd-t2047": _norm("norm_bwd", 2047, 2880),
        # a training step's gradient
        "norm-bwd-t16384": _norm("norm_bwd", 16384, 4096, residual="f32"),
        # a decode step of a large serving batch on the largest share: 14 to 18 of the experts have a few rows each
        "grouped-fwd-decode-t128": _grouped("product_fwd", 128, 7168, 2048, 256, 32, 8, 1.0, act="silu"),
        # prefill of one prompt of odd length
        "grouped-fwd-prefill-t2047": _grouped("product_fwd", 2047, 2880, 2880, 128, 16, 4, 1.0, act="gelu_tanh"),
        # a training step's first product of few large experts
        "grouped-fwd-8x14336": _grouped("product_fwd", 8192, 4096, 14336, 8, 8, 2, 0.3, act="gelu", train=True),
        # an fp32 layer of a size that one debugs with, widths off the tiles
        "grouped-bwd-fp32-t1500": _grouped("product_bwd", 1500, 520, 776, 64, 16, 6, 0.5, act="silu", dtype="f32", train=True),
        # a training step's gradient of the second product of few large experts
        "grouped-bwd-8x14336": _grouped("product_bwd", 4096, 14336, 4096, 8, 8, 2, 0.3, train=True),
        # one decode step of a small batch through a dense expert
        "dense-fwd-decode-t4": _dense("product_fwd", 4, 4096, 14336, act="gelu_tanh"),
        # a dense expert's second product with the residual
        "dense-fwd-t8192": _dense("product_fwd", 8192, 14336, 4096, residual=True),
        # a training step's gradient of a shared expert's first product
        "dense-bwd-t16384": _dense("product_bwd", 16384, 7168, 2048, act="gelu", train=True),
    }
    return [dict(case, name=name) for name, case in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_PRODUCTS = 16384 * 4096 * 14336        # rows x K x N of the largest listed forward; a backward has twice the products


def draw(rng):
    op = rng.choice(("norm_fwd", "norm_bwd", "product_fwd", "product_fwd", "product_bwd", "product_bwd"))
    if op in ("norm_fwd", "norm_bwd"):
        dtype = rng.choice(("bf16", "bf16", "f32"))
        return _norm(op, _log_int(rng, 1, 16384), 8 * _log_int(rng, 8, 896), dtype, "f32" if dtype == "f32" else rng.choice(("bf16", "f32")),
                     add=rng.random() < 0.7, through=rng.random() < 0.7)
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    step, most = (8, 14336) if dtype == "bf16" else (4, 2048)
    if rng.random() < 0.5:      # the sizes that models have
        K, N = (rng.choice([n for n in (768, 1408, 2048, 2880, 4096, 7168, 14336) if n <= most]) for _ in range(2))
    else:
        K, N = (step * _log_int(rng, 64 // step, most // step) for _ in range(2))
    act = rng.choice(ACTS)
    train = op == "product_bwd" or rng.random() < 0.4
    products = (1 if op == "product_fwd" else 0.5) * MOST_PRODUCTS * (1 if dtype == "bf16" else 1 / 16)
    rows = max(1, min(16384, int(products / (K * N))))
    if rng.random() < 0.4:
        return _dense(op, _log_int(rng, 1, rows), K, N, act, dtype, bias=rng.random() < 0.8, residual=op == "product_fwd" and rng.random() < 0.4,
                      train=train)
    E, experts, k = rng.choice(((8, 8, 2), (64, 8, 4), (128, 16, 8), (256, 32, 8), (16, 4, 1), (60, 15, 4)))
    while experts * K * N > 8 * 4096 * 14336:       # (no more weights than the largest listed case)
        E, experts = (E + 1) // 2, (experts + 1) // 2
    k = min(k, E)
    T = max(1, rows * E // (experts * k))
    return _grouped(op, _log_int(rng, 1, min(T, 32768)), K, N, E, experts, k, rng.choice((0.0, 0.5, 1.0)), act, dtype, bias=rng.random() < 0.8,
                    train=train)


# --------------------------------------------------------------------------------------------------------- inputs
class _State:
    pass


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _rows_of(case):
    """Rows of each local expert, the same for all inputs of a case (they are the outputs' shape): the top k of N(0,1) logits with
    a popularity by rank, experts' ranks in a drawn order."""
    E = case["E"]
    g = torch.Generator(device="cuda").manual_seed(case["T"] + E)
    rank = torch.randperm(E, generator=g, device="cuda") + 1
    logits = torch.randn((case["T"], E), generator=g, device="cuda") - case["zipf"] * rank.float().log()
    rows = torch.bincount(logits.topk(case["k"], dim=1).indices.reshape(-1), minlength=E)[:case["experts"]]
    if not int(rows.sum()):         # a share that none of the tokens reached would make no call
        rows[0] = 1
    return rows


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = _State()
    s.case = case
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    empty = lambda *shape, dtype: torch.empty(shape, device="cuda", dtype=dtype)  # noqa: E731
    dt = _dtype(case["dtype"])
    if case["op"] in ("norm_fwd", "norm_bwd"):
        T, d, rt = case["T"], case["d"], _dtype(case["residual"])
        # a residual stream whose channels differ in size and in mean, as trained ones do
        s.h = (randn(T, d) * torch.exp(0.5 * randn(d)) + 0.5 * randn(d)).to(rt)
        s.y = (0.5 * randn(T, d)).to(dt) if case["add"] else None
        s.w, s.b = (1.0 + 0.1 * randn(d)).to(dt), (0.1 * randn(d)).to(dt)
        s.n = empty(T, d, dtype=dt)
        s.h_out = empty(T, d, dtype=rt) if case["add"] else None
        s.mean, s.rstd = empty(T, dtype=torch.float32), empty(T, dtype=torch.float32)
        if case["op"] == "norm_bwd":
            h, mean, rstd = _moments(s)
            s.h_out = h.to(rt)
            s.mean.copy_(mean[:, 0])
            s.rstd.copy_(rstd[:, 0])
            del s.h, s.y
            s.dn = randn(T, d).to(dt)
            s.dh_out = randn(T, d).to(rt) if case["through"] else None
            s.dh = empty(T, d, dtype=rt)
            # the gradient of y is that of h; a stream in another type is written in both
            s.dy = empty(T, d, dtype=dt) if case["add"] and rt != dt else None
            s.dw, s.db = empty(d, dtype=dt), empty(d, dtype=dt)
            s.ws = empty((1 << 20) + 2 * 4 * 4096 * d, dtype=torch.uint8)
        return s
    K, N, experts = case["K"], case["N"], case["experts"]
    lead = (experts,) if experts else ()
    if experts:
        rows = _rows_of(case)
        s.rows = rows.tolist()
        s.offsets = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
        s.offsets[1:] = rows.cumsum(0)
        R = sum(s.rows)
        cap = R + R // 20 + 8       # a program's buffers hold more rows than a step's routing fills
    else:
        s.rows, s.offsets, R = [case["T"]], None, case["T"]
        cap = R
    s.x = randn(cap, K).to(dt)
    s.w = empty(*lead, K, N, dtype=dt)
    for w in s.w if experts else (s.w,):
        w.copy_(randn(K, N) * K ** -0.5)
    s.bias = (0.1 * randn(*lead, N)).to(dt) if case["bias"] else None
    if case["op"] == "product_fwd":
        s.residual = randn(cap, N).to(dt) if case["residual"] else None
        s.z = empty(cap, N, dtype=dt) if case["train"] and case["act"] != "none" else None
        s.y = empty(cap, N, dtype=dt)
        s.ws = empty(256 << 20, dtype=torch.uint8)
    else:
        s.z = randn(cap, N).to(dt) if case["act"] != "none" else None
        s.dy = randn(cap, N).to(dt)
        s.dx = empty(cap, K, dtype=dt)
        s.dw = empty(*lead, K, N, dtype=dt)
        s.db = empty(*lead, N, dtype=dt) if case["bias"] else None
        s.ws = empty((1 << 30) + 2 * cap * N * s.x.element_size(), dtype=torch.uint8)
    return s


# --------------------------------------------------------------------------------------------------------- plain forms
def _moments(s):
    h = s.h.float() if s.y is None else s.h.float() + s.y.float()
    mean = h.mean(dim=1, keepdim=True)
    return h, mean, torch.rsqrt((h - mean).square().mean(dim=1, keepdim=True) + EPS)


def _norm_fwd(s):
    h, mean, rstd = _moments(s)
    out = {"n": ((h - mean) * rstd * s.w.float() + s.b.float()).to(s.n.dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if s.y is not None:
        out["h_out"] = h.to(s.h.dtype)
    return out


def _norm_bwd(s):
    dn, rstd = s.dn.float(), s.rstd[:, None]
    xh = (s.h_out.float() - s.mean[:, None]) * rstd
    t = dn * s.w.float()
    dh = rstd * (t - t.mean(dim=1, keepdim=True) - xh * (t * xh).mean(dim=1, keepdim=True))
    if s.dh_out is not None:
        dh = dh + s.dh_out.float()
    out = {"dh": dh.to(s.dh.dtype), "dw": (dn * xh).sum(dim=0).to(s.dw.dtype), "db": dn.sum(dim=0).to(s.db.dtype)}
    if s.dy is not None:
        out["dy"] = dh.to(s.dy.dtype)
    return out


def _tanh_of(z):
    """tanh(sqrt(2/pi) (z + 0.044715 z^3))"""
    u = math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)
    return 2 / (1 + torch.exp(-2 * u)) - 1


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + _tanh_of(z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return torch.where(z > 0, 1.0, 0.0)
    if act == "silu":
        sg = 1 / (1 + torch.exp(-z))
        return sg * (1 + z * (1 - sg))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    t = _tanh_of(z)
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)


def _segments(s):
    """Rows, matrix and bias of each expert, one after the other: experts differ in rows."""
    at = 0
    for e, rows in enumerate(s.rows):
        yield slice(at, at + rows), (e if s.offsets is not None else ...)
        at += rows


def _product_fwd(s):
    R, N = sum(s.rows), s.case["N"]
    z = torch.empty((R, N), dtype=torch.float32, device="cuda")
    for part, e in _segments(s):
        if part.stop > part.start:
            z[part] = s.x[part].float() @ s.w[e].float()
            if s.bias is not None:
                z[part] += s.bias[e].float()
    out = {} if s.z is None else {"z": z.to(s.z.dtype)}
    y = _act(z, s.case["act"])
    if s.residual is not None:
        y = y + s.residual.float()
    out["y"] = y.to(s.y.dtype)
    return out


def _product_bwd(s):
    R, case = sum(s.rows), s.case
    dz = s.dy[:R].float()
    if case["act"] != "none":
        dz = dz * _act_slope(s.z[:R].float(), case["act"])
    dx = torch.empty((R, case["K"]), dtype=s.dx.dtype, device="cuda")
    dw, db = torch.empty_like(s.dw), None if s.db is None else torch.empty_like(s.db)
    for part, e in _segments(s):
        dx[part] = (dz[part] @ s.w[e].float().t()).to(dx.dtype)
        dw[e] = (s.x[part].float().t() @ dz[part]).to(dw.dtype)
        if db is not None:
            db[e] = dz[part].sum(dim=0).to(db.dtype)
    return {"dx": dx, "dw": dw} if db is None else {"dx": dx, "dw": dw, "db": db}


_PLAIN = {"norm_fwd": _norm_fwd, "norm_bwd": _norm_bwd, "product_fwd": _product_fwd, "product_bwd": _product_bwd}


# --------------------------------------------------------------------------------------------------------- a pass
def run(s):
    case = s.case
    if not own:
        return _PLAIN[case["op"]](s)
    from paper_2605_11005_amd import binding as B
    if case["op"] == "norm_fwd":
        B.moe_layer_norm_fwd(s.y, s.h, s.w, s.b, EPS, s.h_out, s.n, s.mean, s.rstd)
        out = {"n": s.n, "mean": s.mean, "rstd": s.rstd, "h_out": s.h_out}
    elif case["op"] == "norm_bwd":
        B.moe_layer_norm_bwd(s.h_out, s.w, s.mean, s.rstd, s.dh_out, s.dn, s.dh, s.dy, s.dw, s.db, False, s.ws)
        out = {"dh": s.dh, "dy": s.dy, "dw": s.dw, "db": s.db}
    elif case["op"] == "product_fwd":
        R = sum(s.rows)
        B.moe_linear_fwd(s.x, s.offsets, s.w, s.bias, B.ACTIVATIONS[case["act"]], s.residual, s.z, s.y, s.ws)
        out = {"y": s.y[:R], "z": None if s.z is None else s.z[:R]}
    else:
        B.moe_linear_bwd(s.x, s.z, s.dy, s.offsets, s.w, B.ACTIVATIONS[case["act"]], s.dx, s.dw, s.db, False, s.ws)
        out = {"dx": s.dx[:sum(s.rows)], "dw": s.dw, "db": s.db}
    return {name: t for name, t in out.items() if t is not None}


def _expected_rows(case):
    """Expected rows of each local expert, popularity taken as proportional to rank^-zipf and no expert above T rows: their sum, and how
    many have any."""
    if not case["experts"]:
        return case["T"], 1
    p = [r ** -case["zipf"] for r in range(1, case["E"] + 1)]
    rows = [min(1.0, case["k"] * v / sum(p)) * case["T"] for v in p]
    share = case["experts"] / case["E"]
    return sum(rows) * share, sum(1 - math.exp(-r) for r in rows) * share


def work(case):
    """Inputs read once, outputs written once; of the forward's matrices those of experts that have rows."""
    size = {"bf16": 2, "f32": 4}
    b = size[case["dtype"]]
    if case["op"] in ("norm_fwd", "norm_bwd"):
        r, elements = size[case["residual"]], case["T"] * case["d"]
        if case["op"] == "norm_fwd":        # h and y -> h' and n
            return {"bytes": (r + b + ((b + r) if case["add"] else 0)) * elements + 8 * case["T"], "flops": 9 * elements}
        # h', dn and dh' -> dh (and dy)
        return {"bytes": (2 * r + b + (r if case["through"] else 0) + (b if case["add"] and r != b else 0)) * elements + 8 * case["T"],
                "flops": 14 * elements}
    R, active = _expected_rows(case)
    K, N, all_experts = case["K"], case["N"], max(1, case["experts"])
    if case["op"] == "product_fwd":
        outs = 1 + (1 if case["residual"] else 0) + (1 if case["train"] and case["act"] != "none" else 0)
        return {"bytes": b * (R * K + active * K * N + outs * R * N), "flops": 2 * R * K * N}
    ins = 2 if case["act"] != "none" else 1
    return {"bytes": b * (2 * R * K + ins * R * N + (active + all_experts) * K * N), "flops": 4 * R * K * N}


# --------------------------------------------------------------------------------------------------------- in 64 bits
def _exact_norm(s, case):
    def normed(h, w, b):
        c = h - h.sum(dim=1, keepdim=True) / case["d"]
        return c / (c.pow(2).sum(dim=1, keepdim=True) / case["d"] + EPS).sqrt() * w + b

    w, b = s.w.double(), s.b.double()
    if case["op"] == "norm_fwd":
        h = s.h.double()
        if s.y is not None:
            h = h + s.y.double()
        var, mean = torch.var_mean(h, dim=1, correction=0)
        out = {"n": normed(h, w, b), "mean": mean, "rstd": (var + EPS) ** -0.5}
        if s.y is not None:
            out["h_out"] = h
        return out
    # (mean and 1/deviation are inputs of the gradient: they are those of the sum before its rounding)
    h, dn = s.h_out.double(), s.dn.double()
    xh = (h - s.mean.double().unsqueeze(1)) * s.rstd.double().unsqueeze(1)
    t = w * dn
    dh = s.rstd.double().unsqueeze(1) * (t - (t.sum(dim=1, keepdim=True) + xh * (t * xh).sum(dim=1, keepdim=True)) / case["d"])
    if s.dh_out is not None:
        dh = dh + s.dh_out.double()
    out = {"dh": dh, "dw": (dn * xh).sum(dim=0), "db": dn.sum(dim=0)}
    if s.dy is not None:
        out["dy"] = dh
    return out


def _exact_act(z, act):
    if act == "none":
        return z
    if act == "gelu":
        return z * (0.5 * torch.special.erfc(-z / math.sqrt(2)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z.pow(3))))
    return torch.relu(z) if act == "relu" else z * torch.sigmoid(z)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm_fwd", "norm_bwd"):
        return _exact_norm(s, case)
    R, K, N, grouped = sum(s.rows), case["K"], case["N"], case["experts"] > 0
    f64 = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    matrices, first = max(1, case["experts"]), 0
    w, bias = s.w.view(matrices, K, N), None if s.bias is None else s.bias.view(matrices, N)
    if case["op"] == "product_fwd":
        out = {"y": f64(R, N)}
        if s.z is not None:
            out["z"] = f64(R, N)
        for e, rows in enumerate(s.rows):
            at = slice(first, first + rows)
            z = torch.mm(s.x[at].double(), w[e].double())
            z = z if bias is None else z + bias[e].double()
            if s.z is not None:
                out["z"][at] = z
            out["y"][at] = _exact_act(z, case["act"]) + (0 if s.residual is None else s.residual[at].double())
            first += rows
        return out
    dz = s.dy[:R].double()
    if case["act"] != "none":
        z = s.z[:R].double().requires_grad_()
        dz, = torch.autograd.grad(_exact_act(z, case["act"]), z, dz)
    dx, dw, db = f64(R, K), f64(matrices, K, N), f64(matrices, N)
    for e, rows in enumerate(s.rows):
        at = slice(first, first + rows)
        dx[at] = torch.mm(w[e].double(), dz[at].t()).t()
        dw[e] = torch.mm(dz[at].t(), s.x[at].double()).t()
        db[e] = dz[at].sum(dim=0)
        first += rows
    out = {"dx": dx, "dw": dw if grouped else dw[0]}
    if s.db is not None:
        out["db"] = db if grouped else db[0]
    return out
