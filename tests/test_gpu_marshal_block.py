"""The native marshalling (csrc/marshal.cpp) of the block norms and of the 4-bit calls: the calls that binding.py's own checks and ctypes
would make, on torch's current stream; every other call is left to them."""
import pytest
import torch

from paper_2605_11005_amd import binding as B

pytestmark = pytest.mark.gpu


class NotTaken:
    def __getattr__(self, name):
        return lambda *args: -1


class Taken:
    """The native marshalling; counts the calls it made."""

    def __init__(self, native):
        self.native, self.calls = native, 0

    def __getattr__(self, name):
        def call(*args):
            rc = getattr(self.native, name)(*args)
            self.calls += rc >= 0
            return rc
        return call


def norm_calls(dt, rt):
    """Every output of the norms' calls: whole, without the optional operands, and the norm in front of a first block."""
    T, d = 21, 192
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *shape, dtype=dt: torch.randn(shape, generator=g, device="cuda").to(dtype)
    y, h, w_post, w_pre, gate = new(T, d), new(T, d, dtype=rt), new(d), new(d), new(T, dtype=torch.float32)
    dn, dh_out = new(T, d), new(T, d, dtype=rt)
    ws = torch.empty(B.moe_workspace_bytes(B.WS_BLOCK_NORM, 0, T, 0, d, 0, 0, 0), dtype=torch.uint8, device="cuda")
    out = []
    for whole in (True, False):
        h_out, n, dh, dy = torch.zeros_like(h), torch.zeros_like(y), torch.zeros_like(h), torch.zeros_like(y)
        r_post, r_pre, dgate = (torch.zeros(T, device="cuda") for _ in range(3))
        dw_post, dw_pre = torch.ones_like(w_post), torch.ones_like(w_pre)
        if whole:
            B.moe_block_norm_fwd(y, gate, w_post, True, h, w_pre, 0.5, 2.0, 1e-5, h_out, n, r_post, r_pre)
            B.moe_block_norm_bwd(y, gate, w_post, True, h_out, w_pre, r_post, r_pre, dh_out, dn, 0.5, 2.0, dh, dy, dgate, dw_post, dw_pre, True, ws)
        else:
            B.moe_block_norm_fwd(None, None, None, False, h, w_pre, 1.0, 1.0, 1e-5, None, n, None, r_pre)
            B.moe_block_norm_bwd(y, None, None, False, None, None, None, None, dh_out, None, 0.5, 2.0, dh, dy, None, None, None, False, ws)
        out += [h_out, n, dh, dy, r_post, r_pre, dgate, dw_post, dw_pre]
    return out, 4


def mx4_calls():
    """The experts' products over quantised weights, and a tensor there and back."""
    d, f, rows = 544, 96, [3, 0, 40]
    g = torch.Generator(device="cuda").manual_seed(4)
    new = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)

    def quantised(x, along_rows, n, K):
        data, scales = (torch.empty(x.shape[:-2] + s, dtype=torch.uint8, device="cuda") for s in B.mx4_shapes(n, K))
        B.moe_mx4_quantize(x, along_rows, data, scales)
        return data, scales

    E = len(rows)
    w1, w3, w2 = (quantised(new(E, K, n), True, n, K) for K, n in ((d, f), (d, f), (f, d)))
    xp = new(sum(rows), d)
    back = torch.empty_like(xp)
    q = quantised(xp, False, *xp.shape)
    B.moe_mx4_dequantize(*q, back)
    off = torch.tensor([0, 3, 3, 43], dtype=torch.int32, device="cuda")
    ws = torch.empty(B.moe_workspace_bytes(B.WS_MX4_EXPERT_FWD, B.MOE_BF16, 0, 0, d, f, E, sum(rows)), dtype=torch.uint8, device="cuda")
    o = torch.empty_like(xp)
    B.moe_mx4_expert_fwd(xp, off, *w1, *w3, *w2, o, ws)
    return [*w1, *w3, *w2, *q, back, o], 6


CALLS = {"norm-bf16": lambda: norm_calls(torch.bfloat16, torch.bfloat16), "norm-mixed": lambda: norm_calls(torch.bfloat16, torch.float32),
         "norm-f32": lambda: norm_calls(torch.float32, torch.float32), "mx4": mx4_calls}


@pytest.mark.parametrize("name", list(CALLS))
def test_native_calls_equal_those_of_ctypes(name, monkeypatch):
    print(f"case marshal-{name}", flush=True)
    native, results = Taken(B._marshal()), []
    for marshal in (native, NotTaken()):
        monkeypatch.setattr(B, "_MARSHAL", marshal)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        torch.cuda._sleep(int(1e8))              # a call on the default stream would not be done when its results are read
        with torch.cuda.stream(side):
            out, calls = CALLS[name]()
            results.append([t.clone() for t in out])
        side.synchronize()
        torch.cuda.synchronize()
    assert native.calls == calls
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("call,fault", [(c, f) for c in ("norm_fwd", "norm_bwd", "quantize", "dequantize", "expert_fwd")
                                        for f in ("dtype", "shape", "strides", "host", "alike", "code")])
def test_refused_calls_are_refused_alike(call, fault, monkeypatch):
    T, d, f = 6, 64, 32
    new = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, device="cuda", dtype=dtype)
    bad = {"dtype": lambda t: t.to(torch.float64), "shape": lambda t: t[..., :-1].contiguous(), "host": lambda t: t.cpu(),
           "strides": lambda t: torch.zeros((*t.shape[:-1], 2 * t.shape[-1]), device="cuda", dtype=t.dtype)[..., ::2], "alike": lambda t: 1.5,
           "code": lambda t: t}[fault]
    code = fault == "code"
    h, y, w, ws = new(T, d), new(T, d), new(d), new(1 << 16, dtype=torch.uint8)
    u8 = lambda n, K, *batch: [new(*batch, *s, dtype=torch.uint8) for s in B.mx4_shapes(n, K)]
    if call == "norm_fwd":
        run = lambda: B.moe_block_norm_fwd(bad(y), None, w, True, h, w, 1.0, 1.0, -1.0 if code else 1e-5, new(T, d), new(T, d))
    elif call == "norm_bwd":
        r = new(T, dtype=torch.float32)
        run = lambda: B.moe_block_norm_bwd(y, None, w, True, h, w, r, r, None, bad(y), 1.0, 1.0, new(T, d), new(T, d), None, new(d), new(d), False,
                                           ws[:256] if code else ws)
    elif call == "quantize":
        q = u8(T, d)
        run = lambda: B.moe_mx4_quantize(new(T, 48) if code else new(T, d), False, bad(q[0]), q[1])
    elif call == "dequantize":
        q = u8(T, d)
        run = lambda: B.moe_mx4_dequantize(q[0], bad(q[1]), new(T, 48) if code else new(T, d))
    else:
        w1, w3, w2 = u8(f, d, 2), u8(f, d, 2), u8(d, f, 2)
        off = new(3, dtype=torch.int32)
        run = lambda: B.moe_mx4_expert_fwd(bad(y), off, *w1, *w3, *w2, new(T, d), ws[:256] if code else ws)
    errors, native = [], B._marshal()
    for marshal in (native, NotTaken()):
        monkeypatch.setattr(B, "_MARSHAL", marshal)
        with pytest.raises(Exception) as e:
            run()
        errors.append((type(e.value), str(e.value)))
    assert errors[0] == errors[1]
