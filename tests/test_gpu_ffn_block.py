"""Two residual blocks of two-matrix experts with biases, dense experts and layer norms in a row, against torch's autograd in float64 with the same
selection of experts.  Tolerances are those of the expert layer's parity tests: the largest difference over the largest value of a tensor, 1e-5 in fp32 and
2e-2 in bf16, where a block rounds its activations half a dozen times by 2^-8 of the value at most."""
import numpy as np
import pytest
import torch

from paper_2605_11005_amd import binding as B
from paper_2605_11005_amd import workloads as W
from paper_2605_11005_amd.ffn_block import FfnBlockBuffers, run_ffn_backward, run_ffn_forward

pytestmark = pytest.mark.gpu
EPS = 1e-5
TOL = {"f32": 2e-5, "bf16": 3e-2}      # two blocks: up to twice a layer's
ACT = dict(relu=torch.relu, gelu=torch.nn.functional.gelu, silu=torch.nn.functional.silu,
           gelu_tanh=lambda z: torch.nn.functional.gelu(z, approximate="tanh"))


def weights(wl, shared_f, dt, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, scale=1.0: (scale * torch.randn(s, generator=g)).to(dt).cuda()  # noqa: E731
    d, f, e, E = wl.d, wl.f, wl.e_cnt, wl.E
    return dict(wr=r(d, E, scale=d ** -0.5), w1=r(e, d, f, scale=d ** -0.5), b1=r(e, f, scale=0.1), w2=r(e, f, d, scale=f ** -0.5), b2=r(e, d, scale=0.1),
                ws1=r(d, shared_f, scale=d ** -0.5), bs1=r(shared_f, scale=0.1), ws2=r(shared_f, d, scale=shared_f ** -0.5), bs2=r(d, scale=0.1),
                w=1 + r(d, scale=0.1), b=r(d, scale=0.1))


def reference(wl, w, h, x, topk, act):
    """One block in float64 with the experts topk [T,k] of each token."""
    logits = x @ w["wr"]
    gate = torch.softmax(torch.gather(logits, 1, topk), dim=1) if wl.gate_mode == B.GATE_SOFTMAX_RENORM else None
    if gate is None:
        s = torch.sigmoid(torch.gather(logits, 1, topk))
        gate = s / s.sum(dim=1, keepdim=True)
    y = act(x @ w["ws1"] + w["bs1"]) @ w["ws2"] + w["bs2"]
    for e in range(wl.e_cnt):
        t, slot = torch.nonzero(topk == wl.e_lo + e, as_tuple=True)
        if len(t):
            o = act(x[t] @ w["w1"][e] + w["b1"][e]) @ w["w2"][e] + w["b2"][e]
            y = y.index_add(0, t, gate[t, slot, None] * o)
    h = h + y
    return h, torch.nn.functional.layer_norm(h, (wl.d,), w["w"], w["b"], EPS)


def check(got, ref, tol, name):
    got, ref = got.double().cpu(), ref.detach().cpu()
    scale = ref.abs().max().item()
    assert torch.isfinite(got).all(), name
    assert (got - ref).abs().max().item() <= tol * scale, (name, (got - ref).abs().max().item() / scale)


@pytest.mark.parametrize("act", ("gelu", "silu"))
@pytest.mark.parametrize("dtype,residual", [("f32", None), ("bf16", None), ("bf16", torch.float32)])
@pytest.mark.parametrize("T", (1, 37, 700))
def test_two_blocks(T, dtype, residual, act):
    print(f"case ffn block {T} {dtype} {residual} {act}", flush=True)
    wl = W.QWEN.scaled(name="ffn", T=T, d=136, f=200, E=12, e_lo=3, e_cnt=6, k=3, dtype=dtype)
    dt, shared_f = (torch.float32 if dtype == "f32" else torch.bfloat16), 264
    g = torch.Generator().manual_seed(T)
    ws = [weights(wl, shared_f, dt, s) for s in (1, 2)]
    first = dict(w=ws[0]["w"].flip(0), b=ws[0]["b"].flip(0))
    h0 = torch.randn((T, wl.d), generator=g).to(residual or dt).cuda()
    x0, mean, rstd = torch.empty((T, wl.d), dtype=dt, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    bufs = [FfnBlockBuffers(wl, T * wl.k + 5, shared_f, act, residual) for _ in ws]
    dh_out = torch.randn((T, wl.d), generator=g).to(residual or dt).cuda()
    dn = torch.randn((T, wl.d), generator=g).to(dt).cuda()

    def step(accumulate=False):
        B.moe_layer_norm_fwd(None, h0, first["w"], first["b"], EPS, None, x0, mean, rstd)
        run_ffn_forward(wl, ws[0], h0, x0, bufs[0], EPS)
        run_ffn_forward(wl, ws[1], bufs[0].h, bufs[0].x, bufs[1], EPS)
        run_ffn_backward(wl, ws[1], bufs[0].x, bufs[1], dh_out, dn, accumulate)
        run_ffn_backward(wl, ws[0], x0, bufs[0], bufs[1].dh, bufs[1].dx, accumulate)

    step()
    tol = TOL[dtype]
    leaves = [{k: v.double().requires_grad_() for k, v in w.items()} for w in ws]
    rh = h0.double().requires_grad_()
    h, x = rh, torch.nn.functional.layer_norm(rh, (wl.d,), first["w"].double(), first["b"].double(), EPS)
    for w, buf in zip(leaves, bufs):
        h, x = reference(wl, w, h, x, buf.topk_idx.long(), ACT[act])
        check(buf.h, h, tol, "h")
        check(buf.x, x, tol, "x")
    ((h * dh_out.double()).sum() + (x * dn.double()).sum()).backward()
    for w, buf in zip(leaves, bufs):
        for name, got in buf.dw.items():
            check(got, w[name].grad, tol if T > 1 else 2 * tol, name)
    # of the stream in front of the first norm
    dh0 = torch.empty_like(h0)
    wsn = torch.empty(B.moe_workspace_bytes(B.WS_LAYER_NORM, 0, T, 0, wl.d, 0, 0, 0), dtype=torch.uint8, device="cuda")
    B.moe_layer_norm_bwd(h0, first["w"], mean, rstd, bufs[0].dh, bufs[0].dx, dh0, None, None, None, False, wsn)
    check(dh0, rh.grad, tol, "dh0")
    # a second micro-batch's gradients are added: the same again doubles them
    once = {k: v.clone() for k, v in bufs[1].dw.items()}
    step(accumulate=True)
    for name, got in bufs[1].dw.items():
        check(got, 2 * once[name].double(), 2.0 ** -7 if dtype == "bf16" else 1e-6, "twice " + name)


def test_serving_needs_no_gradients_buffers():
    wl = W.QWEN.scaled(name="ffn-serve", T=29, d=136, f=200, E=12, e_lo=0, e_cnt=12, k=3)
    w = weights(wl, 72, torch.bfloat16, 4)
    h, x = torch.randn((29, 136), device="cuda").to(torch.bfloat16), torch.randn((29, 136), device="cuda").to(torch.bfloat16)
    train, serve = FfnBlockBuffers(wl, 29 * 3, 72), FfnBlockBuffers(wl, 29 * 3, 72, grads=False)
    for buf in (train, serve):
        run_ffn_forward(wl, w, h, x, buf)
    assert torch.equal(train.h, serve.h) and torch.equal(train.x, serve.x)


def test_a_step_captured_and_replayed():
    """Forward and backward in one graph, replayed between eager steps over the same weights."""
    wl = W.QWEN.scaled(name="ffn-graph", T=130, d=136, f=200, E=12, e_lo=0, e_cnt=12, k=2)
    w = weights(wl, 72, torch.bfloat16, 5)
    h, x = torch.randn((130, 136), device="cuda").to(torch.bfloat16), torch.randn((130, 136), device="cuda").to(torch.bfloat16)
    dn = torch.randn_like(x)
    eager, captured = FfnBlockBuffers(wl, 260, 72), FfnBlockBuffers(wl, 260, 72)

    def step(buf):
        run_ffn_forward(wl, w, h, x, buf)
        run_ffn_backward(wl, w, x, buf, None, dn)

    step(eager)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(captured)
    for i in range(4):
        x.neg_()
        step(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager.x, captured.x) and torch.equal(eager.dx, captured.dx) and torch.equal(eager.dh, captured.dh)
        for name in eager.dw:
            assert torch.equal(eager.dw[name], captured.dw[name]), name
