"""The block of two-matrix experts serving fewer tokens than its buffers are for: the results of buffers of that size."""
import pytest
import torch

from paper_2605_11005_amd import binding as B
from paper_2605_11005_amd import ffn_block as F
from paper_2605_11005_amd import workloads as W

pytestmark = pytest.mark.gpu
SHARED = 200


def weights(wl, dt):
    g = torch.Generator().manual_seed(3)
    new = lambda *shape, std: (std * torch.randn(shape, generator=g)).to(dt).cuda()  # noqa: E731
    d, f, e = wl.d, wl.f, wl.e_cnt
    return dict(wr=new(d, wl.E, std=2 * d ** -0.5), w1=new(e, d, f, std=d ** -0.5), b1=new(e, f, std=0.1), w2=new(e, f, d, std=f ** -0.5), b2=new(e, d, std=0.1),
                ws1=new(d, SHARED, std=d ** -0.5), bs1=new(SHARED, std=0.1), ws2=new(SHARED, d, std=SHARED ** -0.5), bs2=new(d, std=0.1),
                w=1 + new(d, std=0.1), b=new(d, std=0.1))


@pytest.mark.parametrize("dtype,residual", [("bf16", None), ("bf16", torch.float32), ("f32", None)])
def test_a_batch_that_shrinks(dtype, residual):
    wl = W.QWEN.scaled(name="ffn-shrinking", T=150, d=136, f=160, E=32, e_lo=8, e_cnt=16, k=4, dtype=dtype)
    dt, cap = torch.bfloat16 if dtype == "bf16" else torch.float32, 150 * 4
    w = weights(wl, dt)
    buf = F.FfnBlockBuffers(wl, cap, SHARED, residual=residual, grads=False)
    g = torch.Generator(device="cuda").manual_seed(1)
    h, x = torch.empty_like(buf.h).normal_(generator=g), torch.empty_like(buf.x)
    for T in (150, 149, 33, 17, 3, 1, 0, 150):
        print(f"case {T} tokens", flush=True)
        B.moe_layer_norm_fwd(None, h[:T], w["w"], w["b"], 1e-5, None, x[:T])
        buf.h.fill_(float("nan"))
        buf.x.fill_(float("nan"))
        F.run_ffn_forward(wl, w, h[:T], x[:T], buf)
        # (the rows' capacity stays: the order of an expert's sums may go by it)
        exactly = wl.scaled(name=f"ffn-{T}", T=T)
        own = F.FfnBlockBuffers(exactly, cap, SHARED, residual=residual, grads=False)
        F.run_ffn_forward(exactly, w, h[:T], x[:T], own)
        assert torch.equal(buf.h[:T], own.h) and torch.equal(buf.x[:T], own.x)
        assert torch.isfinite(own.h).all() and torch.isfinite(own.x).all() and torch.isnan(buf.h[T:]).all() and torch.isnan(buf.x[T:]).all()


def test_a_shrunken_batch_captured_and_replayed():
    """A graph for each of two batch sizes over the same buffers, replayed in turn between eager passes."""
    wl = W.QWEN.scaled(name="ffn-graphs", T=40, d=136, f=160, E=32, e_lo=0, e_cnt=32, k=4)
    w = weights(wl, torch.bfloat16)
    buf, eager = F.FfnBlockBuffers(wl, 160, SHARED, grads=False), F.FfnBlockBuffers(wl, 160, SHARED, grads=False)
    h, x = (torch.randn(40, wl.d, device="cuda").to(torch.bfloat16) for _ in range(2))
    s = torch.cuda.Stream()
    F.run_ffn_forward(wl, w, h, x, eager)
    s.wait_stream(torch.cuda.current_stream())
    graphs = {}
    for T in (40, 5):
        graphs[T] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[T], stream=s):
            F.run_ffn_forward(wl, w, h[:T], x[:T], buf)
    for i in range(3):
        for T, graph in graphs.items():
            x.neg_()
            F.run_ffn_forward(wl, w, h[:T], x[:T], eager)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(buf.h[:T], eager.h[:T]) and torch.equal(buf.x[:T], eager.x[:T]), (i, T)


def test_more_tokens_than_the_buffers_and_fewer_in_training_are_refused():
    wl = W.QWEN.scaled(name="ffn-small", T=4, d=136, f=160, E=32, e_lo=0, e_cnt=32, k=4)
    w = weights(wl, torch.bfloat16)
    for T, grads in ((5, False), (5, True), (3, True)):
        h, x = (torch.zeros(T, wl.d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        with pytest.raises(B.MoeError):
            F.run_ffn_forward(wl, w, h, x, F.FfnBlockBuffers(wl, 16, SHARED, grads=grads))
