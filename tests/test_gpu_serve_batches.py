"""A block that serves fewer tokens than its buffers are for: the results of buffers of that size."""
import pytest
import torch

from paper_2605_11005_amd import binding as B
from paper_2605_11005_amd import block as K
from paper_2605_11005_amd import workloads as W

pytestmark = pytest.mark.gpu


def weights(wl):
    g = torch.Generator().manual_seed(3)
    new = lambda *shape, std: (std * torch.randn(shape, generator=g)).to(torch.bfloat16).cuda()  # noqa: E731
    return dict(wr=new(wl.d, wl.E, std=2 * wl.d ** -0.5), w1=new(wl.e_cnt, wl.d, wl.f, std=wl.d ** -0.5), w3=new(wl.e_cnt, wl.d, wl.f, std=wl.d ** -0.5),
                w2=new(wl.e_cnt, wl.f, wl.d, std=wl.f ** -0.5), w_post=1 + new(wl.d, std=0.1), w_pre=1 + new(wl.d, std=0.1))


@pytest.mark.parametrize("residual", [None, torch.float32])
def test_a_batch_that_shrinks(residual):
    wl = W.QWEN.scaled(name="serve-shrinking", T=70, d=256, f=160, E=64, e_lo=16, e_cnt=32, k=4)
    w = K.serve_weights(weights(wl))
    buf = K.MoeServeBuffers(wl, wl.T * wl.k, residual)
    g = torch.Generator(device="cuda").manual_seed(1)
    h, x = torch.empty_like(buf.h).normal_(generator=g), torch.empty_like(buf.x)
    for T in (70, 69, 17, 3, 1, 0, 70):
        print(f"case {T} tokens", flush=True)
        B.moe_block_norm_fwd(None, None, None, False, h[:T], w["w_pre"], 1.0, 1.0, 1e-6, None, x[:T])
        buf.h.fill_(float("nan"))
        buf.x.fill_(float("nan"))
        K.run_block_serve(wl, w, h[:T], x[:T], buf)
        exactly = wl.scaled(name=f"serve-{T}", T=T)
        own = K.MoeServeBuffers(exactly, max(T * wl.k, 1), residual)
        K.run_block_serve(exactly, w, h[:T], x[:T], own)
        assert torch.equal(buf.h[:T], own.h) and torch.equal(buf.x[:T], own.x)
        assert torch.isfinite(own.h).all() and torch.isnan(buf.h[T:]).all() and torch.isnan(buf.x[T:]).all()


def test_more_tokens_than_the_buffers_are_refused():
    wl = W.QWEN.scaled(name="serve-small", T=4, d=256, f=160, E=64, e_lo=0, e_cnt=64, k=4)
    w = K.serve_weights(weights(wl))
    buf = K.MoeServeBuffers(wl, wl.T * wl.k)
    h, x = (torch.zeros(5, wl.d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    with pytest.raises(B.MoeError):
        K.run_block_serve(wl, w, h, x, buf)
