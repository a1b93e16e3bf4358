"""Layer norms of more elements than 32 bits count, against float64."""
import pytest
import torch

from paper_2605_11005_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dt,rt,T,d", [(BF16, F32, 270_000, 8192), (BF16, BF16, 140_000, 16384), (F32, F32, 36_000_000, 64)])
def test_more_elements_than_32_bits_count(dt, rt, T, d):
    """Root mean squares of rows at the beginning, beside element 2^31 and at the end, off by a rounding, at most 2^-8 (fp32: a few roundings, 2^-21); column
    sums of 36 million rows in fp32 by 2048 blocks or more, one row after the other: 2^14.2 roundings towards one side at worst, 2^-9.8, and their own."""
    print(f"case layer norm {T} {d} {dt} {rt}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(d)
    new = lambda t: torch.empty(T, d, dtype=t, device="cuda").normal_(generator=g)  # noqa: E731
    h, y, dn = new(rt), new(dt), new(dt)
    w, b = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dt), torch.randn(d, generator=g, device="cuda").to(dt)
    n, mean, rstd = torch.empty_like(y), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    old = h.clone()
    B.moe_layer_norm_fwd(y, h, w, b, 1e-5, h, n, mean, rstd)
    dw, db, dy = torch.empty_like(w), torch.empty_like(b), torch.empty_like(y)
    ws = torch.empty(B.moe_workspace_bytes(B.WS_LAYER_NORM, 0, T, 0, d, 0, 0, 0), dtype=torch.uint8, device="cuda")
    middle = (1 << 31) // d
    at = torch.cat([torch.arange(a, e, device="cuda") for a, e in ((0, 40), (middle - 40, middle + 40), (T - 40, T))])
    half = 2.0 ** -8 if dt == BF16 else 2.0 ** -21
    near = lambda got, ref, bound, name: (got.double() - ref).norm() <= bound * ref.norm() or pytest.fail(f"{name} {float((got.double() - ref).norm() / ref.norm())}")  # noqa: E731
    total = old[at].double() + y[at].double()
    near(h[at], total, 2.0 ** -8 if rt == BF16 else 2.0 ** -21, "h")
    m, v = total.mean(1, keepdim=True), total.var(1, correction=0, keepdim=True)
    near(n[at], (total - m) * (v + 1e-5) ** -0.5 * w.double() + b.double(), half, "n")
    near(mean[at], m[:, 0], 2.0 ** -18, "mean")
    near(rstd[at], (v[:, 0] + 1e-5) ** -0.5, 2.0 ** -18, "rstd")
    dh = torch.empty_like(h)
    B.moe_layer_norm_bwd(h, w, mean, rstd, old, dn, dh, dy, dw, db, False, ws)
    normed = lambda s: (h[s].double() - mean[s].double()[:, None]) * rstd[s].double()[:, None]  # noqa: E731
    xh, t = normed(at), dn[at].double() * w.double()
    ref = old[at].double() + rstd[at].double()[:, None] * (t - t.mean(1, keepdim=True) - xh * (t * xh).mean(1, keepdim=True))
    near(dh[at], ref, 2.0 ** -8 if rt == BF16 else 2.0 ** -20, "dh")
    near(dy[at], ref, 2.0 ** -8 if dt == BF16 else 2.0 ** -20, "dy")
    pieces = [slice(a, a + 65536) for a in range(0, T, 65536)]
    near(dw, sum((dn[s].double() * normed(s)).sum(0) for s in pieces), half + 2.0 ** -9, "dw")
    near(db, sum(dn[s].double().sum(0) for s in pieces), half + 2.0 ** -9, "db")
