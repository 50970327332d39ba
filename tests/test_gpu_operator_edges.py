"""Sizes at the borders between the operators' forms that no other test has: the norm's backward pass on clusters at each width, fp32
products of many tokens off 16 bytes."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def context(name, tokens=8192):
    from paper_2605_06665_b200 import binding as B
    from paper_2605_06665_b200 import build as builder
    builder.build()
    dt = torch.bfloat16 if name == "bf16" else torch.float32
    return B, dt, B.Context(B.make_config(64, 64, 1, 1, 1, tokens, B.BF16 if name == "bf16" else B.FP32, 1e-6, 1.0))


def normal(shape, dt, seed, std=1.0):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dt).cuda()


@pytest.mark.parametrize("name", ["bf16", "fp32"])
@pytest.mark.parametrize("width", [1, 8, 257, 514, 515, 1026, 2049, 2050, 4096, 4098, 8196, 8200, 9287, 9288, 13936, 16384])
@pytest.mark.parametrize("T", [5, 8, 14, 33, 100])
def test_norm_backward_on_clusters(name, width, T):
    """With and without dr, in place over it, aligned and one element off."""
    B, dt, ctx = context(name)
    half, fp32 = torch.finfo(dt).eps / 2, 300 * 2.0 ** -24
    dh, r, dr, w = normal((T, width), dt, 1, 0.1), normal((T, width), dt, 2), normal((T, width), dt, 3, 0.1), 1 + normal((width,), torch.float32, 4, 0.2)
    rstd = torch.rsqrt(r.float().square().mean(1) + 1e-6)
    d, x, W, n = dh.double(), r.double() * rstd.double()[:, None], w.double(), rstd.double()[:, None]
    base = n * (W * d - x * (W * d * x).mean(1, keepdim=True))
    size = n * ((W * d).abs() + x.abs() * (W * d * x).abs().mean(1, keepdim=True))
    off = lambda t: torch.cat([t.reshape(-1)[:1], t.reshape(-1)])[1:].view(t.shape)
    for with_dr, shift in ((False, False), (True, False), (True, True)):
        a = [off(t) if shift else t.clone() for t in (dh, r, dr)]
        dx, dw = a[2] if with_dr else torch.empty_like(a[0]), torch.full((width,), 2.0, device="cuda")
        ctx.rmsnorm_bwd(a[0], a[1], T, width, w, rstd, a[2] if with_dr else None, dx, dw)
        want, mag = (base + dr.double(), size + dr.double().abs()) if with_dr else (base, size)
        assert ((dx.double() - want).abs() <= half * want.abs() + fp32 * mag).all()
        terms = d * x
        assert ((dw.double() - 2 - terms.sum(0)).abs() <= (T + 8) * 2.0 ** -24 * (terms.abs().sum(0) + 2)).all()
    ctx.check_status()
    ctx.close()


def test_fp32_products_of_many_tokens_off_sixteen_bytes():
    B, dt, ctx = context("fp32")
    T, n_in, n_out = 4003, 256, 1088
    off = lambda t: torch.cat([t.reshape(-1)[:1], t.reshape(-1)])[1:].view(t.shape)
    x, W, bias, res = normal((T, n_in), dt, 5), normal((n_out, n_in), dt, 6, 0.1), normal((n_out,), dt, 7), normal((T, n_out), dt, 8)
    dy = normal((T, n_out), dt, 9)
    out = []
    for move in (lambda t: t, off):
        y, pre, dx, dW, db, dp = (move(torch.zeros(s, device="cuda")) for s in ((T, n_out), (T, n_out), (T, n_in), (n_out, n_in), (n_out,), (T, n_out)))
        ctx.linear(move(x), T, n_in, move(W), n_out, move(bias), B.ACTIVATIONS["silu"], move(res), pre, y)
        ctx.linear_bwd(move(dy), T, n_out, pre, B.ACTIVATIONS["silu"], move(x), n_in, move(W), dp, None, dx, dW, db)
        out.append((y, pre, dx, dW, db, dp))
    for a, b in zip(*out[:2]):                               # the same products in the same order; the sums of dbias in another
        assert torch.equal(a, b) or (a.shape == (n_out,) and (a - b).abs().max() <= 2.0 ** -24 * 100 * out[0][5].abs().sum(0).max())
    p = x.double() @ W.double().T + bias.double()
    terms = x.double().abs() @ W.double().abs().T + bias.double().abs()
    assert ((out[1][1].double() - p).abs() <= 2.0 ** -24 * ((n_in + 16) * terms + p.abs())).all()
    ctx.check_status()
    ctx.close()
