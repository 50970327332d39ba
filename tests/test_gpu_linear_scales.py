"""Products of 8-bit operands whose scales' own product leaves fp32's range while the result does not."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,n_out", [(3, 64), (100, 192), (8003, 2112)])         # few tokens, with four and with more warps; CTA pairs
@pytest.mark.parametrize("residual", [False, True])
def test_scales_at_the_ends_of_the_range(T, n_out, residual):
    from paper_2605_06665_b200 import binding as B
    from paper_2605_06665_b200 import build as builder
    builder.build()
    ctx, n_in = B.Context(B.make_config(64, 64, 1, 1, 1, 8192, B.BF16, 1e-6, 1.0)), 4096
    e4m3 = torch.float8_e4m3fn
    x, W = torch.full((T, n_in), 448.0, device="cuda").to(e4m3), torch.full((n_out, n_in), 448.0, device="cuda").to(e4m3)
    x[1] = 0                                                 # a row of zeros
    xs, ws = torch.full((T,), 2.0 ** -80, device="cuda"), torch.full((n_out,), 2.0 ** -72, device="cuda")
    ws[1::2] = 2.0 ** 100                                    # every other feature: 2^-152 and 2^20 to the usual token, 2^28 and 2^200 to two
    xs[1:3] = 2.0 ** 100
    x[2] = 0
    x[2, 7] = 2.0 ** -9                                      # e4m3's smallest number: one term, 2^-9 x 448 x 2^200 beside 2^28
    res = torch.ones(T, n_out, dtype=torch.bfloat16, device="cuda") if residual else None
    pre, y = (torch.empty(T, n_out, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.linear_scaled(x, xs, T, n_in, W, ws, n_out, None, B.ACTIVATIONS["relu"], res, pre, y)
    # exact sums (448 x 448 x 4096 = 49 x 2^24: powers of two and 49), so that only the last rounding is left
    want = (x.double().sum(1) * 448.0)[:, None] * xs.double()[:, None] * ws.double()
    want = torch.where(want > torch.finfo(torch.bfloat16).max, torch.inf, want)
    assert torch.isinf(want[2, 1::2]).all() and torch.isfinite(want[:2]).all() and (want[0, ::2] > 2.0 ** -126).all()
    for got, w in ((pre, want), (y, want + (1.0 if residual else 0.0))):
        fine = torch.isfinite(w)
        assert torch.equal(torch.isfinite(got), fine) and not torch.isnan(got).any()
        # half a step of bf16 (2^-8), and 2^-23 for the sums of the tensor core
        assert ((got[fine].double() - w[fine]).abs() <= (2.0 ** -8 + 2.0 ** -23) * w[fine].abs()).all()
    ctx.check_status()
    ctx.close()
