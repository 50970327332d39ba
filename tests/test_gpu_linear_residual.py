"""Backward of y = x + act(x W^T + b), where dy is the gradient, the residual's part of dx and the memory for dp at once."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [3, 300, 2500])
@pytest.mark.parametrize("name", ["bf16", "fp32"])
def test_dp_over_dy_over_the_residual(name, T):
    from paper_2605_06665_b200 import binding as B
    from paper_2605_06665_b200 import build as builder
    builder.build()
    dt, n, act = (torch.bfloat16 if name == "bf16" else torch.float32), 256, B.ACTIVATIONS["silu"]
    ctx = B.Context(B.make_config(64, 64, 1, 1, 1, 4096, B.BF16 if name == "bf16" else B.FP32, 1e-6, 1.0))
    g = torch.Generator(device="cpu").manual_seed(T)
    normal = lambda *s: torch.randn(s, generator=g).to(dt).cuda()
    x, W, pre, dy = normal(T, n), normal(n, n) * n ** -0.5, normal(T, n), normal(T, n)

    def run(dy, dp, res, dx, frozen=False):
        dW, db = (None, None) if frozen else (torch.empty(n, n, device="cuda"), torch.empty(n, device="cuda"))
        ctx.linear_bwd(dy, T, n, pre, act, x, n, W, dp, res, dx, dW, db, B.WGRAD_OVERWRITE)
        return [dx] if frozen else [dx, dW, db]

    for frozen in (False, True):
        want = run(dy, torch.empty_like(dy), dy.clone(), torch.empty_like(x), frozen)
        for shared in (dy.clone(), pre):                     # dp on dy and the residual; on pre, which is the residual here
            if shared is pre:
                want = run(dy, torch.empty_like(dy), pre.clone(), torch.empty_like(x), frozen)
                pre0 = pre.clone()
                got = run(dy, pre, pre, torch.empty_like(x), frozen)
                pre.copy_(pre0)
            else:
                got = run(shared, shared, shared, torch.empty_like(x), frozen)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    ctx.check_status()
    ctx.close()
