"""The backward call's gradients, whole arrays, against central differences of the activation in float64 at the value before it that
the forward call stored.  Beside that value only what the backward call itself rounds is left: dp to the type of the operands,
the products' sums, and the results."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

MATH = 2.0 ** -20                                            # the activations' slopes through the special-function unit


def value(p, act):
    if act == "relu":
        return p.clamp(min=0)
    if act == "silu":
        return p / (1 + torch.exp(-p))
    if act == "gelu":
        return 0.5 * p * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (p + 0.044715 * p ** 3)))
    return p


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("T", [6, 130, 900])
@pytest.mark.parametrize("name", ["bf16", "fp32"])
def test_gradients_by_differences_of_the_activation(name, act, T):
    from paper_2605_06665_b200 import binding as B
    from paper_2605_06665_b200 import build as builder
    builder.build()
    bf16, n_in, n_out = name == "bf16", 192, 128
    dt = torch.bfloat16 if bf16 else torch.float32
    half, ctx = torch.finfo(dt).eps / 2, B.Context(B.make_config(64, 64, 1, 1, 1, 1024, B.BF16 if bf16 else B.FP32, 1e-6, 1.0))
    g = torch.Generator(device="cpu").manual_seed(T)
    normal = lambda *s, std=1.0, dt=dt: (torch.randn(s, generator=g) * std).to(dt).cuda()
    x, W, bias, dy = normal(T, n_in), normal(n_out, n_in, std=2 * n_in ** -0.5), normal(n_out, dt=torch.float32), normal(T, n_out)
    y, pre, dp = (torch.empty(T, n_out, dtype=dt, device="cuda") for _ in range(3))
    ctx.linear(x, T, n_in, W, n_out, bias, B.ACTIVATIONS[act], None, pre, y)
    dx, dW, db = torch.empty_like(x), torch.empty(n_out, n_in, device="cuda"), torch.empty(n_out, device="cuda")
    ctx.linear_bwd(dy, T, n_out, pre, B.ACTIVATIONS[act], x, n_in, W, dp, None, dx, dW, db, B.WGRAD_OVERWRITE)

    p, h, far = pre.double(), 1e-5, 1e-9                     # (of differences: h^2 / 6 of a third derivative below 2, 2^-53 |p| / h)
    slope = (value(p + h, act) - value(p - h, act)) / (2 * h)
    if act == "relu":                                        # its kink: one side or the other, none at 0 itself
        slope = (p > 0).double()
    want = dy.double() * slope
    slack = dy.double().abs() * (1.2 * MATH + far if act != "relu" else 0.0)
    rounded = half if act != "relu" else 0.0
    assert ((dp.double() - want).abs() <= rounded * want.abs() * (1 + MATH) + slack).all()
    steps = (lambda K: 2 * (K / 16 + 16)) if bf16 else (lambda K: K + 16)
    for got, left, right, K in ((dx, want, W.double(), n_out), (dW, want.T, x.double(), T)):
        exact, terms = left @ right, left.abs() @ right.abs()
        last = half if got.dtype == dt else 2.0 ** -24
        more = slack @ W.double().abs() if got is dx else slack.T @ x.double().abs()
        # (the first T >= 769 is cut into segments of 768 tokens, added up in fp32)
        bound = last * 1.001 * exact.abs() + (rounded * (1 + MATH) + 2.0 ** -24 * (steps(K) + 64)) * terms + more
        assert ((got.double() - exact).abs() <= bound).all()
    assert ((db.double() - want.sum(0)).abs() <= 2.0 ** -24 * (T + 64) * want.abs().sum(0) + slack.sum(0) + MATH * want.abs().sum(0)).all()
    ctx.check_status()
    ctx.close()
