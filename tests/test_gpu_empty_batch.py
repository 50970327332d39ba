"""Batches without tokens as PyTorch hands them over: x[:0] and empty(0, n), which have no address."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(params=["bf16", "fp32"])
def mode(request):
    from paper_2605_06665_b200 import binding as B
    from paper_2605_06665_b200 import build as builder
    builder.build()
    code, dt = (B.BF16, torch.bfloat16) if request.param == "bf16" else (B.FP32, torch.float32)
    ctx = B.Context(B.make_config(64, 64, 1, 1, 1, 64, code, 1e-6, 1.0))
    yield ctx, dt, B
    ctx.check_status()
    ctx.close()


def test_norm(mode):
    ctx, dt, B = mode
    a, w, dw = torch.ones(4, 96, dtype=dt, device="cuda")[:0], torch.ones(96, device="cuda"), torch.ones(96, device="cuda")
    s, q = torch.empty(0, device="cuda"), torch.empty(0, 96, dtype=torch.float8_e4m3fn, device="cuda")
    assert a.data_ptr() == 0
    ctx.rmsnorm(a, a, 0, 96, w, 1e-6, a, s, a, q, s)
    ctx.rmsnorm(a, None, 0, 96, w, 1e-6, None, None, a)
    ctx.quantize_rows(a, 0, 96, q, s)
    ctx.rmsnorm_bwd(a, a, 0, 96, w, s, a, a, dw)
    assert (dw == 1).all()
    ctx.rmsnorm_bwd(a, a, 0, 96, w, s, None, a, dw, B.WGRAD_OVERWRITE)
    assert (dw == 0).all()
    with pytest.raises(B.UniPoolError):
        ctx.rmsnorm(a, None, 1, 96, w, 1e-6, None, None, a)


def test_products(mode):
    ctx, dt, B = mode
    x, y = torch.empty(0, 128, dtype=dt, device="cuda"), torch.ones(3, 64, dtype=dt, device="cuda")[:0]
    W, bias = torch.ones(64, 128, dtype=dt, device="cuda"), torch.ones(64, device="cuda")
    for act in B.ACTIVATIONS.values():
        ctx.linear(x, 0, 128, W, 64, bias, act, y, y, y)
        dW, db = torch.ones(64, 128, device="cuda"), torch.ones(64, device="cuda")
        ctx.linear_bwd(y, 0, 64, y, act, x, 128, W, y, x, x, dW, db)
        assert (dW == 1).all() and (db == 1).all()
        ctx.linear_bwd(y, 0, 64, y, act, x, 128, W, y, None, x, dW, db, B.WGRAD_OVERWRITE)
        assert (dW == 0).all() and (db == 0).all()
        ctx.linear_bwd(y, 0, 64, y, act, None, 128, W, y, None, x, None, None)        # frozen weights
    if dt is torch.bfloat16:
        q, s = x.to(torch.float8_e4m3fn), torch.empty(0, device="cuda")
        ctx.linear_scaled(q, s, 0, 128, W.to(torch.float8_e4m3fn), bias, 64, bias, 1, None, None, y)
