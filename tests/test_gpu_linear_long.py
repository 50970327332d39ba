"""Dense products whose contraction is long.  The tensor core truncates the sums it adds to, in steps of 16 terms (32 in 8 bits) by less than
a unit in the last place, 2^-23, of what it has: sums are taken from the accumulator after 16384 terms (32768), by the kernel for few tokens after
65536 (131072) of a CTA's, and added up in fp32 with rounding to nearest.  So a sum is off by at most 2^-23 x (steps of such a part) of
the terms' magnitudes, and 2^-24 for each part added, however long it is."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8                                             # half a step of bf16
PAIRS, FEW = 2.0 ** -23 * (1024 + 16) + 2.0 ** -24 * 130, 2.0 ** -23 * (4096 + 16) + 2.0 ** -24 * 130


@pytest.fixture(scope="module")
def ctx():
    from paper_2605_06665_b200 import binding as B
    from paper_2605_06665_b200 import build as builder
    builder.build()
    c = B.Context(B.make_config(64, 64, 1, 1, 1, 8192, B.BF16, 1e-6, 1.0))
    yield c
    c.check_status()
    c.close()


def positive(T, K, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(T, K, device="cuda").uniform_(1.0, 2.0, generator=g).bfloat16()


def sums(x):
    return torch.cat([c.double().sum(1) for c in x.split(64)])


@pytest.mark.parametrize("T,K,N", [(4096, 1 << 18, 2048), (300, 1 << 20, 192), (5, 1 << 19, 64), (5, (1 << 19) + 64, 64), (3, 1 << 21, 64)])
def test_terms_of_one_sign(ctx, T, K, N):
    x, w = positive(T, K, 1), torch.exp(torch.linspace(0, 1, N, device="cuda")).bfloat16()
    want = sums(x)[:, None] * w.double()
    # (K / 64 blocks over a cluster of eight: up to 1024 each go to the kernel for few tokens)
    bound = HALF + (FEW if T <= 128 and K <= 1 << 19 else PAIRS)
    W = w[:, None].expand(N, K).contiguous()
    y = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    ctx.linear(x, T, K, W, N, None, 0, None, None, y)
    assert ((y.double() - want).abs() <= bound * want).all()
    W = W.t().contiguous()                                   # the same sums as a gradient: dx = dy W over K outputs
    dx = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    ctx.linear_bwd(x, T, K, None, 0, None, N, W, None, None, dx, None, None)
    assert ((dx.double() - want).abs() <= bound * want).all()


@pytest.mark.parametrize("T,K,N", [(4096, 1 << 20, 2048), (5, 1 << 20, 64)])
def test_terms_of_one_sign_in_eight_bits(ctx, T, K, N):
    """Values with all of e4m3's bits, K equal ones after another: the sums need more than 24 bits from 2^17 terms on."""
    w = torch.full((N,), 1.875, device="cuda")
    x = torch.empty(T, K, dtype=torch.float8_e4m3fn, device="cuda")
    for c in x.split(256):
        c.copy_((1.0 + (torch.arange(K, device="cuda") * 5 % 8) / 8.0).expand(len(c), K))
    want = (x[:1].double().sum(1) * 1.875)[:, None].expand(T, N)
    W = w.to(torch.float8_e4m3fn).view(torch.uint8)[:, None].expand(N, K).contiguous()
    one = torch.ones(max(T, N), device="cuda")
    y = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    ctx.linear_scaled(x, one[:T], T, K, W, one[:N], N, None, 0, None, None, y)
    assert ((y.double() - want).abs() <= (HALF + (PAIRS if T > 128 else FEW)) * want).all()


@pytest.mark.parametrize("T,N", [(1501, 320), (3000, 2112)])
@pytest.mark.parametrize("residual,with_pre", [(False, False), (True, False), (True, True), (False, True)])
@pytest.mark.parametrize("K", [16384, 16448, 40000, 49152])  # one whole part, and one block; three parts, ragged and whole
def test_epilogues_of_several_parts(ctx, T, N, residual, with_pre, K):
    from paper_2605_06665_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(K + T)
    normal = lambda *s, std=1.0, dt=torch.bfloat16: (torch.empty(*s, device="cuda").normal_(0.0, std, generator=g)).to(dt)
    x, W, bias = normal(T, K), normal(N, K, std=K ** -0.5), normal(N, dt=torch.float32)
    res, pre = normal(T, N) if residual else None, torch.empty(T, N, dtype=torch.bfloat16, device="cuda") if with_pre else None
    y = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    ctx.linear(x, T, K, W, N, bias, B.ACTIVATIONS["relu"], res, pre, y)
    p, terms = x.double() @ W.double().T + bias.double(), x.double().abs() @ W.double().abs().T + bias.double().abs()
    if with_pre:
        assert ((pre.double() - p).abs() <= HALF * p.abs() + PAIRS * terms).all()
    want = p.clamp(min=0) + (res.double() if residual else 0)
    assert ((y.double() - want).abs() <= HALF * 1.001 * want.abs() + PAIRS * terms + 2.0 ** -23 * want.abs()).all()


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T,n_in,n_out", [(700, 256, 40000), (1501, 1024, 20032), (200, 64, 49152)])
def test_gradients_of_several_parts(ctx, T, n_in, n_out, residual):
    """dx of many output features beside dW, which may share its launch, and alone."""
    from paper_2605_06665_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(n_out)
    normal = lambda *s, std=1.0: (torch.empty(*s, device="cuda").normal_(0.0, std, generator=g)).bfloat16()
    dy, W, x, res = normal(T, n_out), normal(n_out, n_in, std=n_out ** -0.5), normal(T, n_in), normal(T, n_in) if residual else None
    want, terms = dy.double() @ W.double(), dy.double().abs() @ W.double().abs()
    if residual:
        want, terms = want + res.double(), terms + res.double().abs()
    wantW, termsW = dy.double().T @ x.double(), dy.double().abs().T @ x.double().abs()
    for dW in (torch.empty(n_out, n_in, device="cuda"), None):
        dx = torch.empty_like(x)
        ctx.linear_bwd(dy, T, n_out, None, 0, x, n_in, W, None, res, dx, dW, None, B.WGRAD_OVERWRITE)
        assert ((dx.double() - want).abs() <= HALF * 1.001 * want.abs() + PAIRS * terms).all()
        if dW is not None:
            assert ((dW.double() - wantW).abs() <= 2.0 ** -24 * 300 * termsW).all()
