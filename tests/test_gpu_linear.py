"""Dense products with their epilogue, in bf16, fp32 and with 8-bit operands, and their backward pass, against float64 on the
same inputs.

Bounds: an output is rounded once, by at most half a step of its type.  A sum of K products is taken by the tensor core in
steps of 16 (32 in 8 bits), each of which may cut off a unit in the last place (2^-23) of what it adds up, or by fp32 FMAs (2^-24
each); the weight gradient's sums are 768 tokens long and added up in fp32.  All relative to the sum of the terms' magnitudes.
The activations' values and slopes are at most 1.13 times as far off as their argument, and 2^-20 of their own."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "silu", "gelu"]
MATH = 2.0 ** -20
SHAPES = [(1, 64, 64), (2, 64, 320), (5, 2048, 768), (16, 128, 64), (17, 192, 128), (31, 256, 256), (33, 576, 64), (64, 1536, 512),
          (65, 448, 192), (127, 64, 512), (129, 320, 320), (200, 4096, 128), (255, 128, 768), (256, 256, 512), (257, 768, 256),
          (513, 192, 576), (700, 64, 2048), (1501, 768, 832), (3000, 256, 64)]


def half_step(dt):
    return torch.finfo(dt).eps / 2


class Mode:
    def __init__(self, name):
        from paper_2605_06665_b200 import binding as B
        self.B = B
        self.bf16 = name != "fp32"
        self.q8 = name == "q8"
        self.dt = torch.bfloat16 if self.bf16 else torch.float32
        self.ctx = B.Context(B.make_config(64, 64, 1, 1, 1, 8192, B.BF16 if self.bf16 else B.FP32, 1e-6, 1.0))

    def steps(self, K):
        """Units of 2^-24 of the terms' magnitudes that a sum of K products may be off."""
        return 2 * (K / (32 if self.q8 else 16) + 16) if self.bf16 else K + 16


def make(name):
    from paper_2605_06665_b200 import build as builder
    builder.build()
    return Mode(name)


@pytest.fixture(scope="module", params=["bf16", "fp32", "q8"])
def mode(request):
    m = make(request.param)
    yield m
    m.ctx.check_status()
    m.ctx.close()


@pytest.fixture(scope="module", params=["bf16", "fp32"])
def train(request):
    m = make(request.param)
    yield m
    m.ctx.check_status()
    m.ctx.close()


def normal(shape, dt, seed, std=1.0):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dt).cuda()


def guarded(shape, dt, fill=7.0):
    n = 1
    for v in shape:
        n *= v
    whole = torch.full((n + 2048,), fill, device="cuda").to(dt)
    return whole, whole[1024:1024 + n].view(shape)


def untouched(whole, part, fill=7.0):
    n, off = part.numel(), part.storage_offset()
    f = whole.float()
    return bool((f[:off] == fill).all() and (f[off + n:] == fill).all())


def value(p, act):
    if act == "relu":
        return p.clamp(min=0)
    if act == "silu":
        return p * torch.sigmoid(p)
    if act == "gelu":
        return 0.5 * p * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (p + 0.044715 * p ** 3)))
    return p


def slope(p, act):
    if act == "none":
        return torch.ones_like(p)
    q = p.detach().clone().requires_grad_(True)
    return torch.autograd.grad(value(q, act).sum(), q)[0] if act != "relu" else (p > 0).double()


class Forward:
    """Operands of one call, and the call."""

    def __init__(self, m, T, n_in, n_out, act="none", bias=True, residual=True, seed=1):
        self.m, self.T, self.n_in, self.n_out, self.act = m, T, n_in, n_out, act
        x, W = normal((T, n_in), m.dt, seed), normal((n_out, n_in), m.dt, seed + 1, n_in ** -0.5)
        self.bias = normal((n_out,), torch.float32, seed + 2, 0.3) if bias else None
        self.res = normal((T, n_out), m.dt, seed + 3) if residual else None
        if m.q8:
            self.x, self.xs = torch.empty(T, n_in, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(T, device="cuda")
            self.W, self.ws = torch.empty(n_out, n_in, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(n_out, device="cuda")
            m.ctx.quantize_rows(x, T, n_in, self.x, self.xs)
            m.ctx.quantize_rows(W, n_out, n_in, self.W, self.ws)
            self.x64, self.W64 = self.x.double() * self.xs.double()[:, None], self.W.double() * self.ws.double()[:, None]
        else:
            self.x, self.W = x, W
            self.x64, self.W64 = x.double(), W.double()

    def call(self, y, pre=None, res=None, T=None):
        c, T, act = self.m.ctx, self.T if T is None else T, self.m.B.ACTIVATIONS[self.act]
        res = self.res if res is None else res
        if self.m.q8:
            c.linear_scaled(self.x, self.xs, T, self.n_in, self.W, self.ws, self.n_out, self.bias, act, res, pre, y)
        else:
            c.linear(self.x, T, self.n_in, self.W, self.n_out, self.bias, act, res, pre, y)

    def check(self, y, pre=None):
        m = self.m
        b = 0 if self.bias is None else self.bias.double()
        r = 0 if self.res is None else self.res.double()
        p = self.x64 @ self.W64.T + b
        # (8 bits: two more fp32 products with the scales)
        off = 2.0 ** -24 * (m.steps(self.n_in) * (self.x64.abs() @ self.W64.abs().T) + 8 * p.abs())
        if pre is not None:
            assert ((pre.double() - p).abs() <= half_step(m.dt) * p.abs() + 2 * off).all()
        want = value(p, self.act) + r
        bound = half_step(m.dt) * want.abs() * 1.001 + 1.13 * off + MATH * value(p, self.act).abs() + 2.0 ** -23 * want.abs()
        worst = ((y.double() - want).abs() - bound).max().item()
        assert worst <= 0, worst


@pytest.mark.parametrize("T,n_in,n_out", SHAPES)
def test_forward_sizes(mode, T, n_in, n_out):
    """Bias, residual and the value before the activation together, in the middle of an array that stays as it is."""
    f = Forward(mode, T, n_in, n_out, "silu")
    yw, y = guarded((T, n_out), mode.dt)
    pw, pre = guarded((T, n_out), mode.dt)
    f.call(y, pre)
    torch.cuda.synchronize()
    assert untouched(yw, y) and untouched(pw, pre)
    f.check(y, pre)
    y2 = torch.empty_like(y)
    f.call(y2)
    assert torch.equal(y2, y)                                # without pre, and the same bits again


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T", [3, 100, 700])
def test_forward_epilogues(mode, act, bias, residual, T):
    f = Forward(mode, T, 192, 320, act, bias, residual, seed=5)
    y, pre = (torch.empty(T, 320, dtype=mode.dt, device="cuda") for _ in range(2))
    f.call(y, pre)
    f.check(y, pre)


@pytest.mark.parametrize("act,bias,residual,with_pre", [("none", False, False, False), ("gelu", True, False, True), ("silu", False, True, False),
                                                         ("gelu", True, True, True), ("relu", True, True, False)])
def test_forward_of_many_tokens(mode, act, bias, residual, with_pre):
    """Several rounds of the widest tiles, a ragged last one; in place where there is a residual."""
    T, n_in, n_out = 8003, 256, 2112
    f = Forward(mode, T, n_in, n_out, act, bias, residual, seed=15)
    yw, y = guarded((T, n_out), mode.dt)
    pw, pre = guarded((T, n_out), mode.dt)
    f.call(y, pre if with_pre else None)
    f.check(y, pre if with_pre else None)
    assert untouched(yw, y) and untouched(pw, pre)
    if residual:
        z = f.res.clone()
        f.call(z, pre if with_pre else None, res=z)
        assert torch.equal(z, y)


def test_backward_of_many_tokens(train):
    m, T, n_in, n_out = train, 8003, 2112, 256
    d = backward_case(m, T, n_in, n_out, "relu", seed=25)
    xw, dx = guarded((T, n_in), m.dt)
    ww, dW = guarded((n_out, n_in), torch.float32)
    db = torch.empty(n_out, device="cuda")
    call_backward(m, d, T, n_in, n_out, "relu", dx, dW, db)
    check_backward(m, d, T, "relu", dx, dW, db)
    assert untouched(xw, dx) and untouched(ww, dW)
    res = d["res"].clone()
    call_backward(m, d, T, n_in, n_out, "relu", res, None, None, res=res)
    assert torch.equal(res, dx)


@pytest.mark.parametrize("T", [3, 700])
def test_residual_in_place_and_fewer_tokens(mode, T):
    f = Forward(mode, T, 128, 320, "gelu", seed=7)
    y, z = torch.empty(T, 320, dtype=mode.dt, device="cuda"), f.res.clone()
    f.call(y)
    f.call(z, res=z)
    assert torch.equal(y, z)
    z = torch.full_like(y, 7.0)
    f.call(z, T=T - 1)                                       # the last row is left as it was
    assert torch.equal(z[:-1], y[:-1]) and (z[-1] == 7).all()
    f.call(z, T=0)
    assert torch.equal(z[:-1], y[:-1])


@pytest.mark.parametrize("T", [2, 300])
def test_infinities_and_nan_stay_in_their_row(mode, T):
    f = Forward(mode, T, 128, 128, "relu", bias=False, residual=False, seed=9)
    y, z = torch.empty(T, 128, dtype=mode.dt, device="cuda"), torch.empty(T, 128, dtype=mode.dt, device="cuda")
    f.call(y)
    if mode.q8:
        f.xs[1] = float("nan")
    else:
        f.x[1, 3] = float("nan")
    f.call(z)
    assert torch.isnan(z[1]).all()
    keep = [t for t in range(T) if t != 1]
    assert torch.equal(z[keep], y[keep])


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_large_arguments(train, act):
    """Far out the activations are 0 or their argument, and their slopes 0 or 1, without overflow."""
    m = train
    T, n = 4, 64
    x = torch.zeros(T, n, device="cuda", dtype=m.dt)
    W = torch.zeros(n, n, device="cuda", dtype=m.dt)
    W[:, 0] = 1
    x[:, 0] = torch.tensor([1e15, -1e15, 100.0, -100.0]).to(m.dt)
    y, pre, dp = (torch.empty(T, n, device="cuda", dtype=m.dt) for _ in range(3))
    m.ctx.linear(x, T, n, W, n, None, m.B.ACTIVATIONS[act], None, pre, y)
    assert torch.equal(pre, x[:, :1].expand(T, n))
    assert torch.equal(y[[0, 2]], pre[[0, 2]]) and (y[[1, 3]].abs() < 1e-30).all()
    dy = torch.ones_like(y)
    m.ctx.linear_bwd(dy, T, n, pre, m.B.ACTIVATIONS[act], x, n, W, dp, None, torch.empty_like(x), None, None)
    assert (dp[[0, 2]] == 1).all() and (dp[[1, 3]].abs() < 1e-30).all()


def backward_case(m, T, n_in, n_out, act, seed=11):
    d = dict(dy=normal((T, n_out), m.dt, seed), pre=None if act == "none" else normal((T, n_out), m.dt, seed + 1, 2.0),
             x=normal((T, n_in), m.dt, seed + 2), W=normal((n_out, n_in), m.dt, seed + 3, n_in ** -0.5),
             res=normal((T, n_in), m.dt, seed + 4), dp=None if act == "none" else torch.empty(T, n_out, dtype=m.dt, device="cuda"))
    return d


def call_backward(m, d, T, n_in, n_out, act, dx, dW, db, flags=1, **over):
    d = dict(d, **over)
    m.ctx.linear_bwd(d["dy"], T, n_out, d["pre"], m.B.ACTIVATIONS[act], d["x"], n_in, d["W"], d["dp"], d["res"], dx, dW, db,
                     m.B.WGRAD_OVERWRITE if flags else 0)


def check_backward(m, d, T, act, dx, dW, db):
    dp = d["dy"].double()
    if act != "none":
        dp = dp * slope(d["pre"].double(), act)
    x, W = d["x"].double(), d["W"].double()
    # dp as an operand: rounded to the type where there is an activation (exact with relu), fast math before that
    rough = 0.0 if act in ("none", "relu") else half_step(m.dt) + MATH
    slack = (MATH * d["dy"].double().abs() * 1.2) if act in ("silu", "gelu") else torch.zeros_like(dp)
    mag = dp.abs()
    if dx is not None:
        want = dp @ W + (0 if d["res"] is None else d["res"].double())
        terms, more = mag @ W.abs(), slack @ W.abs()
        bound = half_step(m.dt) * 1.001 * want.abs() + (rough + 2.0 ** -24 * m.steps(W.shape[0])) * terms + more + 2.0 ** -23 * want.abs()
        assert ((dx.double() - want).abs() <= bound).all()
    if dW is not None:
        want, terms, more = dp.T @ x, mag.T @ x.abs(), slack.T @ x.abs()
        steps = 2 * (48 + 2 * T / 768 + 96) if m.bf16 else T + 64
        assert ((dW.double() - want).abs() <= (rough + 2.0 ** -24 * steps) * terms + more).all()
    if db is not None:
        bound = (T + 64) * 2.0 ** -24 * mag.sum(0) + slack.sum(0) + (MATH if rough else 0) * mag.sum(0)
        assert ((db.double() - dp.sum(0)).abs() <= bound).all()


@pytest.mark.parametrize("T,n_in,n_out", SHAPES)
def test_backward_sizes(train, T, n_in, n_out):
    m = train
    d = backward_case(m, T, n_in, n_out, "relu")
    xw, dx = guarded((T, n_in), m.dt)
    ww, dW = guarded((n_out, n_in), torch.float32)
    bw, db = guarded((n_out,), torch.float32)
    call_backward(m, d, T, n_in, n_out, "relu", dx, dW, db)
    torch.cuda.synchronize()
    assert untouched(xw, dx) and untouched(ww, dW) and untouched(bw, db)
    check_backward(m, d, T, "relu", dx, dW, db)
    # once more, the same bits; added to what is there
    dx2, dW2, db2 = torch.empty_like(dx), torch.full_like(dW, 2.0), torch.full_like(db, 2.0)
    call_backward(m, d, T, n_in, n_out, "relu", dx2, dW2, db2, flags=0)
    assert torch.equal(dx2, dx) and torch.equal(dW2, dW + 2.0) and torch.equal(db2, db + 2.0)
    # one at a time (in one launch the products may be cut into other parts than alone)
    call_backward(m, d, T, n_in, n_out, "relu", dx2, None, None)
    call_backward(m, d, T, n_in, n_out, "relu", None, dW2, None)
    call_backward(m, d, T, n_in, n_out, "relu", None, None, db2)
    check_backward(m, d, T, "relu", dx2, dW2, db2)
    dW3, db3 = torch.full_like(dW, 2.0), torch.full_like(db, 2.0)
    call_backward(m, d, T, n_in, n_out, "relu", None, dW3, None, flags=0)
    call_backward(m, d, T, n_in, n_out, "relu", None, None, db3, flags=0)
    assert torch.equal(dW3, dW2 + 2.0) and torch.equal(db3, db2 + 2.0)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T,n_in,n_out", [(129, 832, 448), (600, 3008, 640), (1501, 832, 2048), (2500, 1600, 704), (4111, 1088, 1536),
                                          (6001, 512, 1984), (7003, 704, 704)])
def test_backward_products_of_one_launch(train, T, n_in, n_out, residual):
    """Sizes at which dx and dW share a launch in bf16: both tile widths, ragged in each direction, dW in one part and in several."""
    m = train
    d = backward_case(m, T, n_in, n_out, "relu", seed=5)
    xw, dx = guarded((T, n_in), m.dt)
    ww, dW = guarded((n_out, n_in), torch.float32)
    db = torch.empty(n_out, device="cuda")
    d = d if residual else dict(d, res=None)
    call_backward(m, d, T, n_in, n_out, "relu", dx, dW, db)
    torch.cuda.synchronize()
    assert untouched(xw, dx) and untouched(ww, dW)
    check_backward(m, d, T, "relu", dx, dW, db)
    dx2, dW2 = (d["res"].clone() if residual else torch.empty_like(dx)), torch.full_like(dW, 2.0)
    call_backward(m, d, T, n_in, n_out, "relu", dx2, dW2, None, flags=0, res=dx2 if residual else None)   # dx onto its residual
    assert torch.equal(dx2, dx) and torch.equal(dW2, dW + 2.0)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T", [3, 700, 5000])
def test_backward_activations(train, act, T):
    m = train
    d = backward_case(m, T, 192, 320, act, seed=21)
    dx, dW, db = torch.empty(T, 192, dtype=m.dt, device="cuda"), torch.empty(320, 192, device="cuda"), torch.empty(320, device="cuda")
    call_backward(m, d, T, 192, 320, act, dx, dW, db, res=None)
    check_backward(m, dict(d, res=None), T, act, dx, dW, db)
    # dp over pre, dx over its residual
    pre, res = None if d["pre"] is None else d["pre"].clone(), d["res"].clone()
    dx2 = torch.empty_like(dx)
    call_backward(m, d, T, 192, 320, act, dx, dW, db)
    call_backward(m, d, T, 192, 320, act, res, None, None, pre=pre, dp=pre, res=res)
    assert torch.equal(res, dx)
    if pre is not None:
        assert torch.equal(pre, d["dp"])


def test_gradients_by_differences(train):
    """sum(g y) through the forward call's own definition in float64, against the backward call."""
    m = train
    T, n_in, n_out, act = 6, 64, 64, "gelu"
    f = Forward(m, T, n_in, n_out, act, seed=31)
    y, pre, dp = (torch.empty(T, n_out, dtype=m.dt, device="cuda") for _ in range(3))
    f.call(y, pre)
    g = normal((T, n_out), m.dt, 35)
    dx, dW, db = torch.empty(T, n_in, dtype=m.dt, device="cuda"), torch.empty(n_out, n_in, device="cuda"), torch.empty(n_out, device="cuda")
    m.ctx.linear_bwd(g, T, n_out, pre, m.B.ACTIVATIONS[act], f.x, n_in, f.W, dp, None, dx, dW, db, m.B.WGRAD_OVERWRITE)

    def loss(x, W, b):
        return (g.double() * (value(x @ W.T + b, act) + f.res.double())).sum()

    # bf16: pre and dp are rounded (2^-8 each, slopes change by 2^-8 |pre| at most), sums of 64 terms of size up to 3
    tol = 64 * 3 * 3 * 2.0 ** -8 / 8 if m.bf16 else 1e-4
    args, h = [f.x64, f.W64, f.bias.double()], 1e-5
    for which, out, at in ((0, dx, (2, 5)), (0, dx, (5, 63)), (1, dW, (7, 9)), (1, dW, (63, 0)), (2, db, (11,))):
        lo, hi = [a.clone() for a in args], [a.clone() for a in args]
        lo[which][at] -= h
        hi[which][at] += h
        want = (loss(*hi) - loss(*lo)) / (2 * h)
        assert abs(out[at].double() - want) <= tol


def test_scratch_of_the_callers(train):
    m = train
    for T, n_in, n_out in ((40, 64, 64), (700, 128, 192), (3000, 64, 320)):
        d = backward_case(m, T, n_in, n_out, "relu", seed=81)
        n = m.ctx.linear_bwd_scratch(T, n_in, n_out)
        out = [[torch.empty(n_out, n_in, device="cuda"), torch.empty(n_out, device="cuda")] for _ in range(2)]
        whole = torch.full((n + 64,), 7, dtype=torch.uint8, device="cuda")
        for o, scratch in zip(out, (None, whole[:n])):
            m.ctx.linear_bwd(d["dy"], T, n_out, d["pre"], 1, d["x"], n_in, d["W"], d["dp"], None, None, *o, m.B.WGRAD_OVERWRITE, scratch)
        assert all(torch.equal(a, b) for a, b in zip(*out)) and (whole[n:] == 7).all()
        if n:
            with pytest.raises(ValueError):
                m.ctx.linear_bwd(d["dy"], T, n_out, d["pre"], 1, d["x"], n_in, d["W"], d["dp"], None, None, *out[0], 2, whole[:n - 1])


def test_no_tokens(train):
    m = train
    a, dW, db = torch.ones(64, 64, dtype=m.dt, device="cuda"), torch.ones(64, 64, device="cuda"), torch.ones(64, device="cuda")
    m.ctx.linear_bwd(a, 0, 64, None, 0, a, 64, a, None, None, a, dW, db)
    assert (a == 1).all() and (dW == 1).all() and (db == 1).all()
    m.ctx.linear_bwd(a, 0, 64, None, 0, a, 64, a, None, None, a, dW, db, m.B.WGRAD_OVERWRITE)
    assert (a == 1).all() and (dW == 0).all() and (db == 0).all()


def test_misaligned_fp32():
    """fp32 operands 4 bytes off a 16-byte boundary; a bf16 context refuses them."""
    T, n_in, n_out = 150, 128, 192
    for name in ("fp32", "bf16"):
        m = make(name)

        def off(t):
            whole = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
            whole[1:] = t.reshape(-1)
            return whole[1:].view(t.shape)

        f = Forward(m, T, n_in, n_out, "silu", seed=41)
        d = backward_case(m, T, n_in, n_out, "gelu")
        y, dx, dW, db = (off(torch.empty(s, dtype=t, device="cuda")) for s, t in
                         (((T, n_out), m.dt), ((T, n_in), m.dt), ((n_out, n_in), torch.float32), ((n_out,), torch.float32)))
        if name == "bf16":
            with pytest.raises(m.B.UniPoolError) as e:
                f.call(y)
            assert e.value.code == -1 and "aligned" in str(e.value)
            with pytest.raises(m.B.UniPoolError) as e:
                call_backward(m, d, T, n_in, n_out, "gelu", dx, dW, db)
            assert e.value.code == -1 and "aligned" in str(e.value)
            good = torch.empty(T, n_out, dtype=m.dt, device="cuda")
            f.bias = off(f.bias)                             # the bias needs no alignment
            f.call(good)
            f.check(good)
        else:
            f.x, f.W, f.bias, f.res = off(f.x), off(f.W), off(f.bias), off(f.res)
            f.call(y)
            f.check(y)
            d = {k: off(v) for k, v in d.items()}
            call_backward(m, d, T, n_in, n_out, "gelu", dx, dW, db)
            check_backward(m, d, T, "gelu", dx, dW, db)
        m.ctx.check_status()
        m.ctx.close()


@pytest.mark.parametrize("T", [40, 200, 900])
def test_captured_calls_on_two_streams(train, T):
    """Forward and backward recorded twice, each with scratch of its own, replayed on two streams at once."""
    m = train
    n_in, n_out, act = 256, 384, "silu"
    sets = []
    for i in range(2):
        d = backward_case(m, T, n_in, n_out, act, seed=50 + 10 * i)
        out = [torch.zeros(T, n_in, dtype=m.dt, device="cuda"), torch.zeros(n_out, n_in, device="cuda"),
               torch.zeros(n_out, device="cuda"), torch.zeros(T, n_out, dtype=m.dt, device="cuda")]

        def calls(d=d, out=out):
            m.ctx.linear(d["x"], T, n_in, d["W"], n_out, out[2], m.B.ACTIVATIONS[act], None, None, out[3])
            call_backward(m, d, T, n_in, n_out, act, *out[:3])

        call_backward(m, d, T, n_in, n_out, act, *out[:3])
        calls()
        torch.cuda.synchronize()
        want = [t.clone() for t in out]
        s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            calls()
        sets.append((g, s, out, want, d))                    # (d: the recording reads it)
    for _ in range(3):
        for _, _, out, _, _ in sets:
            out[0].zero_(), out[1].zero_(), out[3].zero_()
        torch.cuda.synchronize()
        for g, s, _, _, _ in sets:
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for _, _, out, want, _ in sets:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_dense_block_in_eight_bits():
    """A run of them as an evaluation uses them: norm with the residual's addition -> 8 bits -> product with silu -> 8 bits ->
    product with bias and residual -> norm; each step against float64 on what the step before it gave."""
    m = make("q8")
    c, B = m.ctx, m.B
    T, d, f = 333, 768, 2048
    x, y0 = normal((T, d), m.dt, 60), normal((T, d), m.dt, 61, 0.5)
    w1, w2 = 1 + normal((d,), torch.float32, 62, 0.1), 1 + normal((d,), torch.float32, 63, 0.1)
    e4m3 = torch.float8_e4m3fn
    W = [normal((f, d), m.dt, 64, d ** -0.5), normal((d, f), m.dt, 65, f ** -0.5)]
    Wq = [(torch.empty(v.shape, dtype=e4m3, device="cuda"), torch.empty(len(v), device="cuda")) for v in W]
    for v, (q, s) in zip(W, Wq):
        c.quantize_rows(v, v.shape[0], v.shape[1], q, s)
    bias = normal((d,), torch.float32, 66, 0.1)
    r, q1, s1 = torch.empty_like(x), torch.empty(T, d, dtype=e4m3, device="cuda"), torch.empty(T, device="cuda")
    a, q2, s2 = torch.empty(T, f, dtype=m.dt, device="cuda"), torch.empty(T, f, dtype=e4m3, device="cuda"), torch.empty(T, device="cuda")
    out, h = torch.empty_like(x), torch.empty_like(x)
    c.rmsnorm(x, y0, T, d, w1, 1e-6, r, None, None, q1, s1)
    c.linear_scaled(q1, s1, T, d, *Wq[0], f, None, B.ACTIVATIONS["silu"], None, None, a)
    c.quantize_rows(a, T, f, q2, s2)
    c.linear_scaled(q2, s2, T, f, *Wq[1], d, bias, 0, r, None, out)
    c.rmsnorm(out, None, T, d, w2, 1e-6, None, None, h)

    def close(got, want, terms, K):
        bound = half_step(m.dt) * 1.001 * want.abs() + 2.0 ** -24 * (m.steps(K) + 300) * terms + MATH * want.abs()
        assert ((got.double() - want).abs() <= bound).all()

    sums = x.double() + y0.double()
    close(r, sums, sums.abs(), 0)
    hh = sums / torch.sqrt((sums ** 2).mean(1, keepdim=True) + 1e-6) * w1.double()
    deq = lambda q, s: q.double() * s.double()[:, None]
    assert ((deq(q1, s1) - hh).abs() <= (2.0 ** -4 + 1e-4) * hh.abs() + 2.0 ** -9 * s1.double()[:, None]).all()
    p = deq(q1, s1) @ deq(*Wq[0]).T
    close(a, p * torch.sigmoid(p), 1.13 * deq(q1, s1).abs() @ deq(*Wq[0]).abs().T, d)
    close(out, deq(q2, s2) @ deq(*Wq[1]).T + bias.double() + r.double(), deq(q2, s2).abs() @ deq(*Wq[1]).abs().T + 1, f)
    o = out.double()
    want = o / torch.sqrt((o ** 2).mean(1, keepdim=True) + 1e-6) * w2.double()
    close(h, want, want.abs(), 0)
    # and the whole run is what the 16-bit arithmetic of the same block gives, to a few percent of its size
    p = hh @ W[0].double().T
    full = (p * torch.sigmoid(p)) @ W[1].double().T + bias.double() + sums
    # relative 2-norm: four roundings to e4m3 (uniform in half a step: 2^-4 / sqrt(3) each at most) of the product's path
    path = full - sums - bias.double()
    assert (out.double() - full).norm() <= 4 * 2.0 ** -4 / 3 ** 0.5 * path.norm() + half_step(m.dt) * 2 * full.norm()
    c.check_status()
    c.close()


def test_more_than_32_bits_of_elements():
    """17000 tokens of 131072 features: the last ones lie 2.2e9 elements behind the first, in the result, the residual and dp."""
    from paper_2605_06665_b200 import binding as B
    T, n_in, n_out, dt = 17_000, 64, 131_072, torch.bfloat16
    ctx = B.Context(B.make_config(64, 64, 1, 1, 1, T, B.BF16, 1e-6, 1.0))
    x, W, bias = normal((T, n_in), dt, 70), normal((n_out, n_in), dt, 71, 0.1), normal((n_out,), torch.float32, 72)
    rows = [0, 255, 16383, 16384, 16385, T - 1]
    y = torch.zeros(T, n_out, dtype=dt, device="cuda")
    y[rows] = normal((len(rows), n_out), dt, 73)
    res = y[rows].double()
    ctx.linear(x, T, n_in, W, n_out, bias, 0, y, None, y)
    want = x[rows].double() @ W.double().T + bias.double() + res
    terms = x[rows].double().abs() @ W.double().abs().T + bias.double().abs() + res.abs()
    assert ((y[rows].double() - want).abs() <= half_step(dt) * 1.001 * want.abs() + 2.0 ** -24 * 48 * terms).all()
    dx, dW = torch.empty_like(x), torch.empty(n_out, n_in, device="cuda")
    keep = torch.zeros(T, dtype=torch.bool, device="cuda")
    keep[rows] = True
    y[~keep] = 0
    db = torch.empty(n_out, device="cuda")
    ctx.linear_bwd(y, T, n_out, None, 0, x, n_in, W, None, None, dx, dW, db, B.WGRAD_OVERWRITE)
    g = y[rows].double()
    want, terms = g @ W.double(), g.abs() @ W.double().abs()
    assert ((dx[rows].double() - want).abs() <= half_step(dt) * 1.001 * want.abs() + 2.0 ** -24 * 2 * (n_out / 16 + 16) * terms).all()
    want, terms = g.T @ x[rows].double(), g.abs().T @ x[rows].double().abs()
    assert ((dW.double() - want).abs() <= 2.0 ** -24 * 500 * terms).all()
    assert ((db.double() - g.sum(0)).abs() <= 64 * 2.0 ** -24 * g.abs().sum(0)).all()
    ctx.check_status()
    ctx.close()
