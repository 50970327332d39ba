"""RMS norm with the residual's addition, its 8-bit output and its backward pass, against float64 on the same inputs.

Bounds: an output is rounded once, by at most half a step of its type (eps / 2 of its value), on top of fp32 arithmetic.  A
thread adds up at most 32 x 8 squares of a row before the tree of its neighbours: FP32 = 2^-24 x 300 covers a sum of them, the
square root, the division and the products, relative to the terms' magnitudes."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FP32 = 300 * 2.0 ** -24
EPS = 1e-6
SIZES = [(1, 768), (3, 1), (5, 7), (33, 64), (130, 768), (37, 1000), (37, 1001), (700, 256), (9, 1536), (9, 2048), (9, 2056),
         (5, 4104), (3, 8192), (2, 8200), (3, 16384), (2, 16383)]


@pytest.fixture(scope="module", params=["bf16", "fp32"])
def mode(request):
    from paper_2605_06665_b200 import binding as B
    from paper_2605_06665_b200 import build as builder
    builder.build()
    code, dt = (B.BF16, torch.bfloat16) if request.param == "bf16" else (B.FP32, torch.float32)
    ctx = B.Context(B.make_config(64, 64, 1, 1, 1, 8192, code, EPS, 1.0))
    yield ctx, dt
    ctx.check_status()
    ctx.close()


def normal(shape, dt, seed, std=1.0):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dt).cuda()


def half_step(dt):
    return torch.finfo(dt).eps / 2


def guarded(shape, dt, fill=7.0, offset=0):
    """An array with as many elements of `fill` in front and behind, `offset` elements off its alignment."""
    n = 1
    for v in shape:
        n *= v
    whole = torch.full((n + 64 + offset,), fill, device="cuda").to(dt)
    return whole, whole[32 + offset:32 + offset + n].view(shape)


def untouched(whole, part, fill=7.0):
    n, off = part.numel(), part.storage_offset()
    f = whole.float()
    return bool((f[:off] == fill).all() and (f[off + n:] == fill).all())


def reference(x, y, w, eps):
    r = x.double() if y is None else x.double() + y.double()
    rstd = 1.0 / torch.sqrt((r * r).mean(1) + eps)
    return r, rstd, r * rstd[:, None] * w.double()


def check_q(q, scale, h):
    """8 bits against the unrounded values: the scale, and each value within half a step of e4m3 (2^-4 of it, or half the
    smallest number).  The bound on values allows for the scale's own error."""
    amax = h.abs().amax(1)
    want = torch.clamp(amax / 448, min=2.0 ** -126)
    assert ((scale.double() - want).abs() <= 2 * FP32 * want).all()
    got = q.double() * scale.double()[:, None]
    assert ((got - h).abs() <= (2.0 ** -4 + 4 * FP32) * h.abs() + 2.0 ** -10 * want[:, None] * (1 + FP32)).all()


@pytest.mark.parametrize("T,width", SIZES)
@pytest.mark.parametrize("with_y", [False, True])
def test_forward(mode, T, width, with_y):
    ctx, dt = mode
    x, y = normal((T, width), dt, 1), normal((T, width), dt, 2, 0.5) if with_y else None
    w = 1 + normal((width,), torch.float32, 3, 0.2)
    hw, h = guarded((T, width), dt)
    rw, r = guarded((T, width), dt)
    sw, rstd = guarded((T,), torch.float32)
    qw, q = guarded((T, width), torch.float8_e4m3fn)
    cw, scale = guarded((T,), torch.float32)
    ctx.rmsnorm(x, y, T, width, w, EPS, r, rstd, h, q, scale)
    torch.cuda.synchronize()
    for whole, part in ((hw, h), (rw, r), (sw, rstd), (qw, q), (cw, scale)):
        assert untouched(whole, part)
    rr, rs, hh = reference(x, y, w, EPS)
    assert ((r.double() - rr).abs() <= (half_step(dt) + FP32) * rr.abs()).all()
    assert ((rstd.double() - rs).abs() <= FP32 * rs).all()
    # h is a product with the sum itself, which fp32 holds to 2^-24 of the larger addend
    slack = FP32 * (x.double().abs() + (0 if y is None else y.double().abs())) * rs[:, None] * w.double().abs()
    assert ((h.double() - hh).abs() <= half_step(dt) * hh.abs() * (1 + FP32) + slack).all()
    check_q(q, scale, hh)
    # single outputs, and the same bits again
    h2, q2, scale2 = torch.empty_like(h), torch.empty_like(q), torch.empty_like(scale)
    ctx.rmsnorm(x, y, T, width, w, EPS, None, None, h2)
    ctx.rmsnorm(x, y, T, width, w, EPS, None, None, None, q2, scale2)
    assert torch.equal(h2, h) and torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(scale2, scale)


@pytest.mark.parametrize("width", [301, 770, 1001, 2187, 4374, 3001, 6002])
def test_forward_of_many_rows_of_any_width(mode, width):
    test_forward(mode, 1301, width, True)


@pytest.mark.parametrize("T,width", SIZES)
@pytest.mark.parametrize("with_dr", [False, True])
def test_backward(mode, T, width, with_dr):
    ctx, dt = mode
    from paper_2605_06665_b200 import binding as B
    dh, r = normal((T, width), dt, 4, 0.1), normal((T, width), dt, 5)
    dr = normal((T, width), dt, 6, 0.1) if with_dr else None
    w = 1 + normal((width,), torch.float32, 7, 0.2)
    rstd = torch.rsqrt(r.float().square().mean(1) + EPS)
    xw, dx = guarded((T, width), dt)
    ww, dw = guarded((width,), torch.float32)
    ctx.rmsnorm_bwd(dh, r, T, width, w, rstd, dr, dx, dw, B.WGRAD_OVERWRITE)
    torch.cuda.synchronize()
    assert untouched(xw, dx) and untouched(ww, dw)
    d, R, n, W = dh.double(), r.double(), rstd.double()[:, None], w.double()
    c, c_abs = (d * W * R).sum(1, keepdim=True), (d * W * R).abs().sum(1, keepdim=True)
    want = n * W * d - R * n ** 3 * c / width
    size = (n * W * d).abs() + R.abs() * n ** 3 * c_abs / width
    if with_dr:
        want, size = want + dr.double(), size + dr.double().abs()
    assert ((dx.double() - want).abs() <= half_step(dt) * want.abs() + FP32 * size).all()
    terms = d * n * R
    assert ((dw.double() - terms.sum(0)).abs() <= (T + 8) * 2.0 ** -24 * terms.abs().sum(0)).all()
    # added to what is there; the same bits again; frozen weights
    dw2, dx2 = torch.full_like(dw, 3.0), torch.empty_like(dx)
    ctx.rmsnorm_bwd(dh, r, T, width, w, rstd, dr, dx2, dw2)
    assert torch.equal(dw2, dw + 3.0) and torch.equal(dx2, dx)
    ctx.rmsnorm_bwd(dh, r, T, width, w, rstd, dr, dx2.zero_(), None)
    assert torch.equal(dx2, dx)


@pytest.mark.parametrize("width", [301, 770, 1001, 1538])
def test_backward_of_many_rows_of_any_width(mode, width):
    test_backward(mode, 5003, width, True)


def test_gradient_by_differences(mode):
    """The gradient of sum(g * h) from the backward call against central differences of the definition in float64."""
    ctx, dt = mode
    from paper_2605_06665_b200 import binding as B
    T, width = 3, 40
    x, g, w = normal((T, width), dt, 8), normal((T, width), dt, 9), 1 + normal((width,), torch.float32, 10, 0.2)
    rstd, dx, dw = torch.empty(T, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    ctx.rmsnorm(x, None, T, width, w, EPS, None, rstd, torch.empty_like(x))
    ctx.rmsnorm_bwd(g, x, T, width, w, rstd, None, dx, dw, B.WGRAD_OVERWRITE)

    def loss(x64, w64):
        return (g.double() * (x64 / torch.sqrt((x64 * x64).mean(1, keepdim=True) + EPS) * w64)).sum()

    step = 1e-5
    for t, j in ((0, 0), (1, 17), (2, 39)):
        a, b = x.double(), x.double()
        a[t, j] += step
        b[t, j] -= step
        want = (loss(a, w.double()) - loss(b, w.double())) / (2 * step)
        # half a step of the result's type, fp32 sums of 40 terms of size about 1, and the differences' own 1e-7
        assert abs(dx[t, j].double() - want) <= half_step(dt) * abs(want) + 1e-5
        a, b = w.double(), w.double()
        a[j] += step
        b[j] -= step
        want = (loss(x.double(), a) - loss(x.double(), b)) / (2 * step)
        assert abs(dw[j].double() - want) <= 1e-5 * (1 + abs(want))


@pytest.mark.parametrize("width", [768, 1001])
def test_misaligned_arrays(mode, width):
    """Arrays one element off a 16-byte boundary go element by element, to the same values."""
    ctx, dt = mode
    from paper_2605_06665_b200 import binding as B
    T = 19
    x, y, w = normal((T, width), dt, 11), normal((T, width), dt, 12), 1 + normal((width,), torch.float32, 13, 0.2)
    want = [torch.empty_like(x) for _ in range(2)] + [torch.empty(T, device="cuda")]
    ctx.rmsnorm(x, y, T, width, w, EPS, want[0], want[2], want[1])

    def off(t):
        whole, part = guarded(t.shape, t.dtype, offset=1)
        part.copy_(t)
        return part

    r, h, rstd = off(want[0]), off(want[1]), off(want[2])
    ctx.rmsnorm(off(x), off(y), T, width, off(w), EPS, r.zero_(), rstd.zero_(), h.zero_())
    bound = half_step(dt) * 2 + FP32
    for got, ref in ((r, want[0]), (h, want[1]), (rstd, want[2])):
        assert ((got.double() - ref.double()).abs() <= bound * ref.double().abs()).all()
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ctx.rmsnorm_bwd(h, r, T, width, w, rstd, y, dx, dw, B.WGRAD_OVERWRITE)
    dx2, dw2 = off(dx), off(dw)
    ctx.rmsnorm_bwd(off(h), off(r), T, width, off(w), off(rstd), off(y), dx2.zero_(), dw2.zero_(), B.WGRAD_OVERWRITE)
    # (h w r sums to `width` terms of size about 1, over width; y of size 1)
    assert ((dx2.double() - dx.double()).abs() <= bound * (dx.double().abs() + 8)).all()
    assert ((dw2.double() - dw.double()).abs() <= FP32 * (h.double() * r.double() * rstd.double()[:, None]).abs().sum(0)).all()


def test_in_place(mode):
    """r over x, h over y; dx over each of the inputs."""
    ctx, dt = mode
    T, width = 70, 768
    x, y, w = normal((T, width), dt, 14), normal((T, width), dt, 15), 1 + normal((width,), torch.float32, 16, 0.2)
    r, h, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(T, device="cuda")
    ctx.rmsnorm(x, y, T, width, w, EPS, r, rstd, h)
    x2, y2 = x.clone(), y.clone()
    ctx.rmsnorm(x2, y2, T, width, w, EPS, x2, None, y2)
    assert torch.equal(x2, r) and torch.equal(y2, h)
    dx = torch.empty_like(x)
    ctx.rmsnorm_bwd(h, r, T, width, w, rstd, y, dx, None)
    for which in range(3):
        args = [h.clone(), r.clone(), y.clone()]
        ctx.rmsnorm_bwd(args[0], args[1], T, width, w, rstd, args[2], args[which], None)
        assert torch.equal(args[which], dx)


@pytest.mark.parametrize("width", [768, 2056, 33])
def test_special_rows(mode, width):
    """A row of zeros, tiny rows, an infinity, a NaN: each row by its formula, none reaches another."""
    ctx, dt = mode
    T = 8
    x, w = normal((T, width), dt, 17), torch.ones(width, device="cuda")
    x[1] = 0.0
    x[2] *= 2.0 ** -70
    x[3, 5] = float("inf")
    x[4, 6] = float("nan")
    x[5] = 0.0
    x[5, 0] = 2.0 ** -120
    h, rstd = torch.empty_like(x), torch.empty(T, device="cuda")
    q, scale = torch.empty(T, width, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(T, device="cuda")
    ctx.rmsnorm(x, None, T, width, w, EPS, None, rstd, h, q, scale)
    for t in (0, 6, 7):
        assert torch.isfinite(h[t]).all() and torch.isfinite(scale[t])
    fine = [0, 1, 2, 5, 6, 7]
    rr, rs, hh = reference(x[fine], None, w, EPS)
    assert ((rstd[fine].double() - rs).abs() <= FP32 * rs).all()
    # (squares below fp32's range are lost beside eps; h of x[5] may be below bf16's normal range: absolute 2^-126)
    assert ((h[fine].double() - hh).abs() <= (half_step(dt) + FP32) * hh.abs() + 2.0 ** -126).all()
    check_q(q[fine], scale[fine], hh)
    assert (h[1] == 0).all() and (q[1].float() == 0).all() and scale[1] == 2.0 ** -126
    assert rstd[3] == 0 and torch.isnan(h[3, 5]) and (h[3, 6:] == 0).all()
    assert torch.isnan(rstd[4]) and torch.isnan(h[4]).all() and torch.isnan(scale[4]) and torch.isnan(q[4].float()).all()


@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** 40])
def test_backward_of_tiny_and_large_rows(mode, scale):
    """The cube of 1 / |r| passes fp32's range, the gradient does not."""
    ctx, dt = mode
    from paper_2605_06665_b200 import binding as B
    T, width = 40, 768
    r, dh = (normal((T, width), torch.float32, 50) * scale).to(dt), normal((T, width), dt, 51)
    w = 1 + normal((width,), torch.float32, 52, 0.2)
    rstd = ((r.double() ** 2).mean(1) ** -0.5).float()
    dx, dw = torch.empty_like(r), torch.empty_like(w)
    ctx.rmsnorm_bwd(dh, r, T, width, w, rstd, None, dx, dw, B.WGRAD_OVERWRITE)
    n, xhat, g = rstd.double()[:, None], r.double() * rstd.double()[:, None], dh.double() * w.double()
    want = n * (g - xhat * (g * xhat).mean(1, keepdim=True))
    size = n * (g.abs() + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True))
    assert torch.isfinite(dx).all()
    assert ((dx.double() - want).abs() <= half_step(dt) * want.abs() + FP32 * size).all()
    terms = dh.double() * xhat
    assert ((dw.double() - terms.sum(0)).abs() <= (T + 8) * 2.0 ** -24 * terms.abs().sum(0)).all()


def test_scratch_of_the_callers(mode):
    ctx, dt = mode
    T, width = 500, 768
    dh, r, w, rstd = normal((T, width), dt, 53), normal((T, width), dt, 54), torch.ones(width, device="cuda"), torch.ones(T, device="cuda")
    n = ctx.rmsnorm_bwd_scratch(T, width)
    want, got = (torch.zeros(width, device="cuda") for _ in range(2))
    dx = torch.empty_like(dh)
    ctx.rmsnorm_bwd(dh, r, T, width, w, rstd, None, dx, want)
    whole = torch.full((n + 64,), 7, dtype=torch.uint8, device="cuda")
    ctx.rmsnorm_bwd(dh, r, T, width, w, rstd, None, dx, got, scratch=whole[:n])
    assert torch.equal(got, want) and (whole[n:] == 7).all()
    with pytest.raises(ValueError):
        ctx.rmsnorm_bwd(dh, r, T, width, w, rstd, None, dx, got, scratch=whole[:n - 1])


def test_scratch_of_many_rows_is_enough_for_fewer(mode):
    ctx, _ = mode
    for width in (1, 64, 768, 1001, 1536, 4096, 9473, 16384):
        sizes = [ctx.rmsnorm_bwd_scratch(T, width) for T in (*range(1, 300), 500, 1000, 3000, 8192)]
        assert sizes == sorted(sizes), width


def test_no_rows(mode):
    ctx, dt = mode
    from paper_2605_06665_b200 import binding as B
    width = 768
    a, w = torch.full((4, width), 2.0, device="cuda", dtype=dt), torch.ones(width, device="cuda")
    rstd, dw = torch.full((4,), 2.0, device="cuda"), torch.full((width,), 2.0, device="cuda")
    ctx.rmsnorm(a, a, 0, width, w, EPS, a, rstd, None, a.view(torch.uint8), rstd)
    ctx.rmsnorm_bwd(a, a, 0, width, w, rstd, a, a, dw)
    ctx.quantize_rows(a, 0, width, a, rstd)
    assert (a == 2).all() and (rstd == 2).all() and (dw == 2).all()
    ctx.rmsnorm_bwd(a, a, 0, width, w, rstd, a, a, dw, B.WGRAD_OVERWRITE)
    assert (dw == 0).all()


@pytest.mark.parametrize("rows,width", [(1, 64), (300, 768), (5, 2049), (9000, 96)])
def test_quantize_rows(mode, rows, width):
    """(More rows than the context has tokens: weights have as many as they like.)"""
    ctx, dt = mode
    x = normal((rows, width), dt, 18, 3.0)
    x[0] = 0
    qw, q = guarded((rows, width), torch.float8_e4m3fn)
    sw, scale = guarded((rows,), torch.float32)
    ctx.quantize_rows(x, rows, width, q, scale)
    assert untouched(qw, q) and untouched(sw, scale)
    check_q(q, scale, x.double())


def test_captured_and_on_another_stream(mode):
    """Two recorded calls with scratch of their own, replayed on two streams at once and beside an eager call."""
    ctx, dt = mode
    from paper_2605_06665_b200 import binding as B
    T, width = 1501, 768
    w = 1 + normal((width,), torch.float32, 19, 0.2)
    rstd = torch.ones(T, device="cuda")
    sets, graphs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(2):
        dh, r = normal((T, width), dt, 20 + i), normal((T, width), dt, 30 + i)
        want = [torch.empty_like(dh), torch.empty_like(w)]
        ctx.rmsnorm_bwd(dh, r, T, width, w, rstd, None, *want, B.WGRAD_OVERWRITE)
        sets.append((dh, r, want, [torch.zeros_like(dh), torch.zeros_like(w)]))
    torch.cuda.synchronize()
    for (dh, r, _, out), s in zip(sets, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ctx.rmsnorm_bwd(dh, r, T, width, w, rstd, None, *out, B.WGRAD_OVERWRITE)
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        dh, r, want, _ = sets[0]
        mine = [torch.empty_like(dh), torch.empty_like(w)]
        ctx.rmsnorm_bwd(dh, r, T, width, w, rstd, None, *mine, B.WGRAD_OVERWRITE)
        torch.cuda.synchronize()
        assert torch.equal(mine[0], want[0]) and torch.equal(mine[1], want[1])
        for _, _, want, out in sets:
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
            out[0].zero_(), out[1].zero_()
        torch.cuda.synchronize()


def test_more_than_32_bits_of_elements():
    """135000 rows of 16384: the last rows lie 2.2e9 elements behind the first."""
    from paper_2605_06665_b200 import binding as B
    T, width, dt = 135_000, 16384, torch.bfloat16
    ctx = B.Context(B.make_config(64, 64, 1, 1, 1, T, B.BF16, EPS, 1.0))
    x, w = torch.zeros(T, width, dtype=dt, device="cuda"), 1 + normal((width,), torch.float32, 40, 0.2)
    rows = [0, 1, 131071, 131072, 131073, T - 2, T - 1]
    x[rows] = normal((len(rows), width), dt, 41)
    h, rstd = torch.empty_like(x), torch.empty(T, device="cuda")
    ctx.rmsnorm(x, None, T, width, w, EPS, None, rstd, h)
    rr, rs, hh = reference(x[rows], None, w, EPS)
    assert ((h[rows].double() - hh).abs() <= (half_step(dt) + FP32) * hh.abs()).all()
    dw, dw1, dx1 = torch.empty(width, device="cuda"), torch.empty(width, device="cuda"), torch.empty(len(rows), width, dtype=dt, device="cuda")
    ctx.rmsnorm_bwd(x, x, T, width, w, rstd, None, h, dw, B.WGRAD_OVERWRITE)
    ctx.rmsnorm_bwd(x[rows], x[rows], len(rows), width, w, rstd[rows], None, dx1, dw1, B.WGRAD_OVERWRITE)
    assert torch.equal(h[rows], dx1)
    assert ((dw - dw1).abs() <= 16 * 2.0 ** -24 * (x[rows].double() ** 2 * rs[:, None]).sum(0)).all()     # seven terms, in another order
    ctx.check_status()
    ctx.close()


@pytest.mark.parametrize("size,weight", [(2.0 ** -60, 2.0 ** 90), (2.0 ** 40, 2.0 ** -112)])
@pytest.mark.parametrize("width", [768, 33, 2056])
def test_weights_at_the_ends_of_the_range(mode, size, weight, width):
    """1 / |r| and w multiply to more than fp32 holds, or to less than its normal numbers, and h does not."""
    ctx, dt = mode
    T = 9
    x = (normal((T, width), torch.float32, 60) * size).to(dt)
    w = (1 + normal((width,), torch.float32, 61, 0.1)) * weight
    h, q, scale = torch.empty_like(x), torch.empty(T, width, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(T, device="cuda")
    ctx.rmsnorm(x, None, T, width, w, 0.0, None, None, h, q, scale)
    _, _, hh = reference(x, None, w, 0.0)
    assert ((h.double() - hh).abs() <= (half_step(dt) + FP32) * hh.abs() + 2.0 ** -133).all()      # (2^-133: bf16's smallest step)
    check_q(q, scale, hh)
