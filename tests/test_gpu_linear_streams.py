"""Dense products of few tokens on several streams at once, alone and recorded: their clusters share SMs, tensor memory and each
other's way, and give the bits that they give one after the other."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# (tokens, inputs, outputs): clusters of eight, four, two and single CTAs; with little and with much shared memory
SHAPES = [(1, 768, 2048), (8, 256, 7680), (1, 64, 64), (5, 2048, 768), (16, 512, 4096), (40, 256, 2048), (128, 1024, 512), (17, 4096, 1536)]


@pytest.fixture(scope="module")
def ctx():
    from paper_2605_06665_b200 import binding as B
    from paper_2605_06665_b200 import build as builder
    builder.build()
    c = B.Context(B.make_config(64, 64, 1, 1, 1, 4096, B.BF16, 1e-6, 1.0))
    yield c
    c.check_status()
    c.close()


def calls(ctx, seed):
    g = torch.Generator(device="cpu").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g)
    made = []
    for T, n, m in SHAPES:
        x, W, y = normal(T, n).bfloat16().cuda(), (normal(m, n) * n ** -0.5).bfloat16().cuda(), torch.zeros(T, m, dtype=torch.bfloat16, device="cuda")
        dx = torch.zeros_like(x)

        def call(x=x, W=W, y=y, dx=dx, T=T, n=n, m=m):
            ctx.linear(x, T, n, W, m, None, 0, None, None, y)
            ctx.linear_bwd(y, T, m, None, 0, None, n, W, None, x, dx, None, None)

        made.append((call, y, dx, (x, W)))
    return made


@pytest.mark.parametrize("recorded", [False, True])
def test_many_streams(ctx, recorded):
    n_streams = 6
    sets = [calls(ctx, 10 * i) for i in range(n_streams)]
    want = []
    for s in sets:
        for call, *_ in s:
            call()
        torch.cuda.synchronize()
        want.append([(y.clone(), dx.clone()) for _, y, dx, _ in s])
    streams = [torch.cuda.Stream() for _ in sets]
    runs = [lambda s=s: [call() for call, *_ in s] for s in sets]
    if recorded:
        graphs = []
        for run, stream in zip(runs, streams):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                run()
            graphs.append(g)
        runs = [g.replay for g in graphs]
    for _ in range(20):
        for s in sets:
            for _, y, dx, _ in s:
                y.zero_(), dx.zero_()
        torch.cuda.synchronize()
        for run, stream in zip(runs, streams):
            with torch.cuda.stream(stream):
                run()
        torch.cuda.synchronize()
        for s, w in zip(sets, want):
            for (_, y, dx, _), (y0, dx0) in zip(s, w):
                assert torch.equal(y, y0) and torch.equal(dx, dx0)


def test_products_beside_a_stack_on_another_stream(ctx):
    """Products of one context while a stack of pre-normalised blocks (another context, kernels that take whole SMs) runs its steps; and
    products and norms of that stack's own context."""
    from paper_2605_06665_b200.stack import UniPoolStack
    T, d = 700, 256
    st = UniPoolStack(3, d, 320, 12, 2, T, "bf16", c=1.7, norm=True)
    g = torch.Generator(device="cpu").manual_seed(3)
    draw = lambda t, std: t.copy_((torch.randn(t.shape, generator=g) * std).to(t.dtype))
    draw(st.W_gu, 0.08), draw(st.W_down, 0.08), draw(st.W_r, 0.3)
    x0, up = (torch.randn(T, d, generator=g).bfloat16().cuda() for _ in range(2))
    names = ("x", "dW_n", "dW_gu", "dW_down", "rstd")
    st.step(x0, up, accumulate=False)
    want = [getattr(st, n).clone() for n in names]
    own, w = calls(ctx, 77), torch.ones(d, device="cuda")
    of_stack = calls(st.ctx, 78)[:2]
    h, h0 = torch.empty_like(x0), torch.empty_like(x0)
    st.ctx.rmsnorm(x0, None, T, d, w, 1e-6, None, None, h0)
    for c, *_ in own + of_stack:
        c()
    torch.cuda.synchronize()
    results = [(y.clone(), dx.clone()) for _, y, dx, _ in own + of_stack]
    a, b, c = (torch.cuda.Stream() for _ in range(3))
    for _ in range(10):
        for n in names:
            getattr(st, n)[:].zero_()
        for _, y, dx, _ in own + of_stack:
            y.zero_(), dx.zero_()
        h.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(a):
            st.step(x0, up, accumulate=False)
        with torch.cuda.stream(b):
            for call, *_ in own:
                call()
        with torch.cuda.stream(c):
            st.ctx.rmsnorm(x0, None, T, d, w, 1e-6, None, None, h)
            for call, *_ in of_stack:
                call()
        torch.cuda.synchronize()
        assert all(torch.equal(getattr(st, n), v) for n, v in zip(names, want)) and torch.equal(h, h0)
        for (_, y, dx, _), (y0, dx0) in zip(own + of_stack, results):
            assert torch.equal(y, y0) and torch.equal(dx, dx0)
    st.ctx.check_status()
    st.close()
