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
