"""Stacks of pre-normalised blocks, x_{l+1} = x_l + MoE_l(norm(x_l)): values and all gradients against float64 autograd with
the kernels' own routing decisions, and the forms of a pass against one another."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

EPS, ALPHA, C = 1e-6, 1e-2, 1.7


def make(L=3, d=128, f=192, M=8, k=2, T=150, dtype="fp32", seed=0, **kw):
    from paper_2605_06665_b200 import build as builder
    from paper_2605_06665_b200.stack import UniPoolStack
    builder.build()
    st = UniPoolStack(L, d, f, M, k, T, dtype, c=C, alpha=ALPHA, norm=True, **kw)
    g = torch.Generator(device="cpu").manual_seed(seed)
    draw = lambda t, std: t.copy_((torch.randn(t.shape, generator=g) * std).to(t.dtype))
    draw(st.W_gu, 0.08)
    draw(st.W_down, 0.08)
    draw(st.W_r, 0.3)
    draw(st.W_n, 0.2)
    st.W_n += 1.0
    x0, up = torch.randn(T, d, generator=g) * 2.0, torch.randn(T, d, generator=g)
    return st, x0.to(st.tdtype).cuda(), up.to(st.tdtype).cuda()


def layer(st, l, x, P, idx):
    """One block in float64 with the given selection; its scores too."""
    h = x / torch.sqrt((x * x).mean(1, keepdim=True) + st.norm_eps) * P["W_n"][l]
    z = h @ P["W_r"][l].T
    n = z.norm(dim=1, keepdim=True)
    s = st.sigma[l] * C * torch.clamp(z, min=0) / (n + EPS)
    gate = torch.gather(s, 1, idx.long())
    y, b = torch.zeros_like(x), st.base(l)
    for e in range(st.m):
        t, j = torch.nonzero(idx == e, as_tuple=True)
        if len(t):
            gu = h[t] @ P["W_gu"][b + e].T
            a = torch.nn.functional.silu(gu[:, :st.f]) * gu[:, st.f:]
            y = y.index_add(0, t, gate[t, j, None] * (a @ P["W_down"][b + e].T))
    return x + y, s


def params(st):
    return {n: getattr(st, n).double().clone().requires_grad_(True) for n in ("W_n", "W_r", "W_gu", "W_down")}


def close(got, want, tol):
    err, size = (got.double() - want).abs().max().item(), want.abs().max().item()
    assert err <= tol * size, (err, size)


@pytest.mark.parametrize("kw", [{}, dict(deferred_wgrad=True), dict(recompute=True), dict(recompute=True, wgrad_layers=1),
                                dict(private=4, L=2), dict(T=1), dict(T=33, d=192)])
def test_fp32_stack_against_autograd(kw):
    """The whole stack: outputs and every gradient within the fp32 mode's 1e-5 of their largest value (per layer; three layers
    in a row: 3e-5)."""
    st, x0, up = make(**kw)
    dx = st.step(x0, up, accumulate=False).clone()
    x, P = x0.double().requires_grad_(True), params(st)
    y, loss = x, 0.0
    for l in range(st.L):
        y, s = layer(st, l, y, P, st.idx[l])
        g = l // st.Lg
        f = st.fbar[g].double()                             # carries no gradient
        loss = loss + ALPHA * st.m * (f * s.mean(0)).sum() / st.Lg
        close(st.x[l + 1], y, 3e-5)
        # the selection is the scores' own
        top = s.topk(st.k, dim=1).values
        assert (torch.gather(s, 1, st.idx[l].long()) >= top - 1e-4).all()
    ((up.double() * y).sum() + loss).backward()
    close(st.loss.sum(), loss.detach(), 1e-5)
    close(dx, x.grad, 3e-5)
    close(st.dW_n, P["W_n"].grad, 3e-5)
    close(st.dW_r, P["W_r"].grad, 3e-5)
    close(st.dW_gu, P["W_gu"].grad, 3e-5)
    close(st.dW_down, P["W_down"].grad, 3e-5)
    st.ctx.check_status()
    st.close()


def test_bf16_layer_against_autograd():
    """One bf16 layer, T beyond one tile: within the bf16 mode's 1e-2 of each array's largest value."""
    st, x0, up = make(L=1, d=256, f=320, M=12, T=700, dtype="bf16")
    dx = st.step(x0, up, accumulate=False).clone()
    x, P = x0.double().requires_grad_(True), params(st)
    y, s = layer(st, 0, x, P, st.idx[0])
    loss = ALPHA * st.m * (st.fbar[0].double() * s.mean(0)).sum()
    ((up.double() * y).sum() + loss).backward()
    close(st.x[1], y, 1e-2)
    close(dx, x.grad, 1e-2)
    for n in ("W_n", "W_r", "W_gu", "W_down"):
        close(getattr(st, "d" + n), P[n].grad, 1e-2)
    st.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_forms_of_a_pass_agree(dtype):
    """The native calls against the layers one by one, a recorded step, and activation recompute: the same bits.  (bf16: the
    layers one by one pad their groups in the weight gradient, which adds zeros.)"""
    st, x0, up = make(dtype=dtype, T=300)
    names = ("x", "dW_n", "dW_r", "dW_gu", "dW_down", "dsigma", "rstd")
    # (the routers' gradients are summed by atomics: to the last bits)
    exact = [n for n in names if n not in ("dW_r", "dsigma")]

    def results(s, dx):
        return {n: getattr(s, n).clone() for n in names} | {"dx": dx.clone()}

    want = results(st, st.step(x0, up, accumulate=False))

    def same(got):
        for n in exact + ["dx"]:
            assert torch.equal(got[n], want[n]), n
        for n in ("dW_r", "dsigma"):
            assert (got[n] - want[n]).abs().max() <= 1e-5 * want[n].abs().max(), n

    same(results(st, st.step(x0, up, accumulate=False)))
    st.W_n = list(st.W_n)                                   # not one array: the layers are issued one by one
    st.zero_router_grad()
    st.forward(x0)
    st.aux_loss()
    same(results(st, st.backward(up, accumulate=False)))
    st.W_n = torch.stack(st.W_n)
    graph = st.capture_step(x0, up, accumulate=False)
    for n in ("x", "dW_n", "dW_gu", "rstd"):
        getattr(st, n)[:].zero_()
    st.zero_router_grad()
    graph.replay()
    torch.cuda.synchronize()
    same(results(st, st.dx[st.L % 2]))
    re, _, _ = make(dtype=dtype, T=300, recompute=True, wgrad_layers=1)
    dx = re.step(x0, up, accumulate=False)
    assert torch.equal(re.x, want["x"]) and torch.equal(dx, want["dx"]) and torch.equal(re.dW_n, want["dW_n"])
    for s in (st, re):
        s.ctx.check_status()
        s.close()


def test_gradients_accumulate_over_microbatches():
    st, x0, up = make(T=64)
    one, x1, up1 = make(T=64, seed=5)
    for n in ("W_n", "W_r", "W_gu", "W_down"):
        getattr(one, n).copy_(getattr(st, n))
    total = []
    for a, b in ((x0, up), (x1, up1)):
        one.zero_grad()
        one.forward(a)
        one.aux_loss(fbar_prev=torch.full((one.m,), 1.0 / one.m, device="cuda") if not total else fbar)
        fbar = one.fbar.clone()
        one.backward(b)
        total.append(one.dW_n.clone())
    st.accumulate_microbatches([(x0, up), (x1, up1)], fbar0=torch.full((st.m,), 1.0 / st.m, device="cuda"))
    want = total[0] + total[1]
    assert (st.dW_n - want).abs().max() <= 1e-5 * want.abs().max()
    st.close()
    one.close()


def test_without_norms_nothing_of_them_is_there():
    from paper_2605_06665_b200.stack import UniPoolStack
    st = UniPoolStack(1, 64, 64, 4, 1, 8, "fp32")
    assert st.W_n is None and st.h is None and st.dW_n is None
    st.close()
    st, x0, _ = make(T=8)
    st.W_n = None
    with pytest.raises(ValueError):
        st.forward(x0)
    st.close()
