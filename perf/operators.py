"""What is measured of the operators around the MoE layer: the RMS norm with the residual's addition (forward, backward,
output in 8 bits with scales) and the matrix product with bias, activation and residual in its epilogue (forward, backward,
8-bit operands).

A case is a dict of plain values:
  op        "norm", "norm_bwd", "linear", "linear_bwd"
  T         tokens
  n         width of the norm; input features of the product
  m         output features of the product (0 for the norm)
  dtype     "bf16" or "fp32": activations and weights (the norm's weight, biases and weight gradients are fp32)
  residual  norm: y is added to x and the sum stored; norm_bwd: the sum's own gradient is added; linear: the residual's
            addition; linear_bwd: a gradient is added to dx
  q8        norm: the output also in e4m3 with a scale per token; linear: e4m3 operands with a scale per token and per
            output feature
  act       "none", "relu", "silu" or "gelu" (tanh form)
  bias      the product has a bias
  pre       linear: the value before the activation is stored too, as a training step does
  frozen    linear_bwd: the weights are frozen, only dx is asked for
"""
import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0
SMALLEST_SCALE = 2.0 ** -126


def _norm(name, op, T, n, dtype="bf16", residual=True, q8=False):
    case = dict(op=op, T=T, n=n, m=0, dtype=dtype, residual=residual, q8=q8, act="none", bias=False, pre=False, frozen=False)
    return dict(case, name=name) if name else case


def _linear(name, op, T, n, m, dtype="bf16", residual=False, q8=False, act="none", bias=True, pre=False, frozen=False):
    case = dict(op=op, T=T, n=n, m=m, dtype=dtype, residual=residual, q8=q8, act=act, bias=bias, pre=pre, frozen=frozen)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one token of a decoding loop through a 182M-shaped block: latency
        _norm("norm_one_token", "norm", 1, 768),
        # the norm in front of the MoE layer of a 182M-shaped training step
        _norm("norm_182m", "norm", 16384, 768),
        # the largest batch and width, 8 bits for the product behind it beside the bf16 output
        _norm("norm_978m_q8", "norm", 32768, 1536, q8=True),
        # its backward pass in the 182M-shaped training step, the residual's gradient added
        _norm("norm_bwd_182m", "norm_bwd", 16384, 768),
        # fp32 mode, a ragged batch of an odd width: rows that 16-byte accesses do not fit
        _norm("norm_bwd_fp32_odd", "norm_bwd", 1501, 1001, dtype="fp32"),
        # a few sequences of a decoding loop: the weights' bytes
        _linear("linear_decode", "linear", 5, 2048, 768, residual=True),
        # the up-projection of a dense layer in a training step: gelu, and the value before it kept for backward
        _linear("linear_182m_up", "linear", 16384, 768, 2048, act="gelu", pre=True),
        # the down-projection onto the residual stream, the largest sizes
        _linear("linear_978m_down", "linear", 32768, 4096, 1536, residual=True),
        # an evaluation in 8 bits, a ragged batch
        _linear("linear_978m_q8", "linear", 9001, 1536, 4096, q8=True, act="silu"),
        # fp32 mode at its smallest configuration
        _linear("linear_fp32", "linear", 512, 256, 512, dtype="fp32", act="silu", residual=True),
        # backward of a projection in a training step: dx, dW, dbias
        _linear("linear_bwd_182m", "linear_bwd", 16384, 768, 2048, act="relu", residual=True),
        # backward of a ragged batch through a frozen projection
        _linear("linear_bwd_frozen", "linear_bwd", 1501, 1536, 4096, act="gelu", bias=False, frozen=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges: norms of 1 to 32768 tokens and 64 to 4096 columns, odd widths among them;
    products of 1 to 32768 tokens with features in multiples of 64."""
    while True:
        op = rng.choice(["norm", "norm", "norm_bwd", "linear", "linear", "linear", "linear_bwd", "linear_bwd"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        T = _log_int(rng, 1, 32768)
        residual = rng.choice([True, False])
        if op in ("norm", "norm_bwd"):
            n = rng.choice([64 * rng.randint(1, 64), _log_int(rng, 64, 4096)])
            c = _norm(None, op, T, n, dtype, residual, q8=op == "norm" and rng.choice([True, False]))
        else:
            n, m = 64 * _log_int(rng, 2, 64), 64 * _log_int(rng, 2, 64)
            if op == "linear":
                q8 = dtype == "bf16" and rng.choice([True, False])
                act = rng.choice(["none", "relu", "silu", "gelu"])
                c = _linear(None, op, T, n, m, dtype, residual, q8, act, rng.choice([True, False]), rng.choice([True, False]))
            else:
                # the weight gradient is fp32 and a product of dp rounded to the activations' type: exact with no
                # activation and with relu; in bf16 the weights are frozen where it is one of the other two
                act = rng.choice(["none", "relu", "silu", "gelu"])
                frozen = dtype == "bf16" and act in ("silu", "gelu")
                c = _linear(None, op, T, n, m, dtype, residual, False, act, not frozen, False, frozen)
        w = work(c)
        if w["bytes"] <= 5.2e8 and w["flops"] <= (4e10 if dtype == "fp32" else 4.1e11):
            return c


def work(case):
    """Each input read once and each output written once; two operations for each product's term."""
    T, n, m = case["T"], case["n"], case["m"]
    b = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "norm":
        streams = 4 if case["residual"] else 2             # x, h, and y, r
        q = T * n + 4 * T if case["q8"] else 0
        return {"bytes": streams * T * n * b + q + 4 * T + 4 * n, "flops": 6 * T * n}
    if case["op"] == "norm_bwd":
        streams = 4 if case["residual"] else 3             # dh, r, dx, and the sum's own gradient
        return {"bytes": streams * T * n * b + 4 * T + 8 * n, "flops": 10 * T * n}
    bias = 4 * m if case["bias"] else 0
    if case["op"] == "linear":
        operands = (T * n + m * n) * (1 if case["q8"] else b) + (4 * (T + m) if case["q8"] else 0)
        return {"bytes": operands + bias + T * m * b * (1 + case["residual"] + case["pre"]), "flops": 2 * T * n * m}
    inputs = (T * m * (1 if case["act"] == "none" else 2) + n * m + T * n * (1 + case["residual"])) * b
    if case["frozen"]:
        return {"bytes": inputs, "flops": 2 * T * n * m}
    return {"bytes": inputs + T * n * b + 4 * n * m + bias, "flops": 4 * T * n * m}


# ------------------------------------------------------------------ inputs
def _quantised(v):
    """Rows in e4m3 and their scales, as a checkpoint or the operator in front hands them over."""
    scale = (v.abs().amax(1) / E4M3_MAX).clamp(min=SMALLEST_SCALE)
    return (v / scale[:, None]).to(torch.float8_e4m3fn), scale


def _data(case, seed):
    """The inputs of a case.  A residual stream of unit deviation whose channels differ in scale, as trained ones do; weights
    and gradients of the size that they have in training."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, n, m = case["T"], case["n"], case["m"]
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16

    def normal(*shape, std=1.0):
        return torch.empty(*shape, device="cuda").normal_(0.0, std, generator=g)

    d = {}
    if case["op"] in ("norm", "norm_bwd"):
        channels = torch.exp(normal(n, std=0.5))
        d["w"] = 1.0 + normal(n, std=0.1)
        if case["op"] == "norm":
            d["x"] = (normal(T, n) * channels).to(dt)
            d["y"] = (normal(T, n, std=0.3) * channels).to(dt) if case["residual"] else None
        else:
            d["r"] = (normal(T, n) * channels).to(dt)
            d["rstd"] = torch.rsqrt(d["r"].float().square().mean(1) + EPS)
            d["dh"] = normal(T, n, std=0.1).to(dt)
            d["dr"] = normal(T, n, std=0.1).to(dt) if case["residual"] else None
        return d
    d["bias"] = normal(m, std=0.1) if case["bias"] else None
    if case["q8"]:
        d["x"], d["x_scale"] = _quantised(normal(T, n))
        d["W"], d["w_scale"] = _quantised(normal(m, n, std=n ** -0.5))
    else:
        d["x"], d["W"] = normal(T, n).to(dt), normal(m, n, std=n ** -0.5).to(dt)
    if case["op"] == "linear":
        d["res"] = normal(T, m).to(dt) if case["residual"] else None
        return d
    d["dy"] = normal(T, m, std=0.1).to(dt)
    d["p"] = normal(T, m).to(dt) if case["act"] != "none" else None
    d["dx_res"] = normal(T, n, std=0.1).to(dt) if case["residual"] else None
    return d


def prepare(case, seed):
    """The inputs, and the buffers that a program allocates once and hands to every call; with the framework also its
    context, which a program keeps for its lifetime."""
    state = dict(case=case, **_data(case, seed))
    T, n, m = case["T"], case["n"], case["m"]
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16

    def empty(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if case["op"] == "norm":
        state["r_out"] = empty(T, n) if case["residual"] else None
        state["rstd_out"], state["h"] = empty(T, dtype=torch.float32), empty(T, n)
        state["q"] = empty(T, n, dtype=torch.float8_e4m3fn) if case["q8"] else None
        state["q_scale"] = empty(T, dtype=torch.float32) if case["q8"] else None
    elif case["op"] == "norm_bwd":
        state["dx"], state["dw"] = empty(T, n), empty(n, dtype=torch.float32)
    elif case["op"] == "linear":
        state["y"], state["pre"] = empty(T, m), empty(T, m) if case["pre"] else None
    else:
        state["dp"] = empty(T, m) if case["act"] != "none" else None
        state["dx"] = empty(T, n)
        state["dW"] = None if case["frozen"] else empty(m, n, dtype=torch.float32)
        state["db"] = empty(m, dtype=torch.float32) if case["bias"] else None
    if own:
        from paper_2605_06665_b200 import binding
        dtype = binding.FP32 if case["dtype"] == "fp32" else binding.BF16
        state["ctx"] = binding.Context(binding.make_config(64, 64, 1, 1, 1, T, dtype, EPS, 1.0))
    return state


# ------------------------------------------------------------------ one pass
def _act(p, act):
    if act == "relu":
        return p.clamp(min=0.0)
    if act == "silu":
        return p / (1.0 + torch.exp(-p))
    if act == "gelu":
        return 0.5 * p * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (p + 0.044715 * p * p * p)))
    return p


def _act_grad(p, act):
    if act == "relu":
        return (p > 0.0).to(p.dtype)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-p))
        return s * (1.0 + p * (1.0 - s))
    a = math.sqrt(2.0 / math.pi)
    t = torch.tanh(a * (p + 0.044715 * p * p * p))
    return 0.5 * (1.0 + t) + 0.5 * p * (1.0 - t * t) * a * (1.0 + 3.0 * 0.044715 * p * p)


def _plain(s):
    case = s["case"]
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    if case["op"] == "norm":
        r = s["x"].float()
        if s["y"] is not None:
            r = r + s["y"].float()
        rstd = 1.0 / torch.sqrt((r * r).mean(1) + EPS)
        h = r * rstd[:, None] * s["w"]
        out = dict(h=h.to(dt), rstd=rstd)
        if s["y"] is not None:
            out["r"] = r.to(dt)
        if case["q8"]:
            out["q"], out["q_scale"] = _quantised(h)
        return out
    if case["op"] == "norm_bwd":
        dh, rstd = s["dh"].float(), s["rstd"][:, None]
        xhat = s["r"].float() * rstd
        g = dh * s["w"]
        dx = rstd * (g - xhat * (g * xhat).mean(1, keepdim=True))
        if s["dr"] is not None:
            dx = dx + s["dr"].float()
        return dict(dx=dx.to(dt), dw=(dh * xhat).sum(0))
    if case["op"] == "linear":
        p = s["x"].float() @ s["W"].float().T
        if case["q8"]:
            p = p * s["x_scale"][:, None] * s["w_scale"]
        if s["bias"] is not None:
            p = p + s["bias"]
        y = _act(p, case["act"])
        if s["res"] is not None:
            y = y + s["res"].float()
        return dict(y=y.to(dt), pre=p.to(dt)) if case["pre"] else dict(y=y.to(dt))
    dp = s["dy"].float()
    if s["p"] is not None:
        dp = dp * _act_grad(s["p"].float(), case["act"])
    dx = dp @ s["W"].float()
    if s["dx_res"] is not None:
        dx = dx + s["dx_res"].float()
    out = dict(dx=dx.to(dt))
    if not case["frozen"]:
        out["dW"] = dp.T @ s["x"].float()
    if case["bias"]:
        out["db"] = dp.sum(0)
    return out


def _own(s):
    from paper_2605_06665_b200 import binding
    case, ctx = s["case"], s["ctx"]
    T, n, m, act = case["T"], case["n"], case["m"], binding.ACTIVATIONS[case["act"]]
    if case["op"] == "norm":
        ctx.rmsnorm(s["x"], s["y"], T, n, s["w"], EPS, s["r_out"], s["rstd_out"], s["h"], s["q"], s["q_scale"])
        out = dict(h=s["h"], rstd=s["rstd_out"])
        if s["y"] is not None:
            out["r"] = s["r_out"]
        if case["q8"]:
            out.update(q=s["q"], q_scale=s["q_scale"])
        return out
    if case["op"] == "norm_bwd":
        ctx.rmsnorm_bwd(s["dh"], s["r"], T, n, s["w"], s["rstd"], s["dr"], s["dx"], s["dw"], binding.WGRAD_OVERWRITE)
        return dict(dx=s["dx"], dw=s["dw"])
    if case["op"] == "linear":
        if case["q8"]:
            ctx.linear_scaled(s["x"], s["x_scale"], T, n, s["W"], s["w_scale"], m, s["bias"], act, s["res"], s["pre"], s["y"])
        else:
            ctx.linear(s["x"], T, n, s["W"], m, s["bias"], act, s["res"], s["pre"], s["y"])
        return dict(y=s["y"], pre=s["pre"]) if case["pre"] else dict(y=s["y"])
    ctx.linear_bwd(s["dy"], T, m, s["p"], act, s["x"], n, s["W"], s["dp"], s["dx_res"], s["dx"], s["dW"], s["db"],
                   binding.WGRAD_OVERWRITE)
    out = dict(dx=s["dx"])
    if not case["frozen"]:
        out["dW"] = s["dW"]
    if case["bias"]:
        out["db"] = s["db"]
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The definitions, element by element in float64; 8-bit outputs as the values that are rounded to them."""
    d = {k: None if v is None else v.double() for k, v in _data(case, seed).items()}
    n, act = case["n"], case["act"]
    if case["op"] == "norm":
        r = d["x"] if d["y"] is None else d["x"] + d["y"]
        rstd = (torch.linalg.vector_norm(r, dim=1) ** 2 / n + EPS) ** -0.5
        h = torch.einsum("tj,t,j->tj", r, rstd, d["w"])
        out = dict(h=h, rstd=rstd)
        if d["y"] is not None:
            out["r"] = r
        if case["q8"]:
            out["q_scale"] = torch.clamp(torch.linalg.vector_norm(h, ord=math.inf, dim=1) / E4M3_MAX, min=SMALLEST_SCALE)
            out["q"] = h / out["q_scale"].unsqueeze(1)
        return out
    if case["op"] == "norm_bwd":
        # the derivative of h = w r / sqrt(mean r^2 + eps), with 1 / sqrt(..) as it was saved
        u = d["rstd"].unsqueeze(1)
        dot = torch.einsum("tj,tj,j->t", d["dh"], d["r"], d["w"]).unsqueeze(1)
        dx = d["w"] * d["dh"] * u - d["r"] * dot * u ** 3 / n
        return dict(dx=dx if d["dr"] is None else dx + d["dr"], dw=torch.einsum("tj,tj,t->j", d["dh"], d["r"], d["rstd"]))
    sig = torch.sigmoid
    k = 2.0 * math.sqrt(2.0 / math.pi)
    if case["op"] == "linear":
        x, W = d["x"], d["W"]
        if case["q8"]:
            x, W = x * d["x_scale"].unsqueeze(1), W * d["w_scale"].unsqueeze(1)
        p = torch.einsum("ti,oi->to", x, W)
        if d["bias"] is not None:
            p += d["bias"]
        y = {"none": lambda: p, "relu": lambda: torch.where(p > 0, p, 0.0), "silu": lambda: p * sig(p),
             "gelu": lambda: p * sig(k * (p + 0.044715 * p ** 3))}[act]()
        if d["res"] is not None:
            y = y + d["res"]
        return dict(y=y, pre=p) if case["pre"] else dict(y=y)
    dp, p = d["dy"], d["p"]
    if act == "relu":
        dp = torch.where(p > 0, dp, 0.0)
    elif act == "silu":
        dp = dp * (sig(p) + p * sig(p) * sig(-p))
    elif act == "gelu":
        v = k * (p + 0.044715 * p ** 3)
        dp = dp * (sig(v) + p * sig(v) * sig(-v) * k * (1.0 + 0.134145 * p ** 2))
    dx = torch.einsum("to,oi->ti", dp, d["W"])
    out = dict(dx=dx if d["dx_res"] is None else dx + d["dx_res"])
    if not case["frozen"]:
        out["dW"] = torch.einsum("to,ti->oi", dp, d["x"])
    if case["bias"]:
        out["db"] = dp.sum(0)
    return out
