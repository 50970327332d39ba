"""What the norm and the dense products refuse, with its code and before anything is launched: the argument checks of the
library linked against stand-ins for the CUDA runtime and the kernels' launchers (each returns 0), so that no GPU is needed."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2605_06665_b200 import binding as B
from paper_2605_06665_b200 import build as builder

ARG, UNSUPPORTED, WORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if not all(shutil.which(t) for t in ("nvcc", "nm", "g++")):
        pytest.skip("needs a compiler")
    builder.build()
    d = tmp_path_factory.mktemp("checks")
    obj = os.path.join(builder.BUILD, "api.o")
    names = [line.split()[-1] for line in subprocess.run(["nm", "-u", obj], check=True, capture_output=True, text=True).stdout.splitlines()]
    stubs = [n for n in names if n.startswith(("_ZN7unipool", "cuda", "__cuda"))]
    assert any("rmsnorm_launch" in n for n in stubs) and any("linear_bwd_launch" in n for n in stubs)
    # (the launchers return 0, the sizes of scratch 64; the current device is the variable fake_device)
    stubs.remove("cudaGetDevice")
    (d / "stubs.s").write_text(".globl fake_device\n.data\nfake_device: .long 0\n.text\n.globl cudaGetDevice\ncudaGetDevice:\n"
                               "  movl fake_device(%rip), %eax\n  movl %eax, (%rdi)\n  xorl %eax, %eax\n  ret\n" + "".join(f".globl {n}\n{n}:\n  movl ${64 if '_scratch' in n else 0}, %eax\n  ret\n" for n in stubs)
                               + '.section .note.GNU-stack,"",@progbits\n')
    so = str(d / "checks.so")
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", obj, str(d / "stubs.s"), "-o", so], check=True)
    L = ctypes.CDLL(so)
    real = B.lib()                                           # its argument types
    for n in B.EXPORTS:
        if hasattr(L, n):
            getattr(L, n).argtypes, getattr(L, n).restype = getattr(real, n).argtypes, getattr(real, n).restype
    return L


@pytest.fixture(scope="module", params=[B.FP32, B.BF16], ids=["fp32", "bf16"])
def ctx(lib, request):
    cfg = B.make_config(64, 64, 4, 1, 1, 100, request.param, 1e-6, 1.0)
    handle, ws = ctypes.c_void_p(), ctypes.create_string_buffer(512)
    base = (ctypes.addressof(ws) + 255) // 256 * 256
    assert lib.unipool_create(ctypes.byref(handle), ctypes.byref(cfg), base, 1 << 40, None) == 0
    handle.bf16, handle.keep = request.param == B.BF16, ws
    return handle


P = 4096                                                     # an aligned address that nothing reads


def call(lib, name, args, **changed):
    args = dict(args, **changed)
    return getattr(lib, "unipool_" + name)(*args.values())


def norm_args(ctx):
    return dict(ctx=ctx, x=P, y=P, T=10, width=768, w=P, eps=1e-6, r=P, rstd=P, h=2 * P, q=None, q_scale=None, stream=None)


def test_norm(lib, ctx):
    a = norm_args(ctx)
    ok = lambda **c: call(lib, "rmsnorm", a, **c)
    assert ok() == 0
    for c in (dict(y=None, r=None, rstd=None), dict(h=None, q=P, q_scale=P), dict(T=0), dict(T=100), dict(width=1),
              dict(width=16384), dict(x=P + 2, h=P + 2), dict(r=P, x=P), dict(eps=0.0)):
        assert ok(**c) == 0, c
    for c in (dict(ctx=None), dict(x=None), dict(w=None), dict(h=None), dict(q=P), dict(q_scale=P), dict(T=-1), dict(T=101),
              dict(eps=-1.0), dict(eps=float("nan")), dict(r=2 * P)):
        assert ok(**c) == ARG and lib.unipool_last_error(), c
    for w in (0, -5, 16385):
        assert ok(width=w) == UNSUPPORTED


def test_norm_backward(lib, ctx):
    a = dict(ctx=ctx, dh=P, r=P, T=10, width=768, w=P, rstd=P, dr=P, dx=P, dw=P, scratch=P, flags=0, stream=None)
    f = lambda **c: call(lib, "rmsnorm_bwd", a, **c)
    for c in ({}, dict(dr=None), dict(dw=None, scratch=None), dict(flags=B.WGRAD_OVERWRITE), dict(T=0, scratch=None)):
        assert f(**c) == 0, c
    for n in ("ctx", "dh", "r", "w", "rstd", "dx"):
        assert f(**{n: None}) == ARG, n
    for c in (dict(T=-1), dict(T=101), dict(flags=1), dict(flags=4)):
        assert f(**c) == ARG, c
    assert f(width=0) == UNSUPPORTED and f(width=16385) == UNSUPPORTED
    assert f(scratch=None) == WORKSPACE and f(scratch=P + 4) == WORKSPACE


def test_quantize_rows(lib, ctx):
    a = dict(ctx=ctx, x=P, rows=1000, width=96, q=P, q_scale=P, stream=None)      # more rows than the context has tokens
    f = lambda **c: call(lib, "quantize_rows", a, **c)
    assert f() == 0 and f(rows=0) == 0
    for n in ("ctx", "x", "q", "q_scale"):
        assert f(**{n: None}) == ARG, n
    assert f(rows=-1) == ARG and f(width=0) == UNSUPPORTED


def linear_args(ctx):
    return dict(ctx=ctx, x=4 * P, T=10, n_in=128, W=P, n_out=192, bias=P, act=1, residual=P, pre=2 * P, y=P, stream=None)


def check_features(f):
    for n in ("n_in", "n_out"):
        for v in (0, -64, 32, 100, 65, (1 << 21) + 64):
            assert f(**{n: v}) == UNSUPPORTED, (n, v)


def test_linear(lib, ctx):
    a = linear_args(ctx)
    f = lambda **c: call(lib, "linear", a, **c)
    for c in ({}, dict(bias=None, residual=None, pre=None, act=0), dict(T=0), dict(T=100), dict(act=3), dict(bias=P + 4), dict(residual=P, y=P), dict(T=0, x=P)):
        assert f(**c) == 0, c
    for n in ("ctx", "x", "W", "y"):
        assert f(**{n: None}) == ARG, n
    for c in (dict(act=-1), dict(act=4), dict(T=-1), dict(T=101), dict(pre=P), dict(x=P), dict(x=2 * P)):   # (x is y, x is pre)
        assert f(**c) == ARG, c
    check_features(f)
    for n in ("x", "W", "residual", "pre", "y"):             # moved by TMA on the tensor-core path
        assert f(**{n: 8 * P + 4}) == (ARG if ctx.bf16 else 0), n


def test_linear_scaled(lib, ctx):
    a = linear_args(ctx)
    a = dict(ctx=ctx, x=4 * P, x_scale=P, T=10, n_in=128, W=P, w_scale=P, **{n: a[n] for n in ("n_out", "bias", "act", "residual", "pre", "y", "stream")})
    f = lambda **c: call(lib, "linear_scaled", a, **c)
    if not ctx.bf16:
        assert f() == UNSUPPORTED
        return
    for c in ({}, dict(bias=None, residual=None, pre=None, act=0), dict(x_scale=P + 4, w_scale=P + 4, bias=P + 4)):
        assert f(**c) == 0, c
    for n in ("ctx", "x", "x_scale", "W", "w_scale", "y"):
        assert f(**{n: None}) == ARG, n
    check_features(f)
    assert f(x=P + 8) == ARG and f(act=9) == ARG


def test_linear_backward(lib, ctx):
    a = dict(ctx=ctx, dy=P, T=10, n_out=192, pre=P, act=2, x=P, n_in=128, W=P, dp=P, dx_residual=P, dx=3 * P, dW=P, dbias=P,
             scratch=P, flags=0, stream=None)
    f = lambda **c: call(lib, "linear_bwd", a, **c)
    for c in ({}, dict(act=0, pre=None, dp=None), dict(dW=None, dbias=None, scratch=None, x=None), dict(dx=None, W=None),
              dict(flags=B.WGRAD_OVERWRITE), dict(T=0, scratch=None), dict(dx_residual=None)):
        assert f(**c) == 0, c
    for c in (dict(ctx=None), dict(dy=None), dict(pre=None), dict(dp=None), dict(x=None), dict(W=None), dict(act=4), dict(T=101),
              dict(dx=None, dW=None, dbias=None), dict(flags=1), dict(flags=8), dict(dx=P), dict(dx=P, x=2 * P), dict(dx=P, dp=2 * P),
              dict(dx=P, x=2 * P, act=0)):
        assert f(**c) == ARG, c
    for c in (dict(dx=P, x=2 * P, dp=2 * P), dict(dx=P, dp=2 * P, dW=None)):   # onto dy or x that no product reads
        assert f(**c) == 0, c
    check_features(f)
    assert f(scratch=None) == WORKSPACE and f(scratch=P + 8) == WORKSPACE
    for n in ("dy", "pre", "dp", "x", "W", "dx_residual", "dx", "dW"):
        assert f(**{n: 8 * P + 4}) == (ARG if ctx.bf16 else 0), n
    assert f(dbias=8 * P + 4) == 0


def test_scratch_sizes_of_nothing(lib, ctx):
    assert lib.unipool_rmsnorm_bwd_scratch(None, 10, 768) == 0 and lib.unipool_rmsnorm_bwd_scratch(ctx, 0, 768) == 0
    assert lib.unipool_linear_bwd_scratch(None, 10, 64, 64) == 0 and lib.unipool_linear_bwd_scratch(ctx, 10, 65, 64) == 0
    # beyond what the calls take
    assert lib.unipool_rmsnorm_bwd_scratch(ctx, 10, 16384) == 64 and lib.unipool_rmsnorm_bwd_scratch(ctx, 10, 16385) == 0
    assert lib.unipool_linear_bwd_scratch(ctx, 10, 64, 1 << 21) == 64 and lib.unipool_linear_bwd_scratch(ctx, 10, 64, (1 << 21) + 64) == 0


def test_another_device_is_current(lib, ctx):
    device = ctypes.c_int.in_dll(lib, "fake_device")
    calls = [("rmsnorm", norm_args(ctx)), ("linear", linear_args(ctx))]
    try:
        device.value = 1
        for name, args in calls:
            assert call(lib, name, args) == ARG and b"device" in lib.unipool_last_error()
        assert lib.unipool_quantize_rows(ctx, P, 10, 64, P, P, None) == ARG
    finally:
        device.value = 0
    for name, args in calls:
        assert call(lib, name, args) == 0


def test_binding_takes_dense_tensors_only():
    torch = pytest.importorskip("torch")
    a = torch.zeros(4, 6)
    assert B._d(a) == a.data_ptr() and B._d(a[1:3]) == a[1:3].data_ptr() and B._d(None) is None
    for t in (a.t(), a[:, :3], a[::2], a[0].expand(4, 6)):
        with pytest.raises(ValueError):
            B._d(t)


def test_no_tokens_need_no_arrays_of_tokens(lib, ctx):
    """What an empty batch hands over: x[:0] has no address.  Weights are checked as ever."""
    norm = dict(norm_args(ctx), T=0, x=None, y=None, r=None, rstd=None, h=None)
    back = dict(ctx=ctx, dh=None, r=None, T=0, width=768, w=P, rstd=None, dr=None, dx=None, dw=P, scratch=None, flags=0, stream=None)
    rows = dict(ctx=ctx, x=None, rows=0, width=96, q=None, q_scale=None, stream=None)
    linear = dict(linear_args(ctx), T=0, x=None, residual=None, pre=None, y=None)
    scaled = dict(ctx=ctx, x=None, x_scale=None, T=0, n_in=128, W=P, w_scale=P, n_out=192, bias=P, act=1, residual=None, pre=None, y=None, stream=None)
    grad = dict(ctx=ctx, dy=None, T=0, n_out=192, pre=None, act=2, x=None, n_in=128, W=P, dp=None, dx_residual=None, dx=None, dW=P, dbias=P,
                scratch=None, flags=B.WGRAD_OVERWRITE, stream=None)
    frozen = dict(grad, dW=None, dbias=None)
    for name, args in (("rmsnorm", norm), ("rmsnorm_bwd", back), ("quantize_rows", rows), ("linear", linear), ("linear_bwd", grad),
                       ("linear_bwd", frozen)) + ((("linear_scaled", scaled),) if ctx.bf16 else ()):
        assert call(lib, name, args) == 0, name
    for name, args, weight in (("rmsnorm", norm, "w"), ("rmsnorm_bwd", back, "w"), ("linear", linear, "W")):
        assert call(lib, name, args, **{weight: None}) == ARG, name
    if ctx.bf16:
        assert call(lib, "linear_scaled", scaled, w_scale=None) == ARG and call(lib, "linear_scaled", scaled, T=-1) == ARG
    for name, args in (("rmsnorm", norm), ("rmsnorm_bwd", back), ("linear", linear), ("linear_bwd", grad)):
        assert call(lib, name, args, T=1) == ARG and call(lib, name, args, T=-1) == ARG, name
    assert call(lib, "quantize_rows", rows, rows=1) == ARG


def test_dp_over_the_residual_of_dx(lib, ctx):
    """The residual is kept in dx, which must not be what dp is formed from."""
    a = dict(ctx=ctx, dy=P, T=10, n_out=128, pre=2 * P, act=2, x=4 * P, n_in=128, W=5 * P, dp=P, dx_residual=P, dx=3 * P, dW=6 * P,
             dbias=P, scratch=P, flags=0, stream=None)
    f = lambda **c: call(lib, "linear_bwd", a, **c)
    for c in ({}, dict(dp=2 * P), dict(dp=2 * P, dx_residual=2 * P), dict(dx=2 * P, dx_residual=3 * P), dict(act=0, dp=None, pre=None),
              dict(dx=2 * P, T=0)):
        assert f(**c) == 0, c
    for c in (dict(dx=2 * P), dict(dx=P, dp=2 * P, dx_residual=2 * P)):
        assert f(**c) == ARG and b"dx_residual" in lib.unipool_last_error(), c
