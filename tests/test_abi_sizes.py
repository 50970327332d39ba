"""Programs built with the header as it was before the stack had norms and before norms and dense products had phases: the
library reads no more of their struct and writes no more of their arrays than they have.  The library's host code linked against stand-ins
for the CUDA runtime and the kernels' launchers (each returns 0), so that no GPU is needed."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2605_06665_b200 import binding as B
from paper_2605_06665_b200 import build as builder

ARG = -1
OLD_PHASES = 18
P = 4096                                                     # an aligned address that nothing reads


class OldStack(ctypes.Structure):
    """The struct as it was."""
    _fields_ = [f for f in B.Stack._fields_ if f[0] not in ("W_n", "dW_n", "h", "dh", "rstd", "norm_scratch", "norm_eps")]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if not all(shutil.which(t) for t in ("nvcc", "nm", "g++")):
        pytest.skip("needs a compiler")
    builder.build()
    d = tmp_path_factory.mktemp("sizes")
    objs = [os.path.join(builder.BUILD, n) for n in ("api.o", "stack.o")]
    names = {line.split()[-1] for o in objs for line in subprocess.run(["nm", "-u", o], check=True, capture_output=True, text=True).stdout.splitlines()}
    stubs = sorted(n for n in names if n.startswith(("_ZN7unipool", "cuda", "__cuda")))
    stubs = [n for n in stubs if n not in subprocess.run(["nm", "--defined-only", *objs], check=True, capture_output=True, text=True).stdout]
    (d / "stubs.s").write_text(".text\n" + "".join(f".globl {n}\n{n}:\n  xorl %eax, %eax\n  ret\n" for n in stubs)
                               + '.section .note.GNU-stack,"",@progbits\n')
    so = str(d / "sizes.so")
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", *objs, str(d / "stubs.s"), "-o", so], check=True)
    return ctypes.CDLL(so)


@pytest.fixture(scope="module")
def ctx(lib):
    cfg = B.make_config(64, 64, 4, 1, 1, 100, B.FP32, 1e-6, 1.0)
    handle, ws = ctypes.c_void_p(), ctypes.create_string_buffer(512)
    lib.unipool_create.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    base = (ctypes.addressof(ws) + 255) // 256 * 256
    assert lib.unipool_create(ctypes.byref(handle), ctypes.byref(cfg), base, 1 << 40, None) == 0
    handle.keep = ws
    return handle


def filled(cls):
    s, sigma = cls(1, 1, 4, 0, 1), (ctypes.c_float * 1)(1.0)
    for n, t in cls._fields_:
        if t is ctypes.c_void_p:
            setattr(s, n, P)
    s.sigma, s.keep = ctypes.addressof(sigma), sigma
    return s


def test_old_struct_with_anything_behind_it(lib, ctx):
    """What lies behind: a weight of the norm without the arrays that belong to it, which would be refused."""
    size = ctypes.sizeof(OldStack)
    assert size == B.Stack.W_n.offset
    memory = (ctypes.c_uint64 * 64)()
    old = filled(OldStack)
    ctypes.memmove(memory, ctypes.byref(old), size)
    memory[size // 8] = P
    for name, args in (("forward", ()), ("aux_loss", None), ("backward", (0,))):
        f = getattr(lib, "unipool_stack_" + name)
        if args is None:
            assert f(ctx, memory, 10, ctypes.c_float(0.01), None, None) == 0
        else:
            assert f(ctx, memory, 10, *args, None) == 0, name
            g = getattr(lib, f"unipool_stack_{name}_sized")
            g.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t] + [ctypes.c_int32] * (1 + len(args)) + [ctypes.c_void_p]
            assert g(ctx, memory, size, 10, *args, None) == 0
            assert g(ctx, memory, ctypes.sizeof(B.Stack), 10, *args, None) == ARG               # told of the norm: it lacks h and rstd
            assert g(ctx, memory, size - 8, 10, *args, None) == ARG and g(ctx, memory, ctypes.sizeof(B.Stack) + 8, 10, *args, None) == ARG
            assert g(ctx, ctypes.byref(filled(B.Stack)), ctypes.sizeof(B.Stack), 10, *args, None) == 0


def test_profile_of_old_arrays(lib, ctx):
    ms, launches = (ctypes.c_double * 32)(*[7.0] * 32), (ctypes.c_int64 * 32)(*[7] * 32)
    assert lib.unipool_profile_read(ctx, ms, launches) == 0
    assert list(ms) == [0.0] * OLD_PHASES + [7.0] * (32 - OLD_PHASES) and list(launches) == [0] * OLD_PHASES + [7] * (32 - OLD_PHASES)
    assert lib.unipool_profile_read_n(ctx, len(B.PHASES), ms, launches) == 0
    assert list(ms) == [0.0] * len(B.PHASES) + [7.0] * (32 - len(B.PHASES))
    assert lib.unipool_profile_read_n(ctx, -1, ms, launches) == ARG


def test_programs_built_with_the_header_say_what_they_know(tmp_path):
    """As C and as C++: the calls' names are those of before, the symbols those with a size."""
    if not (shutil.which("gcc") and shutil.which("g++")):
        pytest.skip("needs a compiler")
    text = """#include "unipool.h"
int run(unipool_ctx* c, unipool_stack* s, float* w) {
  double ms[UNIPOOL_N_PHASES]; int64_t n[UNIPOOL_N_PHASES];
  s->W_n = w;
  if (unipool_stack_forward(c, s, 10, 0) != UNIPOOL_OK || unipool_stack_backward(c, s, 10, UNIPOOL_STACK_NO_AUX, 0) != UNIPOOL_OK) return 1;
  return unipool_profile_read(c, ms, n);
}
"""
    for compiler, name in (("gcc", "a.c"), ("g++", "a.cc")):
        src, obj = tmp_path / name, str(tmp_path / (name + ".o"))
        src.write_text(text)
        subprocess.run([compiler, "-Wall", "-Werror", "-I", builder.INCLUDE, "-c", str(src), "-o", obj], check=True)
        names = subprocess.run(["nm", "-u", obj], check=True, capture_output=True, text=True).stdout.split()
        assert {"unipool_stack_forward_sized", "unipool_stack_backward_sized", "unipool_profile_read_n"} <= set(names)
        assert "unipool_stack_forward" not in names and "unipool_profile_read" not in names
