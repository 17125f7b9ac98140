"""The float layers around int8 products: what the C entry points and the binding refuse before anything is launched (no GPU)."""
import ctypes as C
import os

import pytest

from paper_2207_01405_amd import binding

FAKE = 0x10000          # a non-NULL, 16-byte aligned address that is never dereferenced
E = binding.ERRORS
F32, F16, BF16, I8 = 0, 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2207_01405_amd import build
        build.build_lib()
    return binding.load()


def norm(lib, x=FAKE, ldx=64, r=None, ldr=64, g=FAKE, eps=1e-6, s=None, lds=64, y=FAKE, ldy=64, sc=FAKE, rows=4, cols=64, t=BF16):
    return lib.ivit_rmsnorm_quant(None, x, ldx, r, ldr, g, eps, s, lds, y, ldy, sc, rows, cols, t)


def test_norm_refusals(lib):
    assert norm(lib, x=None) == E["NULL"] and norm(lib, y=None) == E["NULL"]
    assert norm(lib, rows=-1) == E["SHAPE"] and norm(lib, rows=1 << 31) == E["SHAPE"]
    assert norm(lib, cols=0) == E["SHAPE"] and norm(lib, cols=32769, ldx=32769, ldy=32769) == E["SHAPE"]
    assert norm(lib, ldx=63) == E["SHAPE"] and norm(lib, ldy=63) == E["SHAPE"] and norm(lib, ldx=1 << 31) == E["SHAPE"]
    assert norm(lib, r=FAKE, ldr=63) == E["SHAPE"] and norm(lib, s=FAKE, lds=0) == E["SHAPE"]
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert norm(lib, eps=eps) == E["PARAM"]
    assert norm(lib, t=I8) == E["PARAM"] and norm(lib, t=-1) == E["PARAM"] and norm(lib, t=4) == E["PARAM"]
    assert norm(lib, x=FAKE + 1) == E["ALIGN"] and norm(lib, x=FAKE + 2, t=F32) == E["ALIGN"] and norm(lib, g=FAKE + 2) == E["ALIGN"]
    assert norm(lib, r=FAKE + 1) == E["ALIGN"] and norm(lib, s=FAKE + 1) == E["ALIGN"] and norm(lib, sc=FAKE + 1) == E["ALIGN"]
    assert norm(lib, y=FAKE + 1, sc=None) == E["ALIGN"]
    assert norm(lib, x=None, y=None, sc=None, rows=0) == 0


def dense(lib, x=FAKE, ldx=64, xs=FAKE, one=0, w=FAKE, ws=FAKE, b=None, act=0, r=None, ldr=32, y=FAKE, ldy=32, t=BF16, step=1.0, M=4, N=32, K=64):
    return lib.ivit_linear_scaled(None, x, ldx, xs, one, w, ws, b, act, r, ldr, y, ldy, t, step, M, N, K)


def test_dense_refusals(lib):
    for k in ("x", "xs", "w", "ws", "y"):
        assert dense(lib, **{k: None}) == E["NULL"], k
    assert dense(lib, M=-1) == E["SHAPE"] and dense(lib, M=1 << 31) == E["SHAPE"] and dense(lib, N=0) == E["SHAPE"]
    assert dense(lib, K=0) == E["SHAPE"] and dense(lib, K=24) == E["SHAPE"] and dense(lib, K=65552, ldx=65552) == E["SHAPE"]
    assert dense(lib, N=(1 << 24) + 1, ldy=(1 << 24) + 1) == E["SHAPE"]
    assert dense(lib, ldx=48) == E["SHAPE"] and dense(lib, ldx=72) == E["SHAPE"] and dense(lib, ldx=(1 << 22) + 16) == E["SHAPE"]
    assert dense(lib, ldy=31) == E["SHAPE"] and dense(lib, ldy=1 << 31) == E["SHAPE"] and dense(lib, r=FAKE, ldr=31) == E["SHAPE"]
    assert dense(lib, act=-1) == E["PARAM"] and dense(lib, act=6) == E["PARAM"] and dense(lib, t=-1) == E["PARAM"] and dense(lib, t=4) == E["PARAM"]
    assert dense(lib, t=I8, r=FAKE) == E["PARAM"]
    for step in (0.0, -1.0, float("nan"), float("inf"), 1e-39, 3e38):      # the last: its reciprocal is below the normal numbers
        assert dense(lib, t=I8, step=step) == E["PARAM"], step
    for k in ("x", "w"):
        assert dense(lib, **{k: FAKE + 8}) == E["ALIGN"], k
    for k in ("xs", "ws", "b"):
        assert dense(lib, **{k: FAKE + 2}) == E["ALIGN"], k
    assert dense(lib, y=FAKE + 1) == E["ALIGN"] and dense(lib, y=FAKE + 2, t=F32) == E["ALIGN"] and dense(lib, r=FAKE + 1) == E["ALIGN"]
    assert dense(lib, x=None, xs=None, y=None, M=0) == 0


def gate(lib, x=FAKE, ldx=128, y=FAKE, ldy=64, sc=FAKE, rows=4, cols=64, t=BF16, act=2, gated=1):
    return lib.ivit_gated_quant(None, x, ldx, y, ldy, sc, rows, cols, t, act, gated)


def test_gate_refusals(lib):
    for k in ("x", "y", "sc"):
        assert gate(lib, **{k: None}) == E["NULL"], k
    assert gate(lib, rows=-1) == E["SHAPE"] and gate(lib, rows=1 << 31) == E["SHAPE"] and gate(lib, cols=0) == E["SHAPE"]
    assert gate(lib, cols=32769, ldx=70000, ldy=32769) == E["SHAPE"]
    assert gate(lib, ldx=127) == E["SHAPE"] and gate(lib, ldx=63, gated=0) == E["SHAPE"] and gate(lib, ldy=63) == E["SHAPE"]
    assert gate(lib, t=I8) == E["PARAM"] and gate(lib, act=6) == E["PARAM"] and gate(lib, act=-1) == E["PARAM"]
    assert gate(lib, x=FAKE + 1) == E["ALIGN"] and gate(lib, sc=FAKE + 2) == E["ALIGN"]
    assert gate(lib, x=None, y=None, sc=None, rows=0) == 0


def test_constants_of_the_header_are_those_of_the_binding(tmp_path):
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "c.c"
    names = ["IVIT_ACT_" + n.upper() for n in binding.ACTIVATIONS] + ["IVIT_F32", "IVIT_F16", "IVIT_BF16", "IVIT_I8"]
    src.write_text('#include <stdio.h>\n#include "ivit.h"\nint main(void) { printf("%s", %s); return 0; }\n' % ("%d " * len(names), ", ".join(names)))
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "c")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "c")], check=True, capture_output=True, text=True).stdout.split()]
    assert got == list(binding.ACTIVATIONS.values()) + [F32, F16, BF16, I8]


def test_the_binding_refuses_tensors_that_are_not_as_stated(lib):
    """Host tensors never reach a kernel, nor do wrong types, shapes or strides (here on the host's memory: each is refused)."""
    import torch
    z = torch.zeros
    x, y, s = z(4, 64, dtype=torch.bfloat16), z(4, 64, dtype=torch.int8), z(4)
    bad = [lambda: binding.ivit_rmsnorm_quant(x, None, y, s, 1e-6),                              # on the host
           lambda: binding.ivit_rmsnorm_quant(x.double(), None, y, s, 1e-6),
           lambda: binding.ivit_rmsnorm_quant(x, z(63), y, s, 1e-6),
           lambda: binding.ivit_rmsnorm_quant(x.t(), None, y, s, 1e-6),
           lambda: binding.ivit_rmsnorm_quant(x, None, x.float(), None, 1e-6),
           lambda: binding.ivit_gated_quant(z(4, 64), y, s, gated=True),                          # rows of 128 wanted
           lambda: binding.ivit_gated_quant(z(4, 128), y, s, act="swish"),
           lambda: binding.ivit_gated_quant(z(4, 128), y, s),
           lambda: binding.ivit_linear_scaled(z(4, 64, dtype=torch.int8), s, z(8, 64, dtype=torch.int8), z(8), z(4, 8)),
           lambda: binding.ivit_linear_scaled(z(4, 64, dtype=torch.int8), s, z(8, 48, dtype=torch.int8), z(8), z(4, 8)),
           lambda: binding.ivit_linear_scaled(z(4, 64, dtype=torch.int8), z(3), z(8, 64, dtype=torch.int8), z(8), z(4, 8)),
           lambda: binding.ivit_linear_scaled(z(4, 64, dtype=torch.int8), s, z(8, 128, dtype=torch.int8)[:, :64], z(8), z(4, 8)),
           lambda: binding.ivit_linear_scaled(z(4, 64, dtype=torch.int8), s, z(8, 64, dtype=torch.int8), z(8), z(4, 8, dtype=torch.int8)),
           lambda: binding.ivit_linear_scaled(z(4, 64, dtype=torch.int8), s, z(8, 64, dtype=torch.int8), z(8), z(4, 8), residual=z(4, 8).half())]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was not refused" % i)


def test_no_vector_register_is_spilled(lib):
    """Loads of the Dense kernels are counted by hand (s_waitcnt): a reload from scratch memory between them would wait for all."""
    import re
    from test_spilled_registers import _spills
    of = {name: n for name, n in _spills().items() if re.search(r"\d(gemm_scaled(_rows)?|rmsnorm|gated)_kernel", name)}
    assert len(of) > 40 and not [(name, n) for name, n in of.items() if n]
