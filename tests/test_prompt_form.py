"""Which workgroups attention over prompts takes: the rule (host code, compiled here) on both sides of its lines, and that tests/test_gpu_prompt_forms.py reaches
every form."""
import ctypes
import subprocess

import pytest

from paper_2207_01405_amd import build
from test_gpu_prompt_forms import CASES

FORMS = R64X4_K32, R64_K32, R128X2_K64, R128_K64 = range(4)
I64 = ctypes.c_int64


@pytest.fixture(scope="module")
def form(tmp_path_factory):
    d = tmp_path_factory.mktemp("prompt")
    (d / "r.cpp").write_text('#include "prompt_form.hpp"\n'
                             'extern "C" int form(int64_t n_q, int64_t n_seq, int H, int causal) { return ivit::prompt::form_of(n_q, n_seq, H, causal, 256); }\n')
    subprocess.run(["g++", "-std=c++20", "-shared", "-fPIC", "-I", build.CSRC, str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    lib = ctypes.CDLL(str(d / "r.so"))
    lib.form.argtypes = [I64, I64, ctypes.c_int, ctypes.c_int]
    return lib.form


@pytest.mark.parametrize("rows,seqs,heads,causal,want", [
    (1, 1, 1, True, R64X4_K32), (500, 1, 32, True, R64X4_K32), (512, 1, 32, True, R64X4_K32), (513, 1, 32, True, R128X2_K64), (1024, 1, 32, True, R128X2_K64),
    (1025, 1, 32, True, R128_K64), (8192, 1, 32, True, R128_K64), (8 * 197, 8, 6, False, R64X4_K32), (128 * 197, 128, 6, False, R128_K64),
    (200 * 80, 80, 32, True, R64_K32), (201 * 80, 80, 32, True, R128_K64), (128 * 80, 80, 32, False, R64_K32), (129 * 80, 80, 32, False, R128_K64),
    (100 * 4, 4, 33, True, R64_K32), (100 * 4, 4, 32, True, R64X4_K32), (0, 3, 4, True, R64X4_K32)])
def test_form(form, rows, seqs, heads, causal, want):
    assert form(rows, seqs, heads, causal) == want


def test_the_cases_on_a_gpu_reach_every_form(form):
    """Causal ones and others alike, each by the form that it names."""
    for name, lengths, past, heads, causal in CASES:
        assert form(sum(lengths), len(lengths), heads, causal) == FORMS[["64x4", "64", "128x2", "128"].index(name)], (name, lengths, heads, causal)
    assert {(c[0], c[4]) for c in CASES} == {(n, causal) for n in ("64x4", "64", "128x2", "128") for causal in (True, False)}
