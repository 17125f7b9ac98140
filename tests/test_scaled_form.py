"""Which form of the Dense layer with real scales a shape takes: the rule (host code, compiled here) on both sides of its lines."""
import ctypes
import subprocess

import pytest

from paper_2207_01405_amd import build

ROWS, T64, T128X64, T128X8, T256X128, T256, T128 = range(7)


@pytest.fixture(scope="module")
def form(tmp_path_factory):
    d = tmp_path_factory.mktemp("form")
    (d / "r.cpp").write_text('#include "scaled_form.hpp"\n'
                             'extern "C" int form(int64_t M, int64_t N, int64_t K) { return ivit::scaled::form_of(M, N, K, 256); }\n')
    subprocess.run(["g++", "-std=c++20", "-shared", "-fPIC", "-I", build.CSRC, str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    lib = ctypes.CDLL(str(d / "r.so"))
    lib.form.argtypes = [ctypes.c_int64] * 3
    return lib.form


@pytest.mark.parametrize("M,N,K,want", [
    (1, 4096, 4096, ROWS), (32, 32000, 4096, ROWS), (33, 16384, 4096, T64), (33, 16448, 4096, T128X8), (128, 4096, 4096, ROWS), (129, 4096, 4096, T64), (394, 384, 384, ROWS),
    (1024, 1024, 1024, T64), (512, 4096, 4096, T128X64), (1024, 4096, 4096, T128X8), (512, 11008, 4096, T256X128), (1024, 11008, 4096, T256),
    (1576, 1536, 384, T64), (3152, 1536, 384, T128), (300000, 64, 64, T64), (25216, 1152, 384, T128),
    # half the rounds: 256 x 256 from 768 bytes of K on
    (4096, 4096, 768, T256), (8192, 8192, 768, T256), (8192, 8192, 4096, T256), (4096, 8192, 1024, T256),
    # three of five rounds: from 2048 bytes on; four of seven: from 1536
    (50432, 768, 768, T128), (50432, 768, 1024, T128), (50432, 768, 2032, T128), (50432, 768, 2048, T256), (25216, 2304, 768, T128), (25216, 2304, 1520, T128),
    (25216, 2304, 1536, T256)])
def test_form(form, M, N, K, want):
    assert form(M, N, K) == want
