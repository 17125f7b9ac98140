"""Into how many parts attention over the cache cuts its keys: the rule (host code, compiled here) against what the kernel makes of it."""
import ctypes
import random
import subprocess

import pytest

from paper_2207_01405_amd import build

CUS, BK = 256, 32
NAMES = ("prefix_tiles", "own_tiles", "prefix_parts", "own_parts", "prefix_least", "own_least", "wide")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("cached")
    (d / "r.cpp").write_text('#include "cached_form.hpp"\n'
                             'extern "C" void plan(int B, int H, int G, int d, int i8, int page, int pages, int prefix, int* o) {\n'
                             '    const ivit::cached::Plan p = ivit::cached::plan_of(B, H, G, d, i8, page, pages, prefix, %d);\n'
                             '    const int all[] = {%s};\n    for (int i = 0; i < %d; ++i) o[i] = all[i];\n}\n'
                             % (CUS, ", ".join("p." + n for n in NAMES), len(NAMES)))
    subprocess.run(["g++", "-std=c++20", "-shared", "-fPIC", "-I", build.CSRC, str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    lib = ctypes.CDLL(str(d / "r.so"))

    def of(B, H, G, d, prefix, keys, i8=False, page=64):
        out = (ctypes.c_int * len(NAMES))()
        lib.plan(B, H, G, d, i8, page, -(-keys // page), prefix, out)
        return dict(zip(NAMES, out))
    return of


def sizes(keys, parts, least):
    """blocks of each part, as the kernel cuts them"""
    blocks = -(-keys // BK)
    each = max(-(-blocks // parts), least)
    return [max(0, min(blocks, (p + 1) * each) - min(blocks, p * each)) for p in range(parts)]


def check(p, prefix, keys, what):
    if prefix:
        s = sizes(prefix, p["prefix_parts"], p["prefix_least"])
        assert min(s) > 0, (what, "prefix", p, s)
    if keys:
        s = sizes(keys, p["own_parts"], p["own_least"])
        assert min(s) > 0, (what, "own", p, s)


@pytest.mark.parametrize("B,H,G,prefix,i8", [(20, 32, 8, 1000, False), (17, 32, 8, 512, False), (24, 16, 4, 2000, True), (64, 32, 8, 8000, False), (1, 32, 8, 300, False)])
def test_every_part_of_a_prefix_has_keys(plan, B, H, G, prefix, i8):
    p = plan(B, H, G, 128, prefix, 64, i8)
    check(p, prefix, 64, (B, H, G, prefix))
    # a workgroup that shares tiles takes a block a wavefront at the least
    assert p["prefix_least"] == (4 if B * H // G > 64 else 8) and bool(p["wide"]) == (B * H // G > 64)


def test_every_part_has_keys_at_the_greatest_length(plan):
    r = random.Random(1)
    for _ in range(20000):
        G = r.choice((1, 2, 4, 8, 16))
        B, H = int(2 ** r.uniform(0, 9)), G * r.choice((1, 2, 4, 5, 8))
        prefix, keys = r.choice((0, int(2 ** r.uniform(0, 16)))), r.choice((0, 64 * int(2 ** r.uniform(0, 10))))
        p = plan(B, H, G, r.choice((64, 128)), prefix, keys, r.random() < 0.5)
        assert (p["prefix_parts"] > 0) == (prefix > 0) and (p["own_parts"] > 0) == (keys > 0)
        check(p, prefix, keys, (B, H, G, prefix, keys))


def test_more_than_64_parts(plan):
    """What the tests of the join go by: one request with a table of 32768 keys and 8 key heads, and a prefix before it."""
    assert plan(1, 32, 8, 128, 0, 33024)["own_parts"] > 64 and plan(1, 32, 8, 128, 20000, 20032)["own_parts"] > 64
    p = plan(1, 32, 8, 128, 9000, 13056)
    assert p["prefix_parts"] < 64 and p["own_parts"] < 64 and p["prefix_parts"] + p["own_parts"] > 64
