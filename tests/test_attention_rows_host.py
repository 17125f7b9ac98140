"""Rotary positions, the paged cache and attention over float rows: what the C entry points and the binding refuse before anything is launched (no GPU)."""
import ctypes as C
import os

import pytest

from paper_2207_01405_amd import binding

FAKE = 0x10000          # a non-NULL, 256-byte aligned address that is never dereferenced
E = binding.ERRORS
F32, F16, BF16, I8 = 0, 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2207_01405_amd import build
        build.build_lib()
    return binding.load()


def turn(pos=FAKE, ld=4, axes=1, freq=FAKE, axis=None, rot=64, adjacent=0):
    return binding.RotaryParams(pos, ld, axes, freq, axis, rot, adjacent)


def pool(k=FAKE, v=FAKE, ks=None, vs=None, ld=None, pages=8, page=32, heads=2, d=64, t=BF16):
    return binding.Cache(k, v, ks, vs, heads * page * d if ld is None else ld, pages, page, heads, d, t)


def rotary(lib, x=FAKE, ldx=128, y=FAKE + 4096, ldy=128, rows=4, heads=2, d=64, t=BF16, r=None, none=False):
    return lib.ivit_rotary(None, x, ldx, y, ldy, rows, heads, d, t, None if none else C.byref(turn() if r is None else r))


def test_rotary_refusals(lib):
    assert rotary(lib, x=None) == E["NULL"] and rotary(lib, y=None) == E["NULL"] and rotary(lib, none=True) == E["NULL"]
    assert rotary(lib, r=turn(pos=None)) == E["NULL"] and rotary(lib, r=turn(freq=None)) == E["NULL"]
    assert rotary(lib, rows=-1) == E["SHAPE"] and rotary(lib, rows=1 << 31, r=turn(ld=1 << 31)) == E["SHAPE"] and rotary(lib, heads=0) == E["SHAPE"]
    for d in (0, 1, 65, 1026):
        assert rotary(lib, d=d, ldx=4096, ldy=4096, r=turn(rot=2)) == E["SHAPE"], d
    assert rotary(lib, heads=(1 << 24) // 64 + 1, ldx=1 << 25, ldy=1 << 25) == E["SHAPE"]
    for rot in (0, 1, -2, 63, 66):
        assert rotary(lib, r=turn(rot=rot)) == E["SHAPE"], rot
    assert rotary(lib, ldx=127) == E["SHAPE"] and rotary(lib, ldy=127) == E["SHAPE"] and rotary(lib, r=turn(ld=3)) == E["SHAPE"]
    assert rotary(lib, t=I8) == E["PARAM"] and rotary(lib, t=-1) == E["PARAM"] and rotary(lib, r=turn(axes=0)) == E["PARAM"] and rotary(lib, r=turn(axes=9)) == E["PARAM"]
    assert rotary(lib, y=FAKE, ldy=256) == E["PARAM"]                                   # in place with other rows
    assert rotary(lib, x=FAKE + 1) == E["ALIGN"] and rotary(lib, y=FAKE + 2, t=F32) == E["ALIGN"] and rotary(lib, r=turn(pos=FAKE + 2)) == E["ALIGN"]
    assert rotary(lib, r=turn(freq=FAKE + 4)) == E["ALIGN"] and rotary(lib, r=turn(axis=FAKE + 1)) == E["ALIGN"]
    assert rotary(lib, x=None, y=None, rows=0, r=turn(pos=None, ld=0)) == 0


def append(lib, q=None, ldq=256, qo=None, ldqo=256, H=4, k=FAKE, ldk=128, v=FAKE, ldv=128, slots=FAKE, rows=4, t=BF16, r=None, c=None, none=False):
    return lib.ivit_cache_append(None, q, ldq, qo, ldqo, H, k, ldk, v, ldv, slots, rows, t, None if r is None else C.byref(r),
                                 None if none else C.byref(pool() if c is None else c))


def test_append_refusals(lib):
    assert append(lib, none=True) == E["NULL"]
    for name in ("k", "v", "slots"):
        assert append(lib, **{name: None}) == E["NULL"], name
    assert append(lib, q=FAKE) == E["NULL"] and append(lib, qo=FAKE) == E["NULL"]
    assert append(lib, c=pool(k=None)) == E["NULL"] and append(lib, c=pool(v=None)) == E["NULL"] and append(lib, c=pool(t=I8, ks=FAKE)) == E["NULL"]
    assert append(lib, t=F32) == E["PARAM"] and append(lib, t=I8) == E["PARAM"] and append(lib, t=F16) == E["PARAM"] and append(lib, c=pool(t=F32)) == E["PARAM"]
    assert append(lib, r=turn(axes=0)) == E["PARAM"] and append(lib, r=turn(rot=66)) == E["SHAPE"] and append(lib, r=turn(ld=2)) == E["SHAPE"]
    for d in (32, 96, 256):
        assert append(lib, c=pool(d=d), ldk=1024, ldv=1024) == E["SHAPE"], d
    for page in (0, 8, 24, 2048, -16):
        assert append(lib, c=pool(page=page, ld=1 << 20)) == E["SHAPE"], page
    assert append(lib, c=pool(pages=0)) == E["SHAPE"] and append(lib, c=pool(pages=1 << 26)) == E["SHAPE"] and append(lib, c=pool(heads=0, ld=4096)) == E["SHAPE"]
    assert append(lib, c=pool(ld=4095 * 1)) == E["SHAPE"] and append(lib, c=pool(heads=4097), ldk=1 << 20, ldv=1 << 20) == E["SHAPE"]
    assert append(lib, rows=-1) == E["SHAPE"] and append(lib, rows=1 << 31) == E["SHAPE"] and append(lib, ldk=127) == E["SHAPE"] and append(lib, ldv=127) == E["SHAPE"]
    assert append(lib, q=FAKE, qo=FAKE, H=0) == E["SHAPE"] and append(lib, q=FAKE, qo=FAKE, ldq=255) == E["SHAPE"] and append(lib, q=FAKE, qo=FAKE, ldqo=255) == E["SHAPE"]
    assert append(lib, k=FAKE + 1) == E["ALIGN"] and append(lib, slots=FAKE + 2) == E["ALIGN"] and append(lib, c=pool(k=FAKE + 8)) == E["ALIGN"]
    assert append(lib, c=pool(ld=4100)) == E["ALIGN"] and append(lib, c=pool(t=I8, ks=FAKE + 2, vs=FAKE)) == E["ALIGN"] and append(lib, q=FAKE + 1, qo=FAKE) == E["ALIGN"]
    assert append(lib, k=None, v=None, slots=None, rows=0) == 0


def test_append_in_place_and_prompts_beyond_31_bits_are_refused(lib):
    """Queries turned in place would be read by one lane while another turns them; the numbers of 2^30 rows and of a tile behind them fit 32 bits."""
    assert append(lib, q=FAKE, qo=FAKE) == E["PARAM"] and append(lib, q=FAKE, qo=FAKE, r=turn()) == E["PARAM"]
    assert prompt(lib, nk=(1 << 30) + 1, ks=FAKE) == E["SHAPE"] and prompt(lib, nq=(1 << 30) + 1, ks=FAKE, H=1, G=1) == E["SHAPE"]


def prompt(lib, q=FAKE, ldq=256, k=FAKE, ldk=128, v=FAKE, ldv=128, o=FAKE, ldo=256, qs=FAKE, ks=None, n=1, nq=8, nk=8, H=4, G=2, d=64, t=BF16, scale=0.125, causal=1):
    return lib.ivit_prompt_attention(None, q, ldq, k, ldk, v, ldv, o, ldo, qs, ks, n, nq, nk, H, G, d, t, scale, causal)


def test_prompt_refusals(lib):
    for name in ("q", "k", "v", "o", "qs"):
        assert prompt(lib, **{name: None}) == E["NULL"], name
    assert prompt(lib, t=F32) == E["PARAM"] and prompt(lib, t=I8) == E["PARAM"]
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert prompt(lib, scale=scale) == E["PARAM"]
    assert prompt(lib, nq=-1) == E["SHAPE"] and prompt(lib, nk=1 << 31, ks=FAKE) == E["SHAPE"] and prompt(lib, n=-1) == E["SHAPE"] and prompt(lib, n=1 << 20) == E["SHAPE"]
    assert prompt(lib, nk=9) == E["SHAPE"]                                              # other keys than queries without k_start
    for d in (32, 96, 256):
        assert prompt(lib, d=d, ldq=2048, ldk=2048, ldv=2048, ldo=2048) == E["SHAPE"], d
    assert prompt(lib, H=0) == E["SHAPE"] and prompt(lib, G=0) == E["SHAPE"] and prompt(lib, G=3) == E["SHAPE"] and prompt(lib, G=8) == E["SHAPE"]
    assert prompt(lib, H=4098, G=2, ldq=1 << 20, ldo=1 << 20) == E["SHAPE"] and prompt(lib, n=(1 << 20) - 1, H=4096, ldq=1 << 20, ldo=1 << 20) == E["SHAPE"]
    assert prompt(lib, ldq=248) == E["SHAPE"] and prompt(lib, ldk=120) == E["SHAPE"] and prompt(lib, ldv=120) == E["SHAPE"] and prompt(lib, ldo=248) == E["SHAPE"]
    assert prompt(lib, ldk=(1 << 24) + 8) == E["SHAPE"] and prompt(lib, ldv=(1 << 24) + 8) == E["SHAPE"]
    for name in ("q", "k", "v", "o"):
        assert prompt(lib, **{name: FAKE + 8}) == E["ALIGN"] and prompt(lib, **{"ld" + name: 260}) == E["ALIGN"], name
    assert prompt(lib, qs=FAKE + 2) == E["ALIGN"] and prompt(lib, ks=FAKE + 2) == E["ALIGN"]
    assert prompt(lib, q=None, o=None, nq=0, ks=FAKE) == 0 and prompt(lib, n=0) == 0


def cached(lib, q=FAKE, ldq=256, o=FAKE, ldo=256, c=None, pp=None, pl=0, pages=FAKE, ldp=4, mp=4, lens=FAKE, B=3, H=4, t=BF16, scale=0.125, ws=FAKE, n=1 << 40, none=False):
    return lib.ivit_cached_attention(None, q, ldq, o, ldo, None if none else C.byref(pool() if c is None else c), pp, pl, pages, ldp, mp, lens, B, H, t, scale, ws, n)


def size(lib, B=3, H=4, c=None, mp=4, pl=0, none=False):
    return lib.ivit_cached_attention_workspace_bytes(B, H, None if none else C.byref(pool() if c is None else c), mp, pl)


def test_cached_refusals(lib):
    assert cached(lib, none=True) == E["NULL"]
    for name in ("q", "o", "pages", "lens"):
        assert cached(lib, **{name: None}) == E["NULL"], name
    assert cached(lib, pl=1) == E["NULL"]
    assert cached(lib, t=F32) == E["PARAM"] and cached(lib, t=F16) == E["PARAM"] and cached(lib, t=F16, c=pool(t=I8, ks=FAKE, vs=FAKE), B=0) == 0
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert cached(lib, scale=scale) == E["PARAM"]
    assert cached(lib, B=-1) == E["SHAPE"] and cached(lib, B=65537) == E["SHAPE"] and cached(lib, H=0) == E["SHAPE"] and cached(lib, H=3, ldq=192) == E["SHAPE"]
    assert cached(lib, H=1) == E["SHAPE"] and cached(lib, B=65536, H=4096, ldq=1 << 20, ldo=1 << 20) == E["SHAPE"]
    assert cached(lib, pl=-1, pp=FAKE) == E["SHAPE"] and cached(lib, pl=(1 << 30) + 1, pp=FAKE) == E["SHAPE"] and cached(lib, mp=-1) == E["SHAPE"]
    assert cached(lib, mp=(1 << 25) + 1, ldp=1 << 26) == E["SHAPE"] and cached(lib, ldp=3) == E["SHAPE"]
    assert cached(lib, ldq=248) == E["SHAPE"] and cached(lib, ldo=248) == E["SHAPE"] and cached(lib, c=pool(page=8)) == E["SHAPE"]
    assert cached(lib, q=FAKE + 8) == E["ALIGN"] and cached(lib, o=FAKE + 8) == E["ALIGN"] and cached(lib, ldq=260) == E["ALIGN"] and cached(lib, ldo=260) == E["ALIGN"]
    assert cached(lib, pages=FAKE + 2) == E["ALIGN"] and cached(lib, lens=FAKE + 2) == E["ALIGN"] and cached(lib, pl=1, pp=FAKE + 2) == E["ALIGN"]
    assert cached(lib, ws=None) == E["WORKSPACE"] and cached(lib, n=size(lib) - 1) == E["WORKSPACE"] and cached(lib, ws=FAKE + 128) == E["ALIGN"]
    assert cached(lib, q=None, o=None, pages=None, lens=None, B=0, ws=None, n=0) == 0


def test_workspace(lib):
    assert size(lib, none=True) == 0 and size(lib, c=pool(page=8)) == 0 and size(lib, B=-1) == 0 and size(lib, H=3) == 0
    # a part's largest score, sum and output for every head of every request
    assert size(lib) >= 3 * 4 * (64 + 2) * 4
    assert size(lib, pl=1000) > size(lib)
    # no requests, no pages of their own: valid calls
    assert 0 < size(lib, B=0) <= 4096 and 0 < size(lib, B=0, pl=1000) <= 4096 and 0 < size(lib, mp=0) and 0 < size(lib, B=0, mp=0) and 0 < size(lib, mp=0, pl=1)
    # of 64 parts of a request's keys at most, however long it may get, where there are many requests
    assert size(lib, B=500, mp=1 << 20) <= 64 * 500 * 4 * (64 + 2) * 4 + 4096


def test_very_many_requests(lib):
    """A workgroup of 256 threads for every key head, 32 query heads and part: less than 2^24 of them fit a launch."""
    for B, H, heads in ((32768, 256, 256), (65536, 128, 128), (65536, 128, 4), (2048, 4096, 4096), (2048, 4096, 64), (4096, 256, 256)):
        for prefix in (0, 1 << 20):
            c = pool(heads=heads, page=16)
            parts = size(lib, B=B, H=H, c=c, mp=1 << 20, pl=prefix) // (B * H * (64 + 2) * 4)
            group = H // heads
            least = (-(-B * group // 128) * heads if prefix else 0) + B * heads * -(-group // 32)          # one part of both
            assert parts >= 1 and least < 1 << 24
            assert (parts - (1 if prefix else 0)) * B * heads * -(-group // 32) < 1 << 24, (B, H, heads, prefix, parts)
        assert size(lib, B=65536, H=129, c=pool(heads=129, page=16)) == 0 and cached(lib, B=65536, H=129, c=pool(heads=129), ldq=129 * 64, ldo=129 * 64) == E["SHAPE"]


def test_the_binding_refuses_tensors_that_are_not_as_stated(lib):
    """Wrong types, shapes and strides, and host tensors (all of these are)."""
    import torch
    z, i32, bf = torch.zeros, torch.int32, torch.bfloat16
    x, pos, freq = z(4, 128, dtype=bf), z(4, dtype=i32), z(32, dtype=torch.float64)
    r = {"positions": pos, "freq": freq}
    c = {"k": z(8, 2, 32, 64, dtype=bf), "v": z(8, 2, 32, 64, dtype=bf)}
    starts, slots, table, lens, ws = z(2, dtype=i32), z(4, dtype=i32), z(4, 3, dtype=i32), z(4, dtype=i32), z(1 << 20, dtype=torch.uint8)
    b = binding
    bad = [lambda: b.ivit_rotary(x, x, 64, r),                                                    # on the host
           lambda: b.ivit_rotary(x, x, 60, r), lambda: b.ivit_rotary(x, x.float(), 64, r), lambda: b.ivit_rotary(x.double(), x, 64, r),
           lambda: b.ivit_rotary(x, x, 64, dict(r, positions=pos.long())), lambda: b.ivit_rotary(x, x, 64, dict(r, positions=z(5, dtype=i32))),
           lambda: b.ivit_rotary(x, x, 64, dict(r, freq=freq.float())), lambda: b.ivit_rotary(x, x, 64, dict(r, axis=z(31, dtype=i32))),
           lambda: b.ivit_cache_append(x, x, slots, c), lambda: b.ivit_cache_append(x, x, slots.long(), c), lambda: b.ivit_cache_append(x[:, :64], x, slots, c),
           lambda: b.ivit_cache_append(x, x, slots, c, q=x), lambda: b.ivit_cache_append(x, x, slots, c, q_out=x),
           lambda: b.ivit_cache_append(x, x, slots, {"k": c["k"], "v": c["v"].half()}), lambda: b.ivit_cache_append(x, x, slots, {"k": c["k"], "v": c["v"][:4]}),
           lambda: b.ivit_cache_append(x, x, slots, {"k": c["k"].transpose(1, 2), "v": c["v"].transpose(1, 2)}),
           lambda: b.ivit_cache_append(x, x, slots, {"k": c["k"][::2], "v": c["v"][:4]}),
           lambda: b.ivit_prompt_attention(x, x, x, x, 64, starts), lambda: b.ivit_prompt_attention(x, x, x, x, 60, starts),
           lambda: b.ivit_prompt_attention(x, x, x[:, :64], x, 64, starts), lambda: b.ivit_prompt_attention(x, x, x, x.float(), 64, starts),
           lambda: b.ivit_prompt_attention(x, x, x, x, 64, starts.long()), lambda: b.ivit_prompt_attention(x, x, x, x, 64, starts, z(3, dtype=i32)),
           lambda: b.ivit_prompt_attention(x, x, x, x, 64, z(0, dtype=i32)),
           lambda: b.ivit_cached_attention(x, x, c, table, lens, ws), lambda: b.ivit_cached_attention(x[:, :96], x, c, table, lens, ws),
           lambda: b.ivit_cached_attention(x, x, c, table.long(), lens, ws), lambda: b.ivit_cached_attention(x, x, c, table[:3], lens, ws),
           lambda: b.ivit_cached_attention(x, x, c, table, lens[:3], ws), lambda: b.ivit_cached_attention(x, x, c, table, lens, ws, prefix_len=33, prefix_pages=z(1, dtype=i32)),
           lambda: b.ivit_cached_attention(x, x, c, table, lens, ws, prefix_len=5), lambda: b.ivit_cached_attention(x, x, c, table, lens, ws[::2])]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was not refused" % i)
    with pytest.raises(KeyError):                                                                 # an int8 cache without its scales
        b.cache_struct({"k": c["k"].to(torch.int8), "v": c["v"].to(torch.int8)}, -1)


def test_no_vector_register_is_spilled(lib):
    """Loads of the attention kernels are counted by hand (s_waitcnt): a reload from scratch memory between them would wait for all."""
    import re
    from test_spilled_registers import _spills
    of = {name: n for name, n in _spills().items() if re.search(r"\d(prompt_attention|cached_attention|join|rotary|append)_kernel", name)}
    assert len(of) > 30 and not [(name, n) for name, n in of.items() if n]
