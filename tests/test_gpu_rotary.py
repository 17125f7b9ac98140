"""Rotary positions and the appending of rows to a paged cache against their definitions in 64 bits.

A turned element is x1 c - x2 s: the angle's sine and cosine are within 2^-22 + |phi| 2^-51, two products and a sum are rounded in 32 bits (3 U), and
the result to its type (half a step).  int8 rows: the exact quotient's nearest whole number, of values with those errors."""
import random

import pytest

from attention_rows import U, dtype, gen, half, rand

pytestmark = pytest.mark.gpu


def turned64(x, heads, d, rotary):
    """(x turned, its bound on errors in 32 bits, without the last rounding)"""
    import torch
    rows, freq = x.shape[0], rotary["freq"]
    n = freq.shape[0]
    pos = rotary["positions"].reshape(-1, rows).double()
    axis = rotary.get("axis")
    axis = torch.zeros(n, dtype=torch.int64, device="cuda") if axis is None else axis.long().clamp(0, pos.shape[0] - 1)
    phi = (pos[axis] * freq[:, None]).t()[:, None, :]
    c, s = phi.cos(), phi.sin()
    x = x.double().reshape(rows, heads, d)
    if rotary.get("adjacent"):
        i1 = torch.arange(0, 2 * n, 2, device="cuda")
        i2 = i1 + 1
    else:
        i1 = torch.arange(n, device="cuda")
        i2 = i1 + n
    x1, x2 = x[..., i1], x[..., i2]
    y, err = x.clone(), torch.zeros_like(x)
    y[..., i1], y[..., i2] = x1 * c - x2 * s, x2 * c + x1 * s
    e = (2.0 ** -22 + phi.abs() * 2.0 ** -51 + 3 * U) * (x1.abs() + x2.abs())
    err[..., i1], err[..., i2] = e, e
    return y.reshape(rows, -1), err.reshape(rows, -1)


def tiny(t):
    return {"f32": 2.0 ** -125, "f16": 2.0 ** -25, "bf16": 2.0 ** -125}[t]


def check(y, want, err, t, what):
    off = (y.double() - want).abs()
    bound = err + half(t) * (want.abs() + err) + tiny(t)
    assert bool((off <= bound).all()), "%s: %g over" % (what, float((off - bound).max()))


def make_rotary(g, rows, rot, axes, adjacent, far=100000):
    import torch
    n = rot // 2
    r = {"freq": 10000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float64) / n), "adjacent": adjacent}
    r["positions"] = torch.randint(-far, far, (rows,) if axes == 1 else (axes, rows), generator=g, device="cuda", dtype=torch.int32)
    r["axis"] = None if axes == 1 else torch.randint(0, axes, (n,), generator=g, device="cuda", dtype=torch.int32)
    return r


SHAPES = [(1, 1, 2, 2), (1, 40, 128, 128), (3, 2, 6, 4), (7, 3, 16, 16), (5, 5, 18, 18), (33, 4, 64, 64), (100, 3, 80, 60), (1000, 2, 96, 32), (257, 7, 128, 64),
          (4, 1, 1024, 1024), (2, 2, 1022, 1018), (50, 9, 10, 2), (2500, 12, 64, 64)]


@pytest.mark.parametrize("rows,heads,d,rot", SHAPES)
def test_rotary(ivit, rows, heads, d, rot):
    import torch
    for i, t in enumerate(("f32", "f16", "bf16")):
        for axes, adjacent in ((1, False), (1, True), (3, False), (2, True)):
            g = gen(17 * rows + d + i)
            r = make_rotary(g, rows, rot, axes, adjacent)
            x = rand(g, rows, heads * d).to(dtype(t))
            want, err = turned64(x, heads, d, r)
            y = torch.empty_like(x)
            assert ivit.ivit_rotary(x, y, d, r) is y
            what = "%d x %d x %d/%d %s axes %d adjacent %s" % (rows, heads, d, rot, t, axes, adjacent)
            check(y, want, err, t, what)
            z = x.clone()
            ivit.ivit_rotary(z, z, d, r)
            assert torch.equal(z, y), what + ": in place"


def test_rotary_in_wider_rows_and_elements_alone_aligned(ivit):
    import torch
    g = gen(5)
    for t in ("f32", "f16", "bf16"):
        wide = rand(g, 19, 3 * 40 + 7).to(dtype(t))
        x, keep = wide[:, 3:123], wide.clone()
        r = make_rotary(g, 19, 34, 1, False)
        want, err = turned64(x, 3, 40, r)
        out = torch.full((19, 131), 7.0, device="cuda", dtype=dtype(t))
        ivit.ivit_rotary(x, out[:, 5:125], 40, r)
        check(out[:, 5:125], want, err, t, t)
        assert bool((out[:, :5] == 7).all()) and bool((out[:, 125:] == 7).all()) and torch.equal(wide, keep)
        ivit.ivit_rotary(x, x, 40, r)
        assert torch.equal(x, out[:, 5:125]) and torch.equal(wide[:, :3], keep[:, :3]) and torch.equal(wide[:, 123:], keep[:, 123:])


def test_far_positions_and_axes_out_of_range(ivit):
    import torch
    g = gen(6)
    r = make_rotary(g, 300, 64, 1, False, far=2 ** 31 - 1)
    r["positions"][:2] = torch.tensor([2 ** 31 - 1, -2 ** 31], dtype=torch.int64, device="cuda").to(torch.int32)
    x = rand(g, 300, 128)
    want, err = turned64(x, 2, 64, r)
    check(ivit.ivit_rotary(x, torch.empty_like(x), 64, r), want, err, "f32", "far")
    r = make_rotary(g, 300, 64, 2, False)
    r["axis"] = torch.randint(-5, 9, (32,), generator=g, device="cuda", dtype=torch.int32)
    want, err = turned64(x, 2, 64, r)
    check(ivit.ivit_rotary(x, torch.empty_like(x), 64, r), want, err, "f32", "axes")


def test_rotary_axes_of_a_larger_table(ivit):
    import torch
    g = gen(7)
    r = make_rotary(g, 70, 32, 3, True)
    table = torch.randint(0, 500, (3, 90), generator=g, device="cuda", dtype=torch.int32)
    r["positions"] = table[:, 11:81]
    x = rand(g, 70, 64)
    want, err = turned64(x, 2, 32, r)
    check(ivit.ivit_rotary(x, torch.empty_like(x), 32, r), want, err, "f32", "table")


def test_turning_back(ivit):
    """A turn by phi and one by -phi leave the row, to twice the stated errors."""
    import torch
    g = gen(8)
    r = make_rotary(g, 64, 128, 1, False)
    x = rand(g, 64, 512)
    y = ivit.ivit_rotary(x, torch.empty_like(x), 128, r)
    back = ivit.ivit_rotary(y, torch.empty_like(x), 128, dict(r, positions=-r["positions"]))
    _, e1 = turned64(x, 4, 128, r)
    assert bool(((back - x).abs() <= 4 * e1.amax(1, keepdim=True) + 4 * U * x.abs()).all())


# -------------------------------------------------------------------------------------------------------------- the cache
def make_cache(g, pages, kv, page, d, t, i8, padded=False):
    import torch
    shape = (pages, kv, page, d)
    if i8:
        c = {n: torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8) for n in "kv"}
        c["k_scale"], c["v_scale"] = (rand(g, *shape[:3]).abs() for _ in range(2))
        return c
    if padded:                                      # keys and values of a page side by side in one tensor
        both = rand(g, pages, 2, *shape[1:]).to(dtype(t))
        return {"k": both[:, 0], "v": both[:, 1]}
    return {n: rand(g, *shape).to(dtype(t)) for n in "kv"}


def check_append(ivit, g, rows, H, G, d, t, i8, page, rot, axes, adjacent, padded=False, wide=0):
    import torch
    what = "%d rows %d/%d x %d %s i8 %s page %d rot %s axes %d adjacent %s" % (rows, H, G, d, t, i8, page, rot, axes, adjacent)
    pages = (rows + page - 1) // page + 3
    c = make_cache(g, pages, G, page, d, t, i8, padded)
    before = {n: x.clone() for n, x in c.items()}
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:rows].to(torch.int32)
    if rows > 3:
        slots[1], slots[-1] = -1, pages * page
    qkv = rand(g, rows, (H + 2 * G) * d + wide).to(dtype(t))
    q, k, v = qkv[:, :H * d], qkv[:, H * d:(H + G) * d], qkv[:, (H + G) * d:(H + 2 * G) * d]
    q_out = torch.full((rows, H * d + wide), 5.0, device="cuda", dtype=dtype(t))
    r = make_rotary(g, rows, rot, axes, adjacent) if rot else None
    ivit.ivit_cache_append(k, v, slots, c, rotary=r, q=q if H else None, q_out=q_out[:, :H * d] if H else None)
    real = (slots >= 0) & (slots < pages * page)
    at = slots[real].long()
    at, off = at // page, at % page
    nothing = torch.zeros(rows, G * d, device="cuda", dtype=torch.float64)
    wk, ek = turned64(k, G, d, r) if r else (k.double(), nothing)
    for name, want, err in (("k", wk, ek), ("v", v.double(), nothing)):
        got = c[name][at, :, off].reshape(-1, d)
        want, err = want[real].reshape(-1, d), err[real].reshape(-1, d)
        if i8:
            s = c[name + "_scale"][at, :, off].reshape(-1, 1)
            top, e = want.abs().amax(1, keepdim=True), err.amax(1, keepdim=True)
            assert bool(((s - top / 127).abs() <= (e + 2 * U * top) / 127 + 2.0 ** -126).all()), what + ": scale"
            assert bool((got.abs().amax(1) == 127).all()), what + ": largest"
            # half a step, the value's error and that of the largest, which the steps go by
            assert bool(((got.double() * top / 127 - want).abs() <= top / 127 * (0.5 + 2.0 ** -44) + err + e * got.double().abs() / 127).all()), what + ": " + name
        else:
            check(got, want, err, t, what + ": " + name)
        rest = torch.ones(pages * page, dtype=torch.bool, device="cuda")
        rest[slots[real].long()] = False
        for n in (name, name + "_scale") if i8 else (name,):
            a, b = (x[n].transpose(1, 2).flatten(0, 1)[rest] for x in (c, before))
            assert torch.equal(a, b), what + ": other slots of " + n
    if H:
        want, err = turned64(q, H, d, r) if r else (q.double(), torch.zeros(rows, H * d, device="cuda", dtype=torch.float64))
        check(q_out[real][:, :H * d], want[real], err[real], t, what + ": q")
        assert bool((q_out[~real] == 5).all()) and bool((q_out[:, H * d:] == 5).all()), what + ": padded rows"


@pytest.mark.parametrize("rows", [1, 2, 15, 64, 257, 1500])
def test_append(ivit, rows):
    r = random.Random(rows)
    for t in ("f16", "bf16"):
        for i8 in (False, True):
            for d in (64, 128):
                for rot, axes, adjacent in ((d, 1, False), (d, 1, True), (d // 2, 3, False), (d - 14, 2, False), (10, 1, True), (0, 1, False)):
                    G = r.choice((1, 2, 3, 8))
                    check_append(ivit, gen(rows + d + rot), rows, G * r.choice((0, 1, 4)), G, d, t, i8, r.choice((16, 32, 64, 1024)), rot, axes, adjacent,
                                 padded=r.random() < 0.3, wide=r.choice((0, 0, 1, 8)))


def test_int8_rows_without_values_or_not_finite(ivit):
    import torch
    g = gen(3)
    for t in ("f16", "bf16"):
        k, v = rand(g, 6, 256).to(dtype(t)), rand(g, 6, 256).to(dtype(t))
        k[0], v[1] = 0, 0
        k[2, 3], v[3, 130], k[4, 200] = float("nan"), float("inf"), float("-inf")
        c = make_cache(g, 2, 2, 16, 128, t, True)
        slots = torch.arange(6, device="cuda", dtype=torch.int32)
        ivit.ivit_cache_append(k, v, slots, c)
        for n, x in (("k", k), ("v", v)):
            for i in range(6):
                for h in range(2):
                    row, s, q = x[i, 128 * h:128 * h + 128].double(), float(c[n + "_scale"][0, h, i]), c[n][0, h, i]
                    if not bool(row.isfinite().all()):
                        assert s != s and not bool(q.any())
                    elif not bool(row.any()):
                        assert s == 0 and not bool(q.any())
                    else:
                        assert abs(s - float(row.abs().max()) / 127) <= 2 * U * s
                        assert torch.equal(q.double(), torch.round(127 * row / row.abs().max()))
