"""The float layers around int8 products against their definitions in 64 bits.

Tolerances count roundings: U = 2^-24 is half a unit of a 32-bit value's last place, HALF[type] half a step of the type a result is
stored in.  Where an int8 value is checked, it has to lie within half a step and the stated error of the unrounded quotient; int8 sums are exact."""
import math
import random

import numpy as np
import pytest

import oracle as orc
from paper_2207_01405_amd import synth

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = ("f32", "f16", "bf16")
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh", "gelu_sigmoid")
# operations of 32 bits (each U, or a unit in the last place of a transcendental, 2 U) between the inputs of an epilogue and its
# result, relative to the largest term on the way: scale, scale, bias 3; activation: slope 4, exponential 2 + 0.3 x 4 (its
# argument's error times s sigma(s) (1 - sigma(s)) <= 0.28), sum 1, reciprocal 2, product 1; gelu: the fit of erfcx 4.4e-7 = 7.4 U
# on at most half of x; gate's product 1; residual 1
OPS = 20


def dtype(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}[name]


def half(name):
    import torch
    return 0.0 if name == "i8" else torch.finfo(dtype(name)).eps / 2


def tiny(name):
    """Half a step of the numbers below the normal ones, and what a value below 2^-126 may lose on the way."""
    return {"f32": 2.0 ** -125, "f16": 2.0 ** -25, "bf16": 2.0 ** -125}[name]


def act64(z, kind):
    import torch
    if kind == "relu":
        return z.clamp_min(0.0)
    if kind == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    s = {"silu": z, "gelu_sigmoid": 1.702 * z, "gelu_tanh": 2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)}.get(kind)
    return z if s is None else z * torch.sigmoid(s)


def rand(g, *shape):
    import torch
    return torch.randn(shape, generator=g, device="cuda")


def gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def check_q(q, scale, v, err, what):
    """int8 rows of values v [rows, C], each known to within err [rows, C]"""
    import torch
    top = v.abs().amax(1)
    s = top / 127.0
    assert bool(((scale.double() - s).abs() <= err.amax(1) / 127.0 + 8 * U * s + 2.0 ** -126).all()), what + ": scale"
    zero = s == 0
    assert not bool(q[zero].any()), what + ": a row of zeros"
    # q s against v: half a step, the errors of v and of the largest value, and those of the quotient (4 U of at most 127 steps)
    off = (q.double() * s[:, None] - v).abs()
    bound = s[:, None] * (0.5 + 127 * 6 * U) + err + err.amax(1, keepdim=True) * (q.double().abs() / 127.0)
    assert bool((off <= bound).all()), "%s: %g over" % (what, float((off - bound).max()))


# ---------------------------------------------------------------------------------------------------------------- norm
def norm_ref(x, r, gamma, eps, C):
    h = x.double() if r is None else x.double() + r.double()
    n = h / ((h * h).mean(1, keepdim=True) + eps).sqrt()
    return h, n if gamma is None else n * gamma.double()


def check_norm(x, r, gamma, eps, t, total, y, scale, what):
    import torch
    C = x.shape[1]
    h, n = norm_ref(x, r, gamma, eps, C)
    if total is not None:
        assert bool(((total.double() - h).abs() <= (half(t) + U) * h.abs() + tiny(t)).all()), what + ": sum"
    # the sum's rounding, and half the error of a sum of squares in chains of at most 32 with a tree of 10 above them, relative to h;
    # then the square root, the quotient, gamma
    err = (32 + 10 + 3) / 2 * U * n.abs() + 6 * U * n.abs()
    if scale is None:
        assert bool(((y.double() - n).abs() <= err + half(t) * n.abs() + tiny(t)).all()), what + ": y"
        return
    top = n.abs().amax(1)
    assert bool(((scale.double() - top / 127).abs() <= 36 * U * top / 127 + 2.0 ** -126).all()), what + ": scale"
    # q comes from h gamma alone: 2 U a value and 2 U its largest, 2 U the quotient 127 / top, 1 U its product with gamma's
    v, s = n, (top / 127)[:, None]
    off, bound = (y.double() * s - v).abs(), s * (0.5 + 127 * 8 * U)
    assert bool((off <= bound).all()), what + ": int8 rows"


NORM_COLS = [1, 2, 3, 7, 8, 9, 15, 16, 17, 63, 64, 65, 96, 127, 128, 129, 192, 255, 256, 257, 384, 511, 512, 513, 768, 1000, 1025, 2047, 2048, 2049,
             4095, 4096, 4097, 5003, 8191, 8192, 8193, 16383, 16384, 16385, 32767, 32768]


@pytest.mark.parametrize("C", NORM_COLS)
def test_norm(ivit, C):
    import torch
    for i, t in enumerate(TYPES):
        for rows, res, i8, with_gamma in ((1, True, True, True), (5, False, True, True), (67, True, False, True), (33, True, True, False)):
            g = gen(1000 * C + i)
            x, r = rand(g, rows, C).to(dtype(t)), rand(g, rows, C).to(dtype(t)) if res else None
            gamma = 1.0 + 0.2 * rand(g, C) if with_gamma else None
            total = torch.empty_like(x) if res else None
            y = torch.empty((rows, C), dtype=torch.int8 if i8 else dtype(t), device="cuda")
            scale = torch.empty(rows, device="cuda") if i8 else None
            assert ivit.ivit_rmsnorm_quant(x, gamma, y, scale, 1e-5, residual=r, sum_out=total) is y
            check_norm(x, r, gamma, 1e-5, t, total, y, scale, "norm %d x %d %s" % (rows, C, t))


def guarded(rows, cols, ld, dt, value, shift=0):
    """A [rows, cols] view with ld elements between rows, `shift` elements into a buffer filled with `value`; (view, buffer, mask of what is not the view's)"""
    import torch
    buf = torch.full((shift + rows * ld + 64,), value, dtype=dt, device="cuda")
    view = buf[shift:shift + rows * ld].view(rows, ld)[:, :cols] if rows else buf[:0].view(0, cols)
    outside = torch.ones(buf.numel(), dtype=torch.bool, device="cuda")
    outside[shift:shift + rows * ld].view(rows, ld)[:, :cols] = False
    return view, buf, outside


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [1, 5, 12, 100, 384, 777, 2049, 6000, 20000])
def test_norm_strides_alignment_and_what_is_not_its_own(ivit, t, C):
    import torch
    g, rows = gen(C), 13
    x, _, _ = guarded(rows, C, C + 3, dtype(t), 0, shift=1)
    r, _, _ = guarded(rows, C, C + 5, dtype(t), 0, shift=3)
    total, tb, to = guarded(rows, C, C + 1, dtype(t), 7, shift=5)
    y, yb, yo = guarded(rows, C, C + 9, torch.int8, 77, shift=3)
    scale, sb, so = guarded(1, rows, rows, torch.float32, 7, shift=1)
    x.copy_(rand(g, rows, C)); r.copy_(rand(g, rows, C))
    gamma = rand(g, C)
    ivit.ivit_rmsnorm_quant(x, gamma, y, scale[0], 1e-6, residual=r, sum_out=total)
    check_norm(x, r, gamma, 1e-6, t, total, y, scale[0], "norm with strides")
    assert bool((tb[to] == 7).all()) and bool((yb[yo] == 77).all()) and bool((sb[so] == 7).all())


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [3, 200, 1001, 4099, 9000])
def test_norm_in_place(ivit, t, C):
    import torch
    g, rows = gen(C + 1), 301
    x, r, gamma = rand(g, rows, C).to(dtype(t)), rand(g, rows, C).to(dtype(t)), rand(g, C)
    want = torch.empty((rows, C), dtype=torch.int8, device="cuda"); ws = torch.empty(rows, device="cuda"); wt = torch.empty_like(x)
    ivit.ivit_rmsnorm_quant(x, gamma, want, ws, 1e-6, residual=r, sum_out=wt)
    for into_x in (True, False):
        a, b = x.clone(), r.clone()
        y, s = torch.empty_like(want), torch.empty_like(ws)
        ivit.ivit_rmsnorm_quant(a, gamma, y, s, 1e-6, residual=b, sum_out=a if into_x else b)
        assert torch.equal(a if into_x else b, wt) and torch.equal(y, want) and torch.equal(s, ws)
    y = torch.empty_like(x)
    ivit.ivit_rmsnorm_quant(x, gamma, y, None, 1e-6)
    a = x.clone()
    ivit.ivit_rmsnorm_quant(a, gamma, a, None, 1e-6)
    assert torch.equal(a, y)


@pytest.mark.parametrize("C", [5, 300, 1001, 5000])
def test_norm_writes_over_both_its_inputs(ivit, C):
    """The sum over the residual, the result over x, and the other way round."""
    import torch
    g, rows = gen(C + 2), 700
    x, r, gamma = rand(g, rows, C).half(), rand(g, rows, C).half(), rand(g, C)
    y, total = torch.empty_like(x), torch.empty_like(x)
    ivit.ivit_rmsnorm_quant(x, gamma, y, None, 1e-6, residual=r, sum_out=total)
    for swap in (False, True):
        a, b = x.clone(), r.clone()
        ivit.ivit_rmsnorm_quant(a, gamma, b if swap else a, None, 1e-6, residual=b, sum_out=a if swap else b)
        assert torch.equal(b if swap else a, y) and torch.equal(a if swap else b, total)


def test_norm_of_odd_rows(ivit):
    """Zeros, NaN, infinities, the smallest and largest numbers: each row by itself, its neighbours untouched by it."""
    import torch
    for C in (5, 64, 385, 3000):
        x = rand(gen(C), 12, C)
        x[1] = 0.0
        x[3, C // 2] = float("nan")
        x[5, 0] = float("inf")
        x[6] = -0.0
        x[7] = 1e-38 * x[7].sign()
        x[8] *= 1e18 / 10
        x[9] = 3e38
        x[11, :-1] = 0.0
        y, s, total = torch.empty((12, C), dtype=torch.int8, device="cuda"), torch.empty(12, device="cuda"), torch.empty_like(x)
        ivit.ivit_rmsnorm_quant(x, None, y, s, 1e-6, residual=torch.zeros_like(x), sum_out=total)
        fine = [0, 2, 4, 8, 10, 11]
        check_norm(x[fine], None, None, 1e-6, "f32", total[fine], y[fine], s[fine], "rows beside odd ones")
        for i in (1, 6, 9):                                       # (row 9: the mean square is beyond the range)
            assert float(s[i]) == 0.0 and not bool(y[i].any())
        for i in (3, 5):
            assert math.isnan(float(s[i])) and not bool(y[i].any())
        assert abs(float(s[7]) * 127 / (1e-38 / 1e-3) - 1) < 1e-3 and bool((y[7].float() == 127 * x[7].sign()).all())
        assert torch.equal(total[[3, 5]].nan_to_num(9.0), x[[3, 5]].nan_to_num(9.0))
        n = torch.empty_like(x)
        ivit.ivit_rmsnorm_quant(x, None, n, None, 1e-6)
        assert not bool(n[[1, 6, 9]].any()) and bool(torch.isnan(n[3]).all()) and math.isnan(float(n[5, 0])) and not bool(n[5, 1:].any())


def test_a_sum_beyond_the_range_of_its_type(ivit):
    import torch
    x = torch.full((2, 40), 60000.0, dtype=torch.float16, device="cuda")
    x[1] = 1.0
    total, y, s = torch.empty_like(x), torch.empty((2, 40), dtype=torch.int8, device="cuda"), torch.empty(2, device="cuda")
    ivit.ivit_rmsnorm_quant(x, None, y, s, 1e-6, residual=x, sum_out=total)
    assert bool(torch.isinf(total[0]).all()) and bool((y == 127).all()) and abs(float(s[0]) * 127 - 1) < 1e-5


def test_no_rows(ivit):
    import torch
    e = lambda *s, d=torch.float32: torch.empty(s, dtype=d, device="cuda")
    ivit.ivit_rmsnorm_quant(e(0, 64), e(64), e(0, 64, d=torch.int8), e(0), 1e-6)
    ivit.ivit_gated_quant(e(0, 128), e(0, 64, d=torch.int8), e(0))
    ivit.ivit_linear_scaled(e(0, 64, d=torch.int8), e(0), torch.zeros((8, 64), dtype=torch.int8, device="cuda"), e(8), e(0, 8))
    torch.cuda.synchronize()


# ---------------------------------------------------------------------------------------------------------------- gate
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", [True, False])
def test_gate_every_activation(ivit, act, gated):
    import torch
    for t in TYPES:
        for C in (1, 7, 8, 50, 192, 1000, 1536, 5001):
            g, rows = gen(C), 37
            x = (2.5 * rand(g, rows, 2 * C if gated else C)).to(dtype(t))
            check_gate(ivit, x, rows, C, t, act, gated)


def check_gate(ivit, x, rows, C, t, act, gated):
    import torch
    y, s = torch.empty((rows, C), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    assert ivit.ivit_gated_quant(x, y, s, act=act, gated=gated) is y
    a = x[:, :C].double()
    u = x[:, C:].double() if gated else torch.ones_like(a)
    err = (OPS * U if act != "none" else U) * (a * u).abs() + 2.0 ** -126 * (1 + u.abs())
    check_q(y, s, act64(a, act) * u, err, "gate %s %d x %d %s" % (act, rows, C, t))


@pytest.mark.parametrize("C", [c for c in NORM_COLS if c > 100])
def test_gate_widths(ivit, C):
    for t in TYPES:
        for rows, gated in ((1, True), (70, True), (3, False)):
            check_gate(ivit, rand(gen(C), rows, 2 * C if gated else C).to(dtype(t)), rows, C, t, "silu", gated)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [1, 6, 33, 384, 1537, 6001, 20000])
def test_gate_strides_and_what_is_not_its_own(ivit, t, C):
    import torch
    rows = 11
    x, _, _ = guarded(rows, 2 * C, 2 * C + 3, dtype(t), 0, shift=3)
    y, yb, yo = guarded(rows, C, C + 5, torch.int8, 77, shift=1)
    s, sb, so = guarded(1, rows, rows, torch.float32, 7, shift=2)
    x.copy_(rand(gen(C), rows, 2 * C))
    ivit.ivit_gated_quant(x, y, s[0], act="gelu", gated=True)
    a, u = x[:, :C].double(), x[:, C:].double()
    check_q(y, s[0], act64(a, "gelu") * u, OPS * U * (a * u).abs() + 2.0 ** -126 * (1 + u.abs()), "gate with strides")
    assert bool((yb[yo] == 77).all()) and bool((sb[so] == 7).all())


def test_gate_of_odd_rows(ivit):
    import torch
    for C in (3, 64, 2000):
        x = rand(gen(C), 8, 2 * C)
        x[1] = 0.0
        x[2, 0] = float("nan")
        x[3, C] = float("inf"); x[3, 0] = 1.0
        x[4, :C] = -200.0                                          # the activation leaves nothing
        x[5] *= 1e-30
        x[6, :C] = 3e38; x[6, C:] = 3e38                            # products beyond the range
        y, s = torch.empty((8, C), dtype=torch.int8, device="cuda"), torch.empty(8, device="cuda")
        ivit.ivit_gated_quant(x, y, s, act="silu", gated=True)
        assert float(s[1]) == 0.0 and not bool(y[1].any())
        for i in (2, 3, 6):
            assert math.isnan(float(s[i])) and not bool(y[i].any())
        a, u = x[[0, 4, 7], :C].double(), x[[0, 4, 7], C:].double()
        check_q(y[[0, 4, 7]], s[[0, 4, 7]], act64(a, "silu") * u, OPS * U * (a * u).abs() + 2.0 ** -126 * (1 + u.abs()), "rows beside odd ones")
        # row 5: x/2 u of 1e-60 leaves 32 bits: zeros
        assert float(s[5]) == 0.0 and not bool(y[5].any())


# --------------------------------------------------------------------------------------------------------------- dense
def dense_case(seed, M, N, K, t, residual, bias, one, full_range=False):
    import torch
    g = gen(seed)
    x = torch.randint(-128, 128, (M, K), generator=g, device="cuda", dtype=torch.int8) if full_range else (rand(g, M, K) * 32).round().clamp(-127, 127).to(torch.int8)
    w = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int8) if full_range else (rand(g, N, K) * 32).round().clamp(-127, 127).to(torch.int8)
    d = dict(x=x, w=w, x_scale=(0.5 + torch.rand(1 if one else M, generator=g, device="cuda")) / 32,
             w_scale=(0.5 + torch.rand(N, generator=g, device="cuda")) / 32 / math.sqrt(K))
    d["bias"] = rand(g, N) if bias else None
    d["residual"] = rand(g, M, N).to(dtype(t)) if residual else None
    return d


def run_dense(ivit, d, t, act, step=None, y=None, **more):
    import torch
    M, N = d["x"].shape[0], d["w"].shape[0]
    if y is None:
        y = torch.full((M, N), 99, dtype=dtype(t), device="cuda")
    assert ivit.ivit_linear_scaled(d["x"], d["x_scale"], d["w"], d["w_scale"], y, bias=d["bias"], act=act, residual=d["residual"], y_step=step, **more) is y
    return y


def check_dense(d, y, t, act, step, what, rows=None):
    import torch
    x, xs, res = d["x"], d["x_scale"], d["residual"]
    if rows is not None:
        x, xs, res, y = x[rows], xs if xs.numel() == 1 else xs[rows], None if res is None else res[rows], y[rows]
    p = torch.mm(x.double(), d["w"].double().t().contiguous()) * xs.double().reshape(-1, 1) * d["w_scale"].double()
    b = d["bias"].double() if d["bias"] is not None else torch.zeros_like(p)
    v, err = act64(p + b, act), OPS * U * (p.abs() + b.abs())
    if step is not None:
        q = (v / step).clamp(-127, 127)
        assert bool(((y.double() - q).abs() <= 0.5 + err / step + 2 * U * 127).all()), what
        return
    if res is not None:
        v = v + res.double()
        err = err + U * res.double().abs()
    assert bool(((y.double() - v).abs() <= err + (half(t) + U) * v.abs() + tiny(t)).all()), what


DENSE = [(1, 1, 16), (1, 16, 64), (1, 4096, 1024), (1, 777, 80), (2, 33, 48), (3, 100, 4096), (5, 257, 8192), (8, 1000, 512), (15, 130, 112), (16, 384, 384),
         (17, 31, 16), (31, 65, 272), (32, 4100, 256), (33, 64, 128), (48, 512, 1040), (63, 63, 63 * 16), (64, 64, 64), (65, 129, 144), (96, 2000, 768),
         (100, 10, 65536), (127, 128, 256), (128, 127, 240), (129, 513, 384), (192, 96, 96), (197, 1536, 384), (200, 5000, 400), (255, 300, 2048),
         (256, 256, 128), (257, 255, 176), (300, 3, 1024), (394, 192, 192), (500, 1000, 1536), (777, 385, 32), (1000, 1000, 1008), (1024, 2048, 512),
         (2000, 16, 640), (2049, 513, 160), (3000, 768, 768), (4097, 1, 64), (5000, 1200, 208), (7000, 2600, 144), (12544, 576, 192)]


@pytest.mark.parametrize("M,N,K", DENSE)
def test_dense(ivit, M, N, K):
    rng = random.Random(M * 7 + N * 3 + K)
    for i, t in enumerate(("f32", "f16", "bf16", "i8")):
        act, res, bias, one = rng.choice(ACTS), t != "i8" and rng.random() < 0.6, rng.random() < 0.7, rng.random() < 0.3
        d = dense_case(i, M, N, K, t, res, bias, one)
        step = 0.037 if t == "i8" else None
        check_dense(d, run_dense(ivit, d, t, act, step), t, act, step, "%d x %d x %d %s %s" % (M, N, K, t, act))


# one tile of 64 x 64, 128 x 64, 128 x 128, 256 x 128, 256 x 256 a CU at most (of 256 CUs); several of 256 x 256, and of 128 x 128, one after
# the other in a workgroup; K that ends inside a stage, rows and channels that end inside a tile
DENSE_TILES = [(1001, 999, 1008), (1500, 1000, 800), (2990, 770, 784), (4001, 1099, 848), (4000, 3999, 1040), (8001, 6099, 784), (9000, 5003, 896), (20000, 1031, 80),
               (12000, 2051, 384)]


@pytest.mark.parametrize("M,N,K", DENSE_TILES)
@pytest.mark.parametrize("t", ("f32", "f16", "bf16", "i8"))
def test_dense_tiles(ivit, M, N, K, t):
    rng = random.Random(M + N + K)
    for act, res in (("none", t != "i8"), (rng.choice(ACTS), False)):
        d = dense_case(9, M, N, K, t, res, rng.random() < 0.7, rng.random() < 0.3)
        step = 0.037 if t == "i8" else None
        check_dense(d, run_dense(ivit, d, t, act, step), t, act, step, "%d x %d x %d %s %s" % (M, N, K, t, act))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("t", ("f32", "f16", "bf16", "i8"))
def test_dense_epilogues(ivit, act, t):
    for M, N, K in ((1, 96, 128), (40, 200, 176), (300, 333, 256), (600, 1100, 384)):
        for res, bias, one in ((True, True, False), (False, True, True), (True, False, True), (False, False, False)):
            if res and t == "i8":
                continue
            d = dense_case(3, M, N, K, t, res, bias, one)
            step = 0.05 if t == "i8" else None
            check_dense(d, run_dense(ivit, d, t, act, step), t, act, step, "%d x %d x %d" % (M, N, K))


@pytest.mark.parametrize("M,N,K", [(1, 40, 65536), (20, 70, 65536), (130, 100, 65536), (300, 260, 16384), (600, 520, 1024)])
def test_dense_full_range_of_int8(ivit, M, N, K):
    """All of -128 .. 127, and the largest sums there are: every term (-128)^2."""
    import torch
    d = dense_case(1, M, N, K, "f32", False, False, False, full_range=True)
    d["x"][0], d["w"][0], d["x"][M // 2], d["w"][N // 2] = -128, -128, 127, -128
    check_dense(d, run_dense(ivit, d, "f32", "none"), "f32", "none", None, "full range")


@pytest.mark.parametrize("M,N,K", [(1, 50, 96), (7, 33, 80), (40, 129, 144), (260, 200, 272), (700, 650, 400)])
@pytest.mark.parametrize("t", ("f32", "f16", "bf16", "i8"))
def test_dense_strides_and_what_is_not_its_own(ivit, M, N, K, t):
    import torch
    d = dense_case(2, M, N, K, t, t != "i8", True, False)
    xb = torch.full((M + 1, K + 48), 55, dtype=torch.int8, device="cuda")
    xv = xb[:M, 16:16 + K]
    xv.copy_(d["x"]); d["x"] = xv
    if t != "i8":
        r, _, _ = guarded(M, N, N + 5, dtype(t), 0, shift=3)
        r.copy_(d["residual"]); d["residual"] = r
    y, buf, outside = guarded(M, N, N + 7, dtype(t), 77, shift=1)
    step = 0.04 if t == "i8" else None
    run_dense(ivit, d, t, "silu", step, y=y)
    check_dense(d, y, t, "silu", step, "strides")
    assert bool((buf[outside] == 77).all())


@pytest.mark.parametrize("M,N,K", [(1, 100, 256), (9, 65, 96), (50, 300, 512), (900, 700, 384)])
@pytest.mark.parametrize("t", TYPES)
def test_dense_residual_in_place(ivit, M, N, K, t):
    import torch
    d = dense_case(4, M, N, K, t, True, True, False)
    want = run_dense(ivit, d, t, "gelu")
    y = d["residual"].clone()
    d["residual"] = y
    run_dense(ivit, d, t, "gelu", y=y)
    assert torch.equal(y, want)


def test_dense_passes_nan_and_infinity_where_they_belong(ivit):
    import torch
    for M, N, K in ((1, 40, 64), (30, 50, 128), (300, 270, 256)):
        d = dense_case(5, M, N, K, "bf16", True, True, False)
        clean = run_dense(ivit, d, "bf16", "silu")
        d["x_scale"][0] = float("nan")                             # as a norm gives it for a row with a NaN
        d["bias"][3] = float("inf")
        y = run_dense(ivit, d, "bf16", "silu")
        assert bool(torch.isnan(y[0]).all()) and (M == 1 or bool((y[1:, 3] == float("inf")).all()))
        rest = torch.ones_like(y, dtype=torch.bool); rest[0] = False; rest[:, 3] = False
        assert torch.equal(y[rest], clean[rest])
        d["residual"] = None
        q = run_dense(ivit, d, "i8", "none", 0.05)
        assert not bool(q[0].any()) and (M == 1 or bool((q[1:, 3] == 127).all()))


def test_dense_equal_calls_give_equal_bits(ivit):
    import torch
    for M, N, K in ((1, 4096, 4096), (16, 1000, 8192), (200, 1000, 2048), (3000, 1500, 512)):
        d = dense_case(6, M, N, K, "f32", True, True, False)
        a = run_dense(ivit, d, "f32", "gelu")
        for _ in range(3):
            assert torch.equal(a, run_dense(ivit, d, "f32", "gelu"))
        one = dict(d, x=d["x"][:1], x_scale=d["x_scale"][:1], residual=d["residual"][:1])      # a row does not depend on the others
        assert torch.equal(a[:1], run_dense(ivit, one, "f32", "gelu"))


@pytest.mark.parametrize("M,N,K,t", [(16411, 1091, 64, "f32"), (16411, 2053, 784, "bf16"), (33333, 1031, 784, "f16"), (33333, 2053, 64, "i8")])
def test_dense_large_results_equal_those_of_their_parts(ivit, M, N, K, t):
    """Results of 64 MB and more, which are stored another way, against calls for a part of the rows: the same bits; a residual in place."""
    import torch
    d = dense_case(8, M, N, K, t, t != "i8", True, False)
    step = 0.05 if t == "i8" else None
    y, buf, outside = guarded(M, N, N + 5, dtype(t), 77, shift=1)
    rows = [(0, 300), (M // 2 - 7, M // 2 + 450), (M - 301, M)]
    part = lambda a, b: dict(d, x=d["x"][a:b], x_scale=d["x_scale"][a:b], residual=None if t == "i8" else d["residual"][a:b])
    want = [run_dense(ivit, part(a, b), t, "silu", step) for a, b in rows]
    run_dense(ivit, d, t, "silu", step, y=y)
    assert all(torch.equal(y[a:b], w) for (a, b), w in zip(rows, want))
    assert bool((buf[outside] == 77).all())
    if t != "i8":
        whole = y.clone()
        y.copy_(d["residual"])
        run_dense(ivit, dict(d, residual=y), t, "silu", y=y)
        assert torch.equal(y, whole) and bool((buf[outside] == 77).all())


@pytest.mark.parametrize("rows,C,t,gated", [(5003, 2049, "bf16", True), (9001, 1023, "f32", False), (2100, 4099, "f16", True)])
def test_gate_of_many_rows_equals_that_of_its_parts(ivit, rows, C, t, gated):
    """32 MB and more, which are loaded another way (16-bit rows of the last case: 34 MB), against calls for a part of the rows."""
    import torch
    x = rand(gen(rows), rows, C * (1 + gated)).to(dtype(t))
    q = torch.empty(rows, C, dtype=torch.int8, device="cuda"); s = torch.empty(rows, device="cuda")
    ivit.ivit_gated_quant(x, q, s, act="gelu", gated=gated)
    for a, b in ((0, 700), (rows // 2 + 3, rows // 2 + 900), (rows - 517, rows)):
        p = torch.empty(b - a, C, dtype=torch.int8, device="cuda"); ps = torch.empty(b - a, device="cuda")
        ivit.ivit_gated_quant(x[a:b], p, ps, act="gelu", gated=gated)
        assert torch.equal(q[a:b], p) and torch.equal(s[a:b], ps)


def test_offsets_beyond_32_bits(ivit):
    """Results and rows more than 2^32 bytes from the first one."""
    import torch
    M, N, K = 70001, 40000, 16
    d = dense_case(7, M, N, K, "bf16", False, True, False)
    y = run_dense(ivit, d, "bf16", "none")
    at = torch.tensor([0, 1, 26843, 26844, 53687, 53688, 60000, M - 1], device="cuda")      # 53687 x 40000 x 2 bytes is just below 2^32
    check_dense(d, y, "bf16", "none", None, "long results", rows=at)
    q, s = torch.empty((M, N // 2), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    ivit.ivit_gated_quant(y, q, s, act="silu", gated=True)
    a, u = y[at, :N // 2].double(), y[at, N // 2:].double()
    check_q(q[at], s[at], act64(a, "silu") * u, OPS * U * (a * u).abs() + 2.0 ** -126 * (1 + u.abs()), "gate of long results")
    n, sn = torch.empty((M, N // 2), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    half_rows = y[:, :N // 2]
    ivit.ivit_rmsnorm_quant(half_rows, None, n, sn, 1e-6, sum_out=half_rows)
    check_norm(half_rows[at], None, None, 1e-6, "bf16", None, n[at], sn[at], "norm of long results")
    del y, q, n
    # x with more than 2^32 bytes, rows 2^16 bytes apart
    M, ld = 66000, 1 << 16
    xb = torch.zeros((M, ld), dtype=torch.int8, device="cuda")
    d = dense_case(8, M, 40, 64, "f32", False, False, True)
    xv = xb[:, 128:192]
    xv.copy_(d["x"]); d["x"] = xv
    check_dense(d, run_dense(ivit, d, "f32", "none"), "f32", "none", None, "x far apart")


def test_rows_of_more_than_one_launch(ivit):
    """More rows than one grid has threads for: 2^31 threads are 2^23 rows of 256 threads, 2^28 rows of x in tiles of 64 rows and 256 threads."""
    import torch
    rows, C = (1 << 23) + 9, 2048
    at = torch.tensor([0, 1, (1 << 23) - 1, 1 << 23, rows - 1], device="cuda")
    x = torch.zeros((rows, C), dtype=torch.bfloat16, device="cuda")
    x[at] = rand(gen(1), at.numel(), C).to(x.dtype)
    q, s = torch.full((rows, C), 77, dtype=torch.int8, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    ivit.ivit_rmsnorm_quant(x, None, q, s, 1e-6)
    check_norm(x[at], None, None, 1e-6, "bf16", None, q[at], s[at], "norm of many rows")
    assert int((s != 0).sum()) == at.numel() and int(torch.count_nonzero(s)) == at.numel()
    q.fill_(77); s.fill_(7.0)
    ivit.ivit_gated_quant(x, q, s, act="silu", gated=False)
    a = x[at].double()
    check_q(q[at], s[at], act64(a, "silu"), OPS * U * a.abs() + 2.0 ** -126, "gate of many rows")
    assert int(torch.count_nonzero(s)) == at.numel()
    del x, q, s
    M = (1 << 28) + 100
    d = dict(x=torch.zeros((M, 16), dtype=torch.int8, device="cuda"), x_scale=torch.rand(M, device="cuda"), bias=rand(gen(2), 16), residual=None,
             w=torch.randint(-127, 128, (16, 16), device="cuda", dtype=torch.int8), w_scale=torch.rand(16, device="cuda"))
    at = torch.tensor([0, 63, (1 << 28) - 1, 1 << 28, M - 1], device="cuda")
    d["x"][at] = torch.randint(-127, 128, (at.numel(), 16), device="cuda", dtype=torch.int8)
    y = run_dense(ivit, d, "i8", "none", 20.0)
    check_dense(d, y, "i8", "none", 20.0, "many rows", rows=at)
    base = (d["bias"] / 20.0).round().to(torch.int8)
    assert int((y != base).any(1).sum()) <= at.numel()


# -------------------------------------------------------------------------------------------------- streams, capture, together
class Block:
    """One pre-norm encoder block of real scales around the integer attention, every intermediate kept."""

    def __init__(self, B, T, C, H, F, t, gated, seed):
        import torch
        g = gen(seed)
        self.d, self.t, self.gated = dict(B=B, T=T, C=C, H=H, F=F), t, gated
        R = B * T

        def weights(n, k):
            w = rand(g, n, k)
            s = w.abs().amax(1) / 127
            return (w / s[:, None]).round().to(torch.int8), s / math.sqrt(k)

        e = lambda n, d: torch.empty((R, n), dtype=d, device="cuda")
        i8, f = torch.int8, dtype(t)
        self.x, self.delta = rand(g, R, C).to(f), rand(g, R, C).to(f)
        self.g1, self.g2 = 1 + 0.1 * rand(g, C), 1 + 0.1 * rand(g, C)
        self.qkv_w, self.proj_w, self.fc1_w, self.fc2_w = weights(3 * C, C), weights(C, C), weights(F * (2 if gated else 1), C), weights(C, F)
        self.b_qkv, self.b1 = 0.1 * rand(g, 3 * C), 0.1 * rand(g, F * (2 if gated else 1))
        self.h0, self.h1, self.out = e(C, f), e(C, f), e(C, f)
        self.u, self.v, self.hid, self.o, self.qkv, self.fc1 = e(C, i8), e(C, i8), e(F, i8), e(C, i8), e(3 * C, i8), e(F * (2 if gated else 1), f)
        self.su, self.sv, self.sh = (torch.empty(R, device="cuda") for _ in range(3))
        self.o_scale = torch.full((1,), 1.0 / 32.0, device="cuda")
        self.step = 1.0 / 32.0
        # scores of 1/32 1/32 sum / sqrt(d), taken at 1/32: a factor of 1 / (32 sqrt d); probabilities of 1/128 times values of 1/32
        self.qk_rq, self.pv_rq, self.sm = (round(2 ** 20 / (32 * math.sqrt(C // H))), 20), (2 ** 14, 21), synth.shift_params(32)

    def run(self, ivit, stream=None):
        n = dict(stream=stream)
        ivit.ivit_rmsnorm_quant(self.x, self.g1, self.u, self.su, 1e-6, residual=self.delta, sum_out=self.h0, **n)
        ivit.ivit_linear_scaled(self.u, self.su, *self.qkv_w, self.qkv, bias=self.b_qkv, y_step=self.step, **n)
        ivit.ivit_attention(self.qkv, self.o, self.d, self.qk_rq, self.sm, self.pv_rq, **n)
        ivit.ivit_linear_scaled(self.o, self.o_scale, *self.proj_w, self.h1, residual=self.h0, **n)
        ivit.ivit_rmsnorm_quant(self.h1, self.g2, self.v, self.sv, 1e-6, **n)
        ivit.ivit_linear_scaled(self.v, self.sv, *self.fc1_w, self.fc1, bias=self.b1, **n)
        ivit.ivit_gated_quant(self.fc1, self.hid, self.sh, act="silu" if self.gated else "gelu", gated=self.gated, **n)
        ivit.ivit_linear_scaled(self.hid, self.sh, *self.fc2_w, self.out, residual=self.h1, **n)

    def outputs(self):
        return [self.h0, self.u, self.su, self.qkv, self.o, self.h1, self.v, self.sv, self.fc1, self.hid, self.sh, self.out]

    def check(self):
        import torch
        t, F = self.t, self.d["F"]
        check_norm(self.x, self.delta, self.g1, 1e-6, t, self.h0, self.u, self.su, "norm 1")
        dn = lambda x, s, w, b, r: dict(x=x, x_scale=s, w=w[0], w_scale=w[1], bias=b, residual=r)
        check_dense(dn(self.u, self.su, self.qkv_w, self.b_qkv, None), self.qkv, "i8", "none", self.step, "qkv")
        want = orc.attention(self.qkv.cpu().numpy(), self.d, self.qk_rq, self.sm, self.pv_rq)
        want = want[0] if isinstance(want, tuple) else want
        assert np.array_equal(self.o.cpu().numpy(), want)
        check_dense(dn(self.o, self.o_scale, self.proj_w, None, self.h0), self.h1, t, "none", None, "proj")
        check_norm(self.h1, None, self.g2, 1e-6, t, None, self.v, self.sv, "norm 2")
        check_dense(dn(self.v, self.sv, self.fc1_w, self.b1, None), self.fc1, t, "none", None, "fc1")
        a = self.fc1[:, :F].double()
        u = self.fc1[:, F:].double() if self.gated else torch.ones_like(a)
        check_q(self.hid, self.sh, act64(a, "silu" if self.gated else "gelu") * u, OPS * U * (a * u).abs() + 2.0 ** -126 * (1 + u.abs()), "gate")
        check_dense(dn(self.hid, self.sh, self.fc2_w, None, self.h1), self.out, t, "none", None, "fc2")


@pytest.mark.parametrize("B,T,C,H,F,t,gated", [(1, 1, 64, 2, 256, "bf16", True), (1, 65, 64, 2, 256, "f32", False), (3, 197, 192, 3, 768, "bf16", False),
                                               (2, 197, 384, 6, 1024, "f16", True), (5, 49, 96, 3, 384, "bf16", True)])
def test_a_block_of_them_together(ivit, B, T, C, H, F, t, gated):
    import torch
    b = Block(B, T, C, H, F, t, gated, 11)
    b.run(ivit)
    torch.cuda.synchronize()
    b.check()
    assert bool((b.out != b.h1).any()) and bool((b.h1 != b.h0).any())


def test_a_block_on_another_stream_and_replayed_from_a_graph(ivit):
    """On a stream of its own, given and current, and captured: every replay on new inputs is what the eager calls give."""
    import torch
    b = Block(2, 49, 64, 2, 256, "bf16", True, 12)
    b.run(ivit)
    torch.cuda.synchronize()
    want = [v.clone() for v in b.outputs()]
    s = torch.cuda.Stream()
    for how in ("given", "current"):
        for v in b.outputs():
            v.zero_()
        torch.cuda.synchronize()
        if how == "given":
            b.run(ivit, stream=s)
        else:
            with torch.cuda.stream(s):
                b.run(ivit)
        s.synchronize()
        assert all(torch.equal(v, w) for v, w in zip(b.outputs(), want)), how
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run(ivit)
    for k in range(4):
        x = rand(gen(50 + k), *b.x.shape).to(b.x.dtype)
        b.x.copy_(x)
        b.run(ivit)
        torch.cuda.synchronize()
        eager = [v.clone() for v in b.outputs()]
        for v in b.outputs():
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(v, w) for v, w in zip(b.outputs(), eager)), "replay %d" % k
        b.check()


def test_two_streams_at_once(ivit):
    import torch
    blocks = [Block(2, 65, 64, 2, 256, t, True, 20 + i) for i, t in enumerate(("bf16", "f32"))]
    want = []
    for b in blocks:
        b.run(ivit)
        torch.cuda.synchronize()
        want.append([v.clone() for v in b.outputs()])
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(20):
        for b, s in zip(blocks, streams):
            b.run(ivit, stream=s)
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        assert all(torch.equal(v, z) for v, z in zip(b.outputs(), w))


def test_trace_names_the_launches(ivit):
    import torch
    b = Block(1, 49, 64, 2, 256, "bf16", True, 30)
    ivit.ivit_trace_begin(32)
    b.run(ivit)
    rec = ivit.ivit_trace_end(32)
    assert [ivit.KIND_NAMES[r[1]] for r in rec] == ["rmsnorm", "gemm_scaled", "attention", "gemm_scaled", "rmsnorm", "gemm_scaled", "gated", "gemm_scaled"]
    assert all(r[0] > 0 and r[3] > 0 for r in rec) and rec[1][2] == 2 * 49 * 192 * 64


def test_refusals_on_the_gpu(ivit):
    import torch
    z = lambda *s, d=torch.float32: torch.zeros(s, dtype=d, device="cuda")
    with pytest.raises(ivit.IvitError) as err:                      # rows of x that are not a multiple of 16 bytes apart
        ivit.ivit_linear_scaled(z(4, 72, d=torch.int8)[:, :64], z(4), z(8, 64, d=torch.int8), z(8), z(4, 8))
    assert err.value.status == ivit.IVIT_ERR_SHAPE
    with pytest.raises(ivit.IvitError) as err:
        ivit.ivit_rmsnorm_quant(z(4, 64), None, z(4, 64, d=torch.int8), z(4), 0.0)
    assert err.value.status == ivit.IVIT_ERR_PARAM
    with pytest.raises(ValueError):
        ivit.ivit_linear_scaled(z(4, 64, d=torch.int8), z(4), z(8, 64, d=torch.int8), z(8).cpu(), z(4, 8))
    with pytest.raises(ValueError):
        ivit.ivit_gated_quant(z(4, 128).cpu(), z(4, 64, d=torch.int8), z(4))
    torch.cuda.synchronize()
