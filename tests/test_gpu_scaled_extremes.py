"""The float layers at the ends of their ranges: infinite values, the tails of the activations, numbers whose squares or products leave 32 bits.

U = 2^-24 is half a unit of a 32-bit value's last place."""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = ("f32", "f16", "bf16")
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh", "gelu_sigmoid")


def dtype(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}[name]


def gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ----------------------------------------------------------------------------------------------------- infinite values
def at_minus_infinity(act):
    return {"none": -math.inf, "relu": 0.0}.get(act, math.nan)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", [True, False])
def test_infinite_hidden_values_mark_their_row(ivit, act, gated):
    import torch
    for t in TYPES:
        for C in (3, 64, 1000, 5001):
            x = torch.randn((6, 2 * C if gated else C), generator=gen(C), device="cuda").to(dtype(t))
            x[1, 0], x[1, C // 2], x[4, C - 1] = 2.0, -math.inf, math.inf
            if gated:
                x[1, C] = x[1, C + C // 2] = x[4, 2 * C - 1] = 1.0
            q, s = torch.full((6, C), 99, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
            ivit.ivit_gated_quant(x, q, s, act=act, gated=gated)
            fine = act == "relu"                        # max(-inf, 0) is 0: that row is an ordinary one
            assert bool(torch.isfinite(s[[0, 2, 3, 5]]).all()) and bool(torch.isfinite(s[1])) == fine and bool(torch.isnan(s[4]))
            assert not bool(q[4].any()) and (fine or not bool(q[1].any()))
            if fine:
                assert int(q[1, C // 2]) == 0 and int(q[1].abs().max()) == 127


@pytest.mark.parametrize("act", ACTS)
def test_infinite_sums_of_the_dense(ivit, act):
    import torch
    for t in TYPES + ("i8",):
        for M, N, K in ((1, 40, 64), (30, 50, 128), (300, 270, 256), (1200, 1300, 96)):
            g = gen(M)
            x = torch.randint(-127, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
            w = torch.randint(-127, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
            bias = torch.randn(N, generator=g, device="cuda")
            bias[3], bias[N - 1] = -math.inf, math.inf
            y = torch.full((M, N), 99, dtype=dtype(t), device="cuda")
            ivit.ivit_linear_scaled(x, torch.full((M,), 1e-3, device="cuda"), w, torch.full((N,), 1e-2, device="cuda"), y, bias=bias, act=act,
                                    y_step=0.05 if t == "i8" else None)
            low = at_minus_infinity(act)
            if t == "i8":
                assert bool((y[:, N - 1] == 127).all()) and bool((y[:, 3] == (-127 if act == "none" else 0)).all())
            else:
                assert bool((y[:, N - 1] == math.inf).all())
                assert bool((torch.isnan(y[:, 3]) if math.isnan(low) else y[:, 3] == low).all())
                rest = torch.ones(N, dtype=torch.bool, device="cuda"); rest[3] = rest[N - 1] = False
                assert bool(torch.isfinite(y[:, rest]).all())


# -------------------------------------------------------------------------------------------------- tails of activations
def exactly(x, act):
    """In 64 bits, the tails to their last places."""
    import torch
    x = x.double()
    if act == "gelu":
        return 0.5 * x * torch.special.erfc(-x / math.sqrt(2.0))
    slope = {"silu": x, "gelu_sigmoid": 1.702 * x, "gelu_tanh": 2.0 * math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)}[act]
    return x / (1.0 + torch.exp(-slope))


def share(x):
    """The stated error of an activation, relative to its value."""
    x = x.double().abs()
    return (12 + 10 * x + x ** 3) * U


TAILS = [("gelu", -9, -4), ("gelu", -12, -8), ("gelu", -4, -1), ("gelu", -1e-3, 0), ("silu", -80, -20), ("gelu_tanh", -8, -4), ("gelu_sigmoid", -45, -10)]


def between(lo, hi, shape, t, seed):
    import torch
    return (lo + (hi - lo) * torch.rand(shape, generator=gen(seed), device="cuda")).to(dtype(t))


def check_rows(q, s, v, rel, more):
    """int8 rows of values known to within rel |v| + more; the quotient's 3 U"""
    import torch
    top, at = v.abs().max(1)
    rel_top = rel.gather(1, at[:, None])[:, 0]
    err_top = rel_top * top + more
    # another element may have come out as the largest, if it is within both errors: its own error counts then
    err_top = torch.maximum(err_top, (rel * v.abs()).amax(1) + more)
    assert bool(((s.double() - top / 127).abs() <= err_top / 127 + 3 * U * top / 127).all()), "scale"
    off, step = (q.double() * (top / 127)[:, None] - v).abs(), (top / 127)[:, None]
    assert bool((off <= 0.5 * step * (1 + 8 * U) + rel * v.abs() + more[:, None] + err_top[:, None] / top[:, None] * v.abs()).all()), "rows"


@pytest.mark.parametrize("act,lo,hi", TAILS)
@pytest.mark.parametrize("gated", [True, False])
def test_rows_that_lie_in_the_tail_have_scales_of_their_own(ivit, act, lo, hi, gated):
    import torch
    for t in TYPES:
        if t == "f16" and act == "gelu" and lo == -1e-3:
            continue                                    # (below its normal numbers)
        for C in (3, 64, 200, 1000, 2049, 5001, 20000):
            rows = 37
            g = between(lo, hi, (rows, C), t, C)
            x = torch.cat([g, torch.randn((rows, C), generator=gen(C + 1), device="cuda").to(dtype(t))], 1) if gated else g
            q, s = torch.full((rows, C), 99, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
            ivit.ivit_gated_quant(x, q, s, act=act, gated=gated)
            v = exactly(g, act) * (x[:, C:].double() if gated else 1.0)
            more = torch.zeros(rows, dtype=torch.float64, device="cuda")
            if act == "gelu":                           # (rows whose largest is no less than an eighth of what goes into it)
                wide = (x[:, C:].double().abs().amax(1) if gated else 1.0) * g.double().abs().amax(1)
                more = torch.where(8 * v.abs().amax(1) >= 0.5 * wide, v.abs().amax(1) * 2.0 ** -20, more)
            check_rows(q, s, v, share(g) + U, more)


@pytest.mark.parametrize("gated", [True, False])
def test_rows_with_some_values_in_the_tail(ivit, gated):
    import torch
    for C in (7, 100, 1536, 5001):
        rows = 70
        g = between(-9, -3, (rows, C), "f32", C)
        g[::2, C // 2] = 10.0 ** torch.linspace(-5, 1, 35, device="cuda")       # (largest values from the tail's size to ordinary ones, by turns)
        x = torch.cat([g, torch.ones_like(g)], 1) if gated else g
        q, s = torch.full((rows, C), 99, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
        ivit.ivit_gated_quant(x, q, s, act="gelu", gated=gated)
        v = exactly(g, "gelu")
        check_rows(q, s, v, share(g) + U, v.abs().amax(1) * 2.0 ** -20)
        # a row's values do not depend on its neighbours
        one, s1 = torch.empty((1, C), dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
        for r in (0, 1, 34, 68, 69):
            ivit.ivit_gated_quant(x[r:r + 1], one, s1, act="gelu", gated=gated)
            assert torch.equal(one[0], q[r]) and float(s1) == float(s[r])


@pytest.mark.parametrize("act,lo,hi", TAILS)
@pytest.mark.parametrize("t", TYPES)
def test_tails_in_the_epilogue_of_the_dense(ivit, act, lo, hi, t):
    """Sums of 0, so that the bias alone, known exactly, goes into the activation."""
    import torch
    half = torch.finfo(dtype(t)).eps / 2
    least = {"f32": 2.0 ** -118, "f16": 2.0 ** -25, "bf16": 2.0 ** -118}[t]
    for M, N, K in ((1, 200, 64), (16, 2000, 512), (40, 515, 128), (300, 270, 256), (1200, 1300, 96), (4000, 2100, 1024), (20000, 1031, 80)):
        bias = between(lo, hi, (N,), "f32", N)
        y = torch.full((M, N), 99, dtype=dtype(t), device="cuda")
        ivit.ivit_linear_scaled(torch.zeros((M, K), dtype=torch.int8, device="cuda"), torch.ones(M, device="cuda"), torch.ones((N, K), dtype=torch.int8, device="cuda"),
                                torch.ones(N, device="cuda"), y, bias=bias, act=act)
        v = exactly(bias, act)
        err = share(bias) * v.abs() if t == "f32" or act != "gelu" else 2.0 ** -23 * bias.double().abs()
        assert bool(((y.double() - v).abs() <= err + half * (v.abs() + err) + least).all()), (M, N, K)


# ------------------------------------------------------------------------------------------- the norm's sums and products
WIDTHS = [5, 64, 100, 500, 1000, 1536, 2049, 4096, 6000, 12000, 32768]


def norm_of(ivit, x, gamma, eps, i8):
    import torch
    y = torch.full(x.shape, 99, dtype=torch.int8 if i8 else x.dtype, device="cuda")
    s = torch.empty(x.shape[0], device="cuda") if i8 else None
    total = torch.empty_like(x)
    ivit.ivit_rmsnorm_quant(x, gamma, y, s, eps, residual=torch.zeros_like(x), sum_out=total)
    assert torch.equal(total, x)
    return y, s


def check_normed(y, s, x, gamma, eps, what):
    """Against 64 bits: half of the error of a sum of squares in chains of 32 and a tree of 10, the root, the quotient, two products; the rounding of the result."""
    import torch
    h = x.double()
    n = h / ((h * h).mean(1, keepdim=True) + eps).sqrt()
    n = n if gamma is None else n * gamma.double()
    rel = ((32 + 10 + 3) / 2 + 8) * U
    if s is None:
        half = torch.finfo(y.dtype).eps / 2
        assert bool(((y.double() - n).abs() <= (rel + half + rel * half) * n.abs() + 2.0 ** -133).all()), what
        return
    top = n.abs().amax(1)
    assert bool(((s.double() - top / 127).abs() <= (rel + 2 * U) * top / 127 + 2.0 ** -149).all()), what + ": scale"
    assert bool(((y.double() * (top / 127)[:, None] - n).abs() <= (top / 127)[:, None] * (0.5 + 127 * 8 * U)).all()), what + ": rows"


@pytest.mark.parametrize("C", WIDTHS)
def test_sums_of_squares_beyond_the_range_of_32_bits(ivit, C):
    """Rows whose mean square is in the range and whose sum of squares is not, beside ordinary ones; and a mean square beyond it."""
    import torch
    for t in ("f32", "bf16"):
        z = torch.randn((9, C), generator=gen(C), device="cuda").clamp(-8, 8)
        z[:, 0] = 1.0
        z *= torch.tensor([1.0, 1e17, 4e17, 1e18, 1.0, 3e18, 8e18, 1e-3, 4e37], device="cuda")[:, None]
        x, gamma = z.to(dtype(t)), 1.0 + 0.1 * torch.randn(C, generator=gen(C + 1), device="cuda")
        for g in (None, gamma):
            for i8 in (True, False):
                y, s = norm_of(ivit, x, g, 1e-6, i8)
                check_normed(y[:8], s[:8] if i8 else None, x[:8], g, 1e-6, "%s %s" % (t, i8))
                assert not bool(y[8].any()) and (not i8 or float(s[8]) == 0.0)      # (counts as infinite)


def test_eps_counts_beside_large_sums(ivit):
    import torch
    x = torch.full((3, 4096), 4e17, device="cuda")
    for eps in (1e35, 3e38):
        for i8 in (True, False):
            y, s = norm_of(ivit, x, None, eps, i8)
            eps32 = float(torch.tensor(eps, dtype=torch.float32))
            check_normed(y, s, x, None, eps32, "eps %g" % eps)


@pytest.mark.parametrize("C", WIDTHS)
def test_products_with_gamma_beyond_the_range_of_32_bits(ivit, C):
    """h gamma beyond the range, or below the normal numbers, where n = h / rms gamma is not; rows of ordinary size with the same gamma."""
    import torch
    z = torch.randn((8, C), generator=gen(C), device="cuda").clamp(-6, 6)
    z[:, C // 2] = 2.0
    base = 1.0 + 0.1 * torch.randn(C, generator=gen(C + 1), device="cuda")
    for by, rows in ((1e30, [1.0, 1e12, 1e18, 1e-15, 0.0, 1e9, 3e18, 1.0]), (1e-30, [1.0, 1e-12, 1e-15, 1e10, 0.0, 3e-14, 1e-8, 1.0])):
        x = z * torch.tensor(rows, device="cuda")[:, None]
        gamma, eps = base * by, 1e-37
        for i8 in (True, False):
            y, s = norm_of(ivit, x, gamma, eps, i8)
            fine = [0, 1, 2, 3, 5, 6, 7]
            check_normed(y[fine], s[fine] if i8 else None, x[fine], gamma, eps, "gamma %g" % by)
            assert not bool(y[4].any()) and (not i8 or float(s[4]) == 0.0)


@pytest.mark.parametrize("C", [5, 64, 1000, 2049, 6000, 32768])
def test_results_beyond_the_range_of_32_bits(ivit, C):
    """The row's largest n beyond the range: NaN as its scale and zeros, and infinite where the result is of the stream's type."""
    import torch
    x = torch.ones((4, C), device="cuda")
    x[2] = 0.0                                              # n of one element: sqrt(C), of the others 0
    x[2, C // 2] = 1.0
    x[3] = 0.0
    gamma = torch.full((C,), 3e38, device="cuda")
    gamma[0], x[:, 0] = 1.0, torch.tensor([1.0, 1e-30, 0.0, 0.0], device="cuda")
    for scale in (1.0, 1e15):
        y, s = norm_of(ivit, x * scale, gamma, 1e-12, True)
        assert bool(torch.isnan(s[2])) and not bool(y[2].any()) and float(s[3]) == 0.0 and not bool(y[3].any())
        assert bool(torch.isfinite(s[:2]).all())
        y, _ = norm_of(ivit, x * scale, gamma, 1e-12, False)
        assert float(y[2, C // 2]) == math.inf and not bool(y[3].any())


# ------------------------------------------------------------------- such rows in place, with strides, and replayed from a graph
def odd_rows(rows, C, t, seed):
    """Ordinary rows, zeros, rows whose squares and products leave the range, tails, NaN and infinities, by turns."""
    import torch
    z = torch.randn((rows, C), generator=gen(seed), device="cuda")
    by = torch.tensor([1.0, 0.0, 1e18, 1.0, 2e-15, 1e17, 1.0, 30.0], device="cuda").repeat(rows // 8 + 1)[:rows]
    if t == "f16":
        by = by.clamp(0.0, 1e3)
    x = z * by[:, None]
    x[3::8] = -4.0 - 5.0 * torch.rand((len(range(3, rows, 8)), C), generator=gen(seed + 1), device="cuda")
    x[6::16, C // 3] = math.nan
    x[14::16, C // 2] = math.inf
    return x.to(dtype(t))


def same(a, b):
    import torch
    return torch.equal(a.nan_to_num(nan=7.0, posinf=8.0, neginf=9.0), b.nan_to_num(nan=7.0, posinf=8.0, neginf=9.0)) if a.is_floating_point() else torch.equal(a, b)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [5, 60, 130, 500, 1000, 2300, 4099, 9000])
def test_odd_rows_written_over_their_inputs(ivit, t, C):
    import torch
    rows = 67
    x, r = odd_rows(rows, C, t, C), (0.5 * odd_rows(rows, C, t, C + 9))
    r[::8] = 0.0
    for by in (1.0, 1e25, 1e-25):
        gamma = by * (1.0 + 0.1 * torch.randn(C, generator=gen(C + 3), device="cuda"))
        q, s, total, n = torch.empty((rows, C), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty_like(x)
        ivit.ivit_rmsnorm_quant(x, gamma, q, s, 1e-37, residual=r, sum_out=total)
        ivit.ivit_rmsnorm_quant(x, gamma, n, None, 1e-37, residual=r)
        for swap in (False, True):
            a, b = x.clone(), r.clone()
            q2, s2 = torch.full_like(q, 99), torch.empty_like(s)
            ivit.ivit_rmsnorm_quant(a, gamma, q2, s2, 1e-37, residual=b, sum_out=b if swap else a)
            assert same(b if swap else a, total) and same(q2, q) and same(s2, s)
            a, b = x.clone(), r.clone()
            ivit.ivit_rmsnorm_quant(a, gamma, b if swap else a, None, 1e-37, residual=b, sum_out=a if swap else b)
            assert same(b if swap else a, n) and same(a if swap else b, total)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [5, 60, 500, 2300, 9000])
def test_odd_rows_with_strides_and_from_a_graph(ivit, t, C):
    import torch
    rows, ld = 67, C + 3
    x = torch.zeros(1 + rows * 2 * ld, dtype=dtype(t), device="cuda")
    xn, xg = x[1:1 + rows * 2 * ld].view(rows, 2 * ld)[:, :C], x[1:1 + rows * 2 * ld].view(rows, 2 * ld)[:, :2 * C]
    xg.copy_(odd_rows(rows, 2 * C, t, C))
    gamma = 1e25 * (1.0 + 0.1 * torch.randn(C, generator=gen(C + 3), device="cuda"))
    bufs = [torch.full((rows, ld), 77, dtype=torch.int8, device="cuda") for _ in range(3)]
    s = [torch.empty(rows, device="cuda") for _ in range(3)]

    def run(y, a, b):
        ivit.ivit_rmsnorm_quant(a, gamma, y[0][:, :C], s[0], 1e-37)
        ivit.ivit_gated_quant(b, y[1][:, :C], s[1], act="gelu")
        ivit.ivit_gated_quant(a, y[2][:, :C], s[2], act="gelu", gated=False)

    run([torch.empty_like(v) for v in bufs], xn.contiguous(), xg.contiguous())
    torch.cuda.synchronize()
    want_s = [v.clone() for v in s]
    dense = [torch.full_like(v, 77) for v in bufs]
    run(dense, xn.contiguous(), xg.contiguous())
    run(bufs, xn, xg)
    assert all(torch.equal(a, b) for a, b in zip(bufs, dense)) and all(same(a, b) for a, b in zip(s, want_s))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(bufs, xn, xg)
    for k in range(3):
        xg.copy_(odd_rows(rows, 2 * C, t, C + 100 + k))
        run(dense, xn, xg)
        torch.cuda.synchronize()
        want_s = [v.clone() for v in s]
        for v in bufs + s:
            v.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bufs, dense)) and all(same(a, b) for a, b in zip(s, want_s))
