"""What the tests of attention over float rows share: inputs, the definitions in 64 bits and how far results may be from them.

U = 2^-24 is half a unit of a 32-bit value's last place, HALF[type] half a step of a type.  With weights w_j of relative errors e_j and the sum of the same
weights below, an output is off by at most max e (sum_j p_j |v_j| + |o|).  e: the score's error times its factor (its d products are exact in 32 bits and
summed with d roundings of at most sum |q k| each; the exponent's argument and the largest score are rounded, 4 U of either), 4 U of the power, and
the weight's own rounding.  Sums of n values add n U (sum_j p_j |v_j|), their quotient 4 U, the result's rounding half a step.  float16 weights below the normal numbers lose at most
2^-25 where the sum is 2^7 at least: 2^-32 a key."""
import math

U = 2.0 ** -24


def dtype(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}[name]


def half(name):
    import torch
    return torch.finfo(dtype(name)).eps / 2


def gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rand(g, *shape):
    import torch
    return torch.randn(shape, generator=g, device="cuda")


def attend64(q, k, v, scale, hidden=None):
    """q [n, d], k, v [m, d] of 64 bits, hidden [n, m] -> (o, sum of p |v|, the largest error of a score times scale, sum of (p (|v| + |o|))^2)"""
    import torch
    if k.shape[0] == 0:
        z = torch.zeros_like(q)
        return z, z, z[:, :1], z
    d, kt = q.shape[1], k.t().contiguous()
    s = torch.mm(q, kt) * scale
    size = torch.mm(q.abs(), kt.abs()) * scale
    if hidden is not None:
        s = s.masked_fill(hidden, -math.inf)
        size = size.masked_fill(hidden, 0.0)
    top = s.amax(1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(1, keepdim=True)
    p = torch.where(total > 0, p / total, torch.zeros_like(p))
    # a key left out takes no part whatever it holds
    gone = torch.zeros_like(v) if hidden is None else torch.where(hidden.all(0)[:, None], torch.zeros_like(v), v)
    v = v if hidden is None else torch.where(hidden.all(0)[:, None], gone, v)
    o, pv = torch.mm(p, v), torch.mm(p, v.abs())
    err = ((d + 8) * U * size).amax(1, keepdim=True)
    spread = torch.mm(p * p, v * v) + 2 * torch.mm(p * p, v.abs()) * o.abs() + (p * p).sum(1, keepdim=True) * o * o
    return o, pv, err, spread


def check(o, want, pv, err, n, t, most, what, scaled=0.0):
    """o against its definition: n keys, values of at most `most`, err the scores' largest error"""
    import torch
    # twice the score's error: the largest score's counts too
    e = half(t) + 2 * err + 8 * U + scaled
    bound = (e + n * U + 4 * U) * (pv + want.abs()) + half(t) * want.abs() + n * 2.0 ** -32 * most + (2.0 ** -25 if t == "f16" else 2.0 ** -125)
    off = (o.double() - want).abs()
    assert bool((off <= bound).all()), "%s: %g over" % (what, float((off - bound).nan_to_num(math.inf).max()))


def check_mean(o, want, spread, t, what):
    """The mean square error of many results: rounding errors of weights and results are independent, at most half a step and of a mean square of a third of
    its square; a half more for what the mean of so many may be off, and for the other errors, which are far below."""
    e2 = half(t) ** 2 / 3
    got, most = float(((o.double() - want) ** 2).mean()), float((e2 * spread + e2 * want * want).mean())
    assert got <= 1.5 * most, "%s: mean square error %g, expected at most %g" % (what, got, most)
