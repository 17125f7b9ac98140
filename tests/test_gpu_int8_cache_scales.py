"""Attention over an int8 cache whose value scales differ by more than float16 holds, against its definition in 64 bits.

The products of weights and value scales are rounded to float16: w_j s_j is off by 2^-11 of itself, or by 2^-25 in units in which the largest product of the row
is 2^7 at least, which is 2^-32 of the largest.  The sum of the weights is not rounded.  So an output sum_j w_j s_j q_j / sum_j w_j is off by at most
  2^-11 sum_j p_j |v_j| + n 2^-32 127 max_j p_j s_j
beside what tests/attention_rows.py counts for scores, 32-bit sums and the result's rounding; two products in 32 bits add 2 U."""
import math

import pytest

from attention_rows import U, half
from test_gpu_cached_attention import Setup

pytestmark = pytest.mark.gpu

HALF16 = 2.0 ** -11


def value_scales(s, b, h):
    """the scales of the values of request b's keys, in the order of Setup.keys"""
    import torch
    parts = []
    for table, count in ((s.prefix_pages, s.prefix), (s.pages[b], max(s.lens_[b], 0))):
        if count:
            parts.append(s.cache["v_scale"][table[:-(-count // s.page)].long(), h].double().reshape(-1)[:count])
    return torch.cat(parts)


def compare(s, what, mean=False, requests=None):
    import torch
    d, group = s.d, s.H // s.G
    sums = [0.0, 0.0, 0]
    for b, n in enumerate(s.lens_):
        if n < 0 or (requests is not None and b not in requests):
            continue
        for h in range(s.G):
            k, v = s.keys(b, h)
            n = k.shape[0]
            if n == 0:
                continue
            sv = value_scales(s, b, h)
            cols = slice(h * group * d, (h + 1) * group * d)
            q = s.q[b, cols].double().reshape(group, d)
            score = torch.mm(q, k.t().contiguous()) * d ** -0.5
            size = torch.mm(q.abs(), k.t().abs().contiguous()) * d ** -0.5
            p = torch.softmax(score, 1)
            want, pv = torch.mm(p, v), torch.mm(p, v.abs())
            err = 2 * ((d + 8) * U * size).amax(1, keepdim=True) + 8 * U          # of a weight, as attention_rows has it
            least = n * 2.0 ** -32 * 127 * (p * sv).amax(1, keepdim=True)
            bound = (HALF16 + 2 * U) * pv + (err + (n + 4) * U) * (pv + want.abs()) + least + half(s.t) * want.abs() + (2.0 ** -25 if s.t == "f16" else 2.0 ** -125)
            got = s.o[b, cols].reshape(group, d).double()
            off = (got - want).abs()
            assert bool((off <= bound).all()), "%s: request %d, head %d: %g over, results of %g" % (
                what, b, h, float((off - bound).nan_to_num(math.inf).max()), float(want.abs().max()))
            spread = torch.mm(p * p, v * v)
            sums[0] += float(((got - want) ** 2).sum())
            sums[1] += float((HALF16 ** 2 / 3 * spread + half(s.t) ** 2 / 3 * want * want).sum())
            sums[2] += want.numel()
    if mean:                                                  # independent errors of at most half a step each: see attention_rows.check_mean
        assert sums[2] > 1000 and sums[0] <= 1.5 * sums[1], "%s: mean square error %g, expected at most %g" % (what, sums[0] / sums[2], 1.5 * sums[1] / sums[2])


def quiet(s, where, power, bits):
    """Key `where` (of the prefix, or of every request's own) gets value scales 2^power times as large and a weight of about 2^-bits of the others' in all rows: queries
    of all rows are alike."""
    import torch
    shared, at = where
    s.q[:] = s.q[:1, :s.d].repeat(1, s.H)
    q = s.q[0, :s.d].double()
    row = torch.where(q > 0, -127, 127).to(torch.int8)
    scale = bits * math.log(2.0) * math.sqrt(s.d) / (127 * float(q.abs().sum()))
    for table in ([s.prefix_pages] if shared else [s.pages[b] for b, n in enumerate(s.lens_) if n > at]):
        page = int(table[at // s.page])
        s.cache["k"][page, :, at % s.page] = row
        s.cache["k_scale"][page, :, at % s.page] = scale
        s.cache["v_scale"][page, :, at % s.page] = 2.0 ** power
    return s


def modest(s):
    """scores of a few units, so that most keys count"""
    s.cache["k_scale"].fill_(1 / 200.0)
    s.cache["v_scale"].clamp_(1 / 200.0, 1 / 20.0)
    return s


@pytest.mark.parametrize("power", [9, 20, 24, 30, 45])
@pytest.mark.parametrize("at", [0, 40, 299])
def test_a_key_of_little_weight_and_large_values(ivit, power, at):
    """The values of the keys that count keep their bits, whether that key comes first, between them or last, and whatever it adds itself."""
    for d, t in ((64, "bf16"), (128, "bf16"), (128, "f16")):
        for bits in (power + 3, 2 * power + 20):
            s = quiet(modest(Setup(at + power, [300, 300], 0, 4, 4, d, t, True, 32)), (False, at), power, bits)
            s.call(ivit)
            compare(s, "own key %d, 2^%d, weight 2^-%d, %d x %s" % (at, power, bits, d, t))
        for B in (3, 70):                                     # rows of their own, and workgroups that share tiles of the prefix
            s = quiet(modest(Setup(at + power + B, [20] * B, 300, 2, 2, d, t, True, 32)), (True, at), power, power + 3)
            s.call(ivit)
            compare(s, "key %d of the prefix of %d, 2^%d, %d x %s" % (at, B, power, d, t), requests=(0, 1, B - 1))


@pytest.mark.parametrize("way", [1, -1])
@pytest.mark.parametrize("B", [2, 70])
def test_scales_that_grow_or_fall_while_weights_do_the_other(ivit, way, B):
    """Weights from 1 to 2^-60 and scales from 1 to 2^60: the products stay alike, the largest score moves often or never."""
    import torch
    for d, t in ((64, "bf16"), (128, "f16")):
        for part in (1.0, 0.5, 2.0):                          # products alike; those of the light keys ahead; those of the heavy ones
            s = modest(Setup(B, [0] * B, 1000, 2, 2, d, t, True, 32))
            s.q[:] = s.q[:1, :d].repeat(1, s.H)
            q = s.q[0, :d].double()
            at = torch.arange(1000, device="cuda")
            x = 60.0 * (at if way > 0 else 999 - at).double() / 999
            page, slot = s.prefix_pages[at // 32].long(), at % 32
            s.cache["k"][:] = torch.where(q > 0, -127, 127).to(torch.int8)
            s.cache["k_scale"][page, :, slot] = (part * x * math.log(2.0) * math.sqrt(d) / (127 * q.abs().sum())).float()[:, None].expand(-1, 2)
            s.cache["v_scale"][page, :, slot] = (2.0 ** (x - (45 if t == "f16" and part < 1 else 0)) / 100).float()[:, None].expand(-1, 2)
            s.call(ivit)
            compare(s, "%d requests %d x %s, way %d, %g" % (B, d, t, way, part), requests=(0, B - 1))


def test_rounding_of_the_products(ivit):
    """The mean square error is that of products rounded to float16, for bfloat16 rows too."""
    for d in (64, 128):
        for t in ("f16", "bf16"):
            s = modest(Setup(7, [2000, 130, 1, 700], 0, 16, 4, d, t, True, 64))
            s.call(ivit)
            compare(s, "own", mean=True)
            s = modest(Setup(8, [30] * 20, 1500, 8, 2, d, t, True, 64))
            s.call(ivit)
            compare(s, "prefix of many rows", mean=True)
            s = modest(Setup(9, [100, 30], 1500, 8, 2, d, t, True, 16))
            s.call(ivit)
            compare(s, "prefix", mean=True)


def test_rows_of_large_and_small_scores(ivit):
    for size in (0.1, 6.0):
        s = Setup(11, [1, 31, 900, 0, -1, 64], 333, 6, 2, 128, "bf16", True, 16, garbage=float("nan"), size=size)
        s.call(ivit)
        compare(s, "size %g" % size)
