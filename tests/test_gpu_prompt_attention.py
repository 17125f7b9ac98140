"""Attention over whole prompts against its definition in 64 bits."""
import math
import random

import pytest

from attention_rows import attend64, check, check_mean, dtype, gen, rand

pytestmark = pytest.mark.gpu


def starts(lengths):
    import torch
    return torch.tensor([0] + lengths).cumsum(0).to(torch.int32).cuda()


def compare(o, q, k, v, nq, nk, H, G, d, causal, scale, t, what, mean=False):
    import torch
    i = j = 0
    sums = [[], [], []]
    for n, m in zip(nq, nk):
        hidden = None
        if causal:
            hidden = torch.arange(m, device="cuda") > torch.arange(n, device="cuda")[:, None] + (m - n)
        for h in range(H):
            cols, kc = slice(h * d, h * d + d), slice(h * G // H * d, h * G // H * d + d)
            vv = v[j:j + m, kc].double()
            want, pv, err, spread = attend64(q[i:i + n, cols].double(), k[j:j + m, kc].double(), vv, scale, hidden)
            got = o[i:i + n, cols]
            if n:
                check(got, want, pv, err, m, t, float(vv.abs().max()) if m else 0.0, "%s: sequence of %d, %d, head %d" % (what, n, m, h))
            for s, x in zip(sums, (got, want, spread)):
                s.append(x)
        i, j = i + n, j + m
    if mean:
        check_mean(*(torch.cat(s) for s in sums), t, what)


def run(ivit, seed, nq, nk, H, G, d, causal, t, scale=None, size=1.0, packed=False, mean=False):
    import torch
    g = gen(seed)
    rows, keys = sum(nq), sum(nk)
    if packed:
        qkv = (rand(g, rows, (H + 2 * G) * d + 24) * size).to(dtype(t))
        q, k, v = qkv[:, 8:8 + H * d], qkv[:, 8 + H * d:8 + (H + G) * d], qkv[:, 8 + (H + G) * d:8 + (H + 2 * G) * d]
    else:
        q, k, v = (rand(g, rows, H * d) * size).to(dtype(t)), rand(g, keys, G * d).to(dtype(t)), rand(g, keys, G * d).to(dtype(t))
    o = torch.full((rows + 3, H * d + 16), 5.0, device="cuda", dtype=dtype(t))
    ks = None if packed else starts(nk)
    out = o[:rows, 8:8 + H * d]
    assert ivit.ivit_prompt_attention(q, k, v, out, d, starts(nq), ks, scale=scale, causal=causal) is out
    assert bool((o[rows:] == 5).all()) and bool((o[:, :8] == 5).all()) and bool((o[:, 8 + H * d:] == 5).all())
    compare(out, q, k, v, nq, nk, H, G, d, causal, d ** -0.5 if scale is None else scale, t,
            "%s %s %d/%d x %d causal %s %s" % (nq, nk, H, G, d, causal, t), mean)


LENGTHS = [([1], [1]), ([2], [2]), ([31], [31]), ([32], [32]), ([33], [33]), ([63], [63]), ([64], [64]), ([65], [65]), ([127], [127]), ([128], [128]), ([129], [129]),
           ([255], [255]), ([256], [256]), ([257], [257]), ([1], [1000]), ([7], [300]), ([130], [131]), ([64], [129]), ([1, 1, 1], [64, 65, 1]), ([40], [513]),
           ([100], [37]), ([200], [100]), ([300], [1]), ([5], [0]), ([3, 0, 9], [0, 4, 9]), ([127, 128, 129, 1, 0, 63], [127, 128, 129, 1, 0, 63]),
           ([17] * 70, [17] * 70), ([1] * 200, [1] * 200), ([0, 0, 70], [5, 0, 70])]


@pytest.mark.parametrize("nq,nk", LENGTHS, ids=["%s-%s" % (str(a)[:24], str(b)[:24]) for a, b in LENGTHS])
def test_lengths(ivit, nq, nk):
    for i, (H, G, d, t) in enumerate(((2, 1, 64, "bf16"), (3, 3, 128, "f16"), (8, 2, 128, "bf16"), (8, 8, 64, "f16"))):
        if len(nq) > 20 and i > 1:
            continue
        for causal in (True, False):
            run(ivit, 10 * sum(nk) + i, nq, nk, H, G, d, causal, t)


@pytest.mark.parametrize("seed", range(8))
def test_drawn(ivit, seed):
    r = random.Random(seed)
    n = r.choice((1, 2, 5))
    nq = [r.randint(0, 700) for _ in range(n)]
    G = r.choice((1, 2, 3))
    run(ivit, seed, nq, [a + r.choice((0, r.randint(0, 500))) for a in nq], G * r.choice((1, 2, 5)), G, r.choice((64, 128)), r.random() < 0.6,
        r.choice(("f16", "bf16")), size=r.choice((1.0, 4.0)), scale=r.choice((None, 0.02, 0.3)))


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_long(ivit, d, t):
    for causal in (True, False):
        run(ivit, 3, [2100], [2100], 8, 2, d, causal, t, mean=True)


def test_in_packed_rows(ivit):
    for t in ("f16", "bf16"):
        run(ivit, 4, [100, 1, 260], [100, 1, 260], 6, 2, 64, True, t, packed=True)
        run(ivit, 4, [100, 1, 260], [100, 1, 260], 4, 4, 128, False, t, packed=True)


def test_large_scores(ivit):
    """Scores of several hundred: the weights of most keys vanish, and the largest score moves often."""
    for t in ("f16", "bf16"):
        for size in (10.0, 60.0):
            run(ivit, 9, [300], [300], 2, 1, 128, True, t, size=size)
            run(ivit, 9, [70], [900], 2, 2, 64, False, t, size=size)


def test_a_largest_score_that_comes_last_or_first(ivit):
    import torch
    for t in ("f16", "bf16"):
        for way in (1, -1):
            g = gen(2)
            n, d = 640, 128
            k = rand(g, n, d)
            k[:, 0] = way * torch.linspace(-8, 8, n, device="cuda")         # scores grow, or fall, along the keys
            q = rand(g, n, d)
            q[:, 0] = 40.0
            q, k, v = q.to(dtype(t)), k.to(dtype(t)), rand(g, n, d).to(dtype(t))
            o = torch.empty_like(q)
            ivit.ivit_prompt_attention(q, k, v, o, d, starts([n]), causal=False)
            compare(o, q, k, v, [n], [n], 1, 1, d, False, d ** -0.5, t, "%s %d" % (t, way))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_is_left_out_has_no_part(ivit, bad):
    """NaN and infinite values at keys behind a query, in another sequence's rows, in rows between and behind them."""
    import torch
    for t in ("f16", "bf16"):
        for d in (64, 128):
            g = gen(11)
            lengths, H, G = [150, 90, 61], 2, 1
            rows = sum(lengths)
            q, k, v = (rand(g, rows + 5, n * d).to(dtype(t)) for n in (H, G, G))
            clean = k.clone(), v.clone()
            at = [100, 101, 149, 150 + 63, 150 + 64, rows, rows + 4]          # tokens that hold them, in their sequences, and rows behind the last
            k[at[::2]], v[at] = bad, bad
            o = torch.empty_like(q[:rows])
            ivit.ivit_prompt_attention(q[:rows], k, v, o, d, starts(lengths), starts(lengths), causal=True)
            compare_q, i = q[:rows], 0
            for n, first in zip(lengths, (100, 63, 61)):                       # rows before the first such token of their sequence
                e = i + first
                compare(o[i:e], compare_q[i:e], clean[0][i:e], clean[1][i:e], [first], [first], H, G, d, True, d ** -0.5, t, "%s %s" % (t, bad))
                assert not bool(o[e:i + n].isfinite().all(1).any())
                i += n


def test_sequences_outside_the_rows_are_left_out(ivit):
    import torch
    g = gen(1)
    q, k, v = (rand(g, 100, 64).bfloat16() for _ in range(3))
    for qs, ks, done in (([0, 40, 120], [0, 40, 100], 40), ([0, 40, 100], [0, 40, 101], 40), ([-3, 40, 100], [0, 40, 100], None), ([50, 40, 100], [0, 40, 100], None)):
        o = torch.full_like(q, 5.0)
        ivit.ivit_prompt_attention(q, k, v, o, 64, torch.tensor(qs, dtype=torch.int32, device="cuda"), torch.tensor(ks, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        if done:
            compare(o[:done], q[:done], k[:done], v[:done], [done], [done], 1, 1, 64, True, 0.125, "bf16", "first")
            assert bool((o[done:] == 5).all())
    o = torch.full_like(q, 5.0)
    ivit.ivit_prompt_attention(q, k, v, o, 64, torch.tensor([10, 30, 30, 70], dtype=torch.int32, device="cuda"))
    assert bool((o[:10] == 5).all()) and bool((o[70:] == 5).all()) and bool((o[10:70] != 5).any(1).all())


def test_equal_calls_give_equal_bits_and_rows_do_not_depend_on_the_batch(ivit):
    import torch
    g = gen(12)
    q, k, v = (rand(g, 900, n * 128).bfloat16() for n in (4, 2, 2))
    a, b, c = (torch.empty_like(q) for _ in range(3))
    ivit.ivit_prompt_attention(q, k, v, a, 128, starts([300, 600]))
    ivit.ivit_prompt_attention(q, k, v, b, 128, starts([300, 600]))
    assert torch.equal(a, b)
    ivit.ivit_prompt_attention(q[300:], k[300:], v[300:], c[300:], 128, starts([600]))
    assert torch.equal(a[300:], c[300:])


def test_many_sequences(ivit):
    import torch
    r = random.Random(3)
    lengths = [r.randint(0, 3) for _ in range(5000)]
    g = gen(13)
    n, d = sum(lengths), 64
    q, k, v = (rand(g, n, d).bfloat16() for _ in range(3))
    o = torch.full_like(q, 5.0)
    ivit.ivit_prompt_attention(q, k, v, o, d, starts(lengths))
    i = 0
    for s, m in enumerate(lengths):
        if m and s % 97 == 0:
            compare(o[i:i + m], q[i:i + m], k[i:i + m], v[i:i + m], [m], [m], 1, 1, d, True, 0.125, "bf16", "sequence %d" % s)
        i += m
    assert not bool((o == 5).all(1).any())


@pytest.mark.parametrize("most", [1, 16, 49, 64, 90, 160])
def test_many_short_sequences(ivit, most):
    r = random.Random(most)
    for H, G, d, t in ((8, 2, 64, "bf16"), (8, 4, 128, "f16"), (7, 1, 128, "bf16")):
        for causal in (True, False):
            nq = [r.randint(0, most) for _ in range(47)] + [most]
            run(ivit, most, nq, nq, H, G, d, causal, t)
            run(ivit, most, nq, [n + r.choice((0, 1, 31, 32, 33, 100)) for n in nq], H, G, d, causal, t)
            run(ivit, most, nq, [r.randint(0, 70) for _ in nq], H, G, d, causal, t)


@pytest.mark.parametrize("causal", [True, False])
def test_what_is_left_out_has_no_part_in_short_sequences(ivit, causal):
    """Rows of one sequence are the keys behind another's last, and keys of NaN and infinite values those that a query does not see."""
    import torch
    for d in (64, 128):
        g = gen(d)
        lengths, heads = [37, 64, 5, 33] * 20, 4
        n = sum(lengths)
        q, k, v = (rand(g, n, heads * d).bfloat16() for _ in range(3))
        clean, at, bad, first = (k.clone(), v.clone()), 0, [], []
        for i, m in enumerate(lengths):
            if i % 2:                                                       # the second half of every other sequence (not causal: all of it)
                cut = m // 2 if causal else 0
                k[at + cut:at + m:3], v[at + cut:at + m:2] = math.nan, math.inf
                bad.append(torch.arange(at + cut, at + m))
                first += list(range(at, at + cut))
            else:
                first += list(range(at, at + m))
            at += m
        o, want = torch.empty_like(q), torch.empty_like(q)
        ivit.ivit_prompt_attention(q, *clean, want, d, starts(lengths), causal=causal)
        ivit.ivit_prompt_attention(q, k, v, o, d, starts(lengths), causal=causal)
        assert bool(o[first].isfinite().all())
        compare(want, q, *clean, lengths, lengths, heads, heads, d, causal, d ** -0.5, "bf16", "%d" % d)
        # either is off by a rounding of the weights and one of the result, 2^-8 each
        assert float((o[first].float() - want[first].float()).abs().max()) <= 2.0 ** -6 * float(want.abs().max())
        assert not bool(o[torch.cat(bad)].reshape(-1, heads * d).isfinite().all(1).any())
