"""Attention over prompts in each of its forms, with keys of NaN and infinite values where a query does not see them: in the tiles that the diagonal cuts, behind
the last key of a sequence and between sequences.  The cases name their forms (at 256 CUs); test_prompt_form.py holds them to the rule."""
import math

import pytest

from attention_rows import dtype, gen, rand
from test_gpu_prompt_attention import compare, starts

pytestmark = pytest.mark.gpu

# form, queries of the sequences, keys before them, heads, causal
CASES = [("64x4", [150, 61], [0, 0], 2, True), ("64x4", [200], [333], 60, True), ("64x4", [197] * 4, [0] * 4, 6, False),
         ("64", [200, 130, 70], [0, 65, 0], 96, True), ("64", [37, 64, 5, 33] * 5, [0] * 20, 16, True), ("64", [128, 97, 33], [0, 40, 0], 96, False),
         ("128x2", [300], [0], 60, True), ("128x2", [300, 513], [64, 0], 20, True), ("128x2", [257, 190], [0, 77], 40, False),
         ("128", [300], [0], 256, True), ("128", [700, 129, 500], [0, 333, 0], 96, True), ("128", [333, 129, 290], [0, 50, 0], 100, False)]
IDS = ["%s-%s-%d-%s" % (c[0], "causal" if c[4] else "all", c[3], str(c[1])[:16].replace(" ", "")) for c in CASES]


def inputs(seed, case, d, t, G=2):
    g = gen(seed)
    _, nq, past, heads, _ = case
    nk = [n + p for n, p in zip(nq, past)]
    gap = 3                                                   # rows of no sequence behind the last
    q, k, v = rand(g, sum(nq), heads * d).to(dtype(t)), rand(g, sum(nk) + gap, G * d).to(dtype(t)), rand(g, sum(nk) + gap, G * d).to(dtype(t))
    return nq, nk, q, k, v


def some_heads(heads):
    """the first and last of each group of two"""
    return sorted({0, heads // 2 - 1, heads // 2, heads - 1})


@pytest.mark.parametrize("case", CASES, ids=IDS)
@pytest.mark.parametrize("d,t", [(64, "bf16"), (128, "f16"), (128, "bf16")])
def test_results(ivit, case, d, t):
    import torch
    nq, nk, q, k, v = inputs(1, case, d, t)
    heads, causal = case[3:]
    o = torch.full_like(q, 5.0)
    ivit.ivit_prompt_attention(q, k, v, o, d, starts(nq), starts(nk), causal=causal)
    for h in some_heads(heads):
        cols, kc = slice(h * d, h * d + d), slice(h * 2 // heads * d, h * 2 // heads * d + d)
        compare(o[:, cols], q[:, cols], k[:, kc], v[:, kc], nq, nk, 1, 1, d, causal, d ** -0.5, t, "%s head %d" % (case, h))
    p = ivit.ivit_prompt_attention(q, k, v, torch.empty_like(q), d, starts(nq), starts(nk), causal=causal)
    assert torch.equal(o, p)


@pytest.mark.parametrize("case", CASES, ids=IDS)
@pytest.mark.parametrize("what", ["keys", "values", "both"])
def test_keys_that_a_query_does_not_see(ivit, case, what):
    """Causal: from some key of a sequence on every third is bad, and the rows before it are held to their definition over the keys before it.  Not causal: every other
    sequence is bad as a whole, and so are the rows behind the last."""
    name, _, _, heads, causal = case
    for d, t, bad in ((64, "f16", math.inf), (128, "bf16", math.nan), (64, "bf16", -math.inf)):
        for cut in (0.1, 0.5, 0.97) if causal else (0.0,):
            nq, nk, q, k, v = inputs(2, case, d, t)
            clean = k.clone(), v.clone()
            kinds = [x for x, n in ((k, "keys"), (v, "values")) if what in (n, "both")]
            j, rows = 0, []
            for s, (n, m) in enumerate(zip(nq, nk)):
                rows.append(int(cut * n) if causal else 0 if s % 2 else n)      # of the sequence, that see no bad key
                first = m - n + rows[s] if causal else 0 if s % 2 else m
                for x in kinds:
                    x[j + first:j + m:3] = bad
                j += m
            for x in kinds:
                x[j:] = bad
            o = ivit.ivit_prompt_attention(q, k, v, q.new_full(q.shape, 5.0), d, starts(nq), starts(nk), causal=causal)
            i = j = 0
            for s, (n, m, c) in enumerate(zip(nq, nk, rows)):
                keys = m - n + c if causal else m
                for h in some_heads(heads) if c else ():
                    cols, kc = slice(h * d, h * d + d), slice(h * 2 // heads * d, h * 2 // heads * d + d)
                    compare(o[i:i + c, cols], q[i:i + c, cols], clean[0][j:j + keys, kc], clean[1][j:j + keys, kc], [c], [keys], 1, 1, d, causal, d ** -0.5, t,
                            "%s %s of %g from %g, sequence %d head %d" % (name, what, bad, cut, s, h))
                if what != "keys" or bad != bad:            # (an infinite key may leave a score of minus infinity: a weight of 0)
                    assert not bool(o[i + c:i + n].isfinite().all(1).any())
                i, j = i + n, j + m


@pytest.mark.parametrize("case", [c for c in CASES if c[4]], ids=[i for i, c in zip(IDS, CASES) if c[4]])
def test_rows_without_keys(ivit, case):
    """Causal with fewer keys than queries: the first rows see none and are zeros, whatever the keys hold."""
    import torch
    name, nq, _, heads, _ = case
    d, t = 64, "bf16"
    g = gen(4)
    nk = [n // 3 for n in nq]
    q, k, v = rand(g, sum(nq), heads * d).to(dtype(t)), rand(g, sum(nk), 2 * d).to(dtype(t)), rand(g, sum(nk), 2 * d).to(dtype(t))
    o = ivit.ivit_prompt_attention(q, k, v, torch.full_like(q, 5.0), d, starts(nq), starts(nk))
    for h in some_heads(heads)[:2]:
        cols, kc = slice(h * d, h * d + d), slice(h * 2 // heads * d, h * 2 // heads * d + d)
        compare(o[:, cols], q[:, cols], k[:, kc], v[:, kc], nq, nk, 1, 1, d, True, d ** -0.5, t, "%s head %d" % (name, h))
    i = j = 0
    for n, m in zip(nq, nk):
        k[j:j + m:2], v[j:j + m] = math.nan, math.inf
        i, j = i + n, j + m
    o = ivit.ivit_prompt_attention(q, k, v, torch.full_like(q, 5.0), d, starts(nq), starts(nk))
    i = 0
    for n, m in zip(nq, nk):
        assert not bool(o[i:i + n - m].any()) and not bool(o[i + n - m:i + n].isfinite().all(1).any()), name
        i += n
