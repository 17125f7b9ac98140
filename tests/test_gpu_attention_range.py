"""Attention over float rows whose values lie near the ends of what 32 bits hold: 2^9 times the sum of a row's |v| within float32, and far below 1."""
import pytest

from attention_rows import attend64, check, dtype, gen, rand
from test_gpu_cached_attention import Setup
from test_gpu_prompt_attention import compare, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [-110, -60, 60, 107])
@pytest.mark.parametrize("n,heads", [(40, 2), (300, 2), (300, 60), (300, 256), (70, 256)])
def test_prompts(ivit, power, n, heads):
    """300 values of up to 4.5 times 2^107 add up to less than 2^119."""
    import torch
    for d in (64, 128):
        g = gen(power + n)
        q, k, v = rand(g, n, heads * d).bfloat16(), rand(g, n, 2 * d).bfloat16(), (rand(g, n, 2 * d).clamp(-4.5, 4.5).double() * 2.0 ** power).bfloat16()
        o = ivit.ivit_prompt_attention(q, k, v, torch.empty_like(q), d, starts([n]))
        for h in {0, heads - 1}:
            cols, kc = slice(h * d, h * d + d), slice(h * 2 // heads * d, h * 2 // heads * d + d)
            compare(o[:, cols], q[:, cols], k[:, kc], v[:, kc], [n], [n], 1, 1, d, True, d ** -0.5, "bf16", "2^%d, %d rows, %d heads of %d" % (power, n, heads, d))


@pytest.mark.parametrize("power", [-110, -60, 60, 106])
@pytest.mark.parametrize("B", [2, 70])
def test_cached(ivit, power, B):
    import torch
    for i8 in (False, True):
        for d in (64, 128):
            for prefix in (0, 150):
                s = Setup(power + B, [150] * B, prefix, 4, 2, d, "bf16", i8, 32)
                if i8:                                        # rows of up to 127 / 73 times the scale's factor
                    s.cache["v_scale"].clamp_(1 / 500.0, 1 / 30.0)
                    s.cache["v_scale"] *= 2.0 ** power
                else:
                    s.cache["v"] = (s.cache["v"].double().clamp(-4.5, 4.5) * 2.0 ** power).bfloat16()
                s.call(ivit)
                for b in (0, B - 1):
                    for h in range(2):
                        k, v = s.keys(b, h)
                        cols = slice(h * 2 * d, (h + 1) * 2 * d)
                        want, pv, err, _ = attend64(s.q[b, cols].double().reshape(2, d), k, v, d ** -0.5)
                        check(s.o[b, cols].reshape(2, d), want, pv, err, k.shape[0], "bf16", float(v.abs().max()), "2^%d, %d requests, prefix %d, i8 %s" % (power, B, prefix, i8),
                              scaled=4 * 2.0 ** -24)
