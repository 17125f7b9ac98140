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
