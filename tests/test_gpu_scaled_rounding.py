"""int8 rows of the float layers, value by value: q = round(127 v / max |v|) is a whole number that 64 bits give exactly, so every one has to be
equal.  127 v / max |v| of 24-bit numbers that is no tie is 2^-32 from one at least, and the quotient of two 64-bit numbers is rounded
correctly: what the tests compute is exact, ties included."""
import pytest

pytestmark = pytest.mark.gpu

TYPES = ("f32", "f16", "bf16")
WIDTHS = [3, 8, 50, 64, 127, 200, 384, 600, 1000, 1500, 2049, 4000, 5001, 9000, 20000]


def dtype(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def levels(v):
    """The int8 rows of exactly known values."""
    import torch
    v = v.double()
    return torch.round(127.0 * v / v.abs().amax(1, keepdim=True)).to(torch.int8)


def tied_rows(rows, C, t, seed, power=0):
    """Rows on coarse grids: their largest is 127 times a small number, with every k + 1/2 of its 127th parts beside it, or any number, with its half beside it."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    v = torch.randint(-126, 127, (rows, C), generator=g, device="cuda").double() + 0.5
    v[:, C // 2] = 127.0
    odd = torch.arange(rows, device="cuda") % 2 == 1
    top = torch.randint(128, 256, (rows, 1), generator=g, device="cuda").double()
    halves = torch.where(torch.rand((rows, C), generator=g, device="cuda") < 0.5, 0.5, 0.25) * top * torch.sign(v)
    halves[:, C // 2:C // 2 + 1] = top
    v = torch.where(odd[:, None], halves, v) * 2.0 ** power
    x = v.to(dtype(t))
    assert torch.equal(x.double(), v)
    return x


def quantised(ivit, x, act="none", gated=False):
    import torch
    rows, C = x.shape[0], x.shape[1] // (2 if gated else 1)
    q, s = torch.full((rows, C), 99, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    ivit.ivit_gated_quant(x, q, s, act=act, gated=gated)
    return q, s


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", WIDTHS)
def test_ties_go_to_even(ivit, C, t):
    import torch
    powers = (0, -130, 100) if t == "f32" else (0, -100, 100) if t == "bf16" else (0, -7)
    for power in powers:
        x = tied_rows(41, C, t, C, power)
        q, s = quantised(ivit, x)
        assert torch.equal(q, levels(x))
        u = 2.0 ** torch.randint(-3, 4, (41, 1), device="cuda").to(dtype(t))
        g = torch.cat([x.abs(), (u * torch.sign(x)).to(x.dtype)], 1)
        if power == 0:
            q, s = quantised(ivit, g, act="relu", gated=True)
            assert torch.equal(q, levels(x))
            y, sy = torch.empty_like(q), torch.empty_like(s)
            ivit.ivit_rmsnorm_quant(x, None, y, sy, 1e-6)
            assert torch.equal(y, levels(x))
            ivit.ivit_rmsnorm_quant(x, torch.full((C,), 0.25, device="cuda"), y, sy, 1e-6)
            assert torch.equal(y, levels(x))


@pytest.mark.parametrize("t", TYPES)
def test_every_value_of_many_is_the_nearest(ivit, t):
    """Among millions of values some lie next to a tie, where the quotient's last place decides."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    for rows, C in ((20000, 384), (3000, 2049), (1000, 12000)):
        x = torch.randn((rows, C), generator=g, device="cuda").to(dtype(t))
        assert torch.equal(quantised(ivit, x)[0], levels(x))
        y, sy = torch.empty((rows, C), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
        ivit.ivit_rmsnorm_quant(x, None, y, sy, 1e-6)
        assert torch.equal(y, levels(x))
        h = torch.empty_like(x)
        gamma = 1.0 + 0.1 * torch.randn(C, generator=g, device="cuda")
        ivit.ivit_rmsnorm_quant(x, gamma, y, sy, 1e-6, residual=x, sum_out=h)
        assert torch.equal(y, levels((x.float() + x.float()) * gamma))      # (x + x is exact; the product is rounded to 32 bits once)


@pytest.mark.parametrize("M,N,K", [(1, 253, 16), (20, 253, 64), (40, 253, 512), (300, 253, 256), (3000, 506, 96)])
def test_int8_at_a_fixed_step(ivit, M, N, K):
    """Values exactly between two steps, by the bias alone: as the header has it, round(v * (1 / step)) in 32 bits; even at a power of two."""
    import numpy as np
    import torch
    k = torch.arange(-126, 127, device="cuda").repeat(N // 253).float()
    for step in (1.0, 0.25, 2.0 ** -7, 0.75, 7.0, 0.21875, 0.40625, 100.0):
        bias = (k + 0.5) * step
        assert torch.equal(bias.double(), (k.double() + 0.5) * step)
        y = torch.full((M, N), 99, dtype=torch.int8, device="cuda")
        ivit.ivit_linear_scaled(torch.zeros((M, K), dtype=torch.int8, device="cuda"), torch.ones(M, device="cuda"), torch.ones((N, K), dtype=torch.int8, device="cuda"),
                                torch.ones(N, device="cuda"), y, bias=bias, y_step=step)
        f = np.float32(1) / np.float32(step)
        want = torch.from_numpy(np.clip(np.rint(bias.cpu().numpy() * f), -127, 127).astype(np.int8)).cuda()
        assert bool((y == want).all()), step
        if step in (1.0, 0.25, 2.0 ** -7):
            assert torch.equal(want, torch.round(k + 0.5).to(torch.int8))
