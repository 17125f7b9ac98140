"""The float layers at the bounds of their sizes: the largest int8 sums with every number of tokens, and every row of calls that take several launches."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [1, 2, 8, 9, 16, 17, 32, 40, 130, 300])
def test_the_largest_sums_of_every_form(ivit, M):
    """All terms (-128)^2, 127^2 and 127 (-128), of every token; with scales of 1 a sum is rounded to 32 bits once."""
    import torch
    for N, K in ((40, 65536), (300, 65536), (4500, 8192)):
        for a in (-128, 127):
            x = torch.full((M, K), a, dtype=torch.int8, device="cuda")
            w = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
            w[1::3] = 127
            w[2::3, ::2] = 127
            y = torch.full((M, N), 99.0, device="cuda")
            ivit.ivit_linear_scaled(x, torch.ones(M, device="cuda"), w, torch.ones(N, device="cuda"), y)
            want = torch.empty(N, dtype=torch.float64, device="cuda")
            want[0::3], want[1::3], want[2::3] = a * -128 * K, a * 127 * K, a * (127 - 128) * (K // 2)
            assert torch.equal(y, want.float().expand(M, N)), (N, K, a)
    assert 128 * 128 * 65536 == 1 << 30


def test_every_row_of_several_launches_is_written(ivit):
    """2^31 threads are 2^23 rows of 256 threads: rows of zeros have the scale 0 and zeros, all of them, and the few others are where they belong."""
    import torch
    rows, C = (1 << 23) + 9, 2048
    at = torch.tensor([0, 7, (1 << 23) - 1, 1 << 23, rows - 1], device="cuda")
    x = torch.zeros((rows, C), dtype=torch.bfloat16, device="cuda")
    x[at] = 1.0 + torch.rand((at.numel(), C), device="cuda").to(x.dtype)
    q, s = torch.full((rows, C), 77, dtype=torch.int8, device="cuda"), torch.full((rows,), 7.0, device="cuda")

    def check():
        assert torch.equal(torch.nonzero(s)[:, 0], at)
        assert bool((q[at] > 0).all())
        q[at] = 0
        for part in q.split(1 << 20):
            assert not bool(part.any())

    ivit.ivit_rmsnorm_quant(x, None, q, s, 1e-6)
    check()
    q.fill_(77); s.fill_(7.0)
    ivit.ivit_gated_quant(x, q, s, act="silu", gated=False)
    check()
