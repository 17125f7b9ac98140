"""Attention over float rows: calls whose arguments would leave the range of 32 bits or lie in memory otherwise than stated, refused before anything is launched (no GPU)."""
import math

import pytest

from paper_2207_01405_amd import binding
from test_attention_rows_host import E, I8, FAKE, cached, lib, pool, prompt  # noqa: F401 (lib: a fixture)


def test_a_scale_beyond_the_range_of_its_exponents(lib):
    """Weights are powers of two of scale log2 e q . k: of 2.4e38 on that factor is infinite, and a score of 0 would be NaN."""
    most = 3.4028234e38 / 1.4426951
    for scale in (most * 1.0001, 3.0e38, 3.4e38):
        assert math.isfinite(scale)
        assert prompt(lib, scale=scale) == E["PARAM"] and cached(lib, scale=scale) == E["PARAM"]
        assert cached(lib, scale=scale, c=pool(t=I8, ks=FAKE, vs=FAKE)) == E["PARAM"]
    for scale in (most * 0.9999, 1.0e-38, 1.4e-45):
        assert prompt(lib, scale=scale, nq=0, nk=0, q=None, o=None) == 0 and cached(lib, scale=scale, B=0) == 0
