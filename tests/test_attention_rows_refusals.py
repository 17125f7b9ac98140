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


def test_the_structures_alone_before_any_call(monkeypatch):
    """rotary_params and cache_struct take tensors before another call of the binding has looked up torch's types."""
    import torch
    for name in ("_TYPES", "_INT8", "_INT32", "_FLOAT32", "_FLOAT64"):
        monkeypatch.setattr(binding, name, None)
    r = binding.rotary_params({"positions": torch.zeros(4, dtype=torch.int32), "freq": torch.ones(32, dtype=torch.float64)}, 4, -1)
    assert r.n_axes == 1 and r.rotary_dim == 64
    for name in ("_TYPES", "_INT8", "_INT32", "_FLOAT32", "_FLOAT64"):
        monkeypatch.setattr(binding, name, None)
    c = {n: torch.zeros(2, 1, 16, 64, dtype=torch.int8) for n in "kv"}
    c.update({n + "_scale": torch.zeros(2, 1, 16) for n in "kv"})
    assert binding.cache_struct(c, -1).n_pages == 2


def test_positions_expanded_over_their_axes_and_other_strides():
    """The binding names what is wrong, as for every other tensor, in place of the C call's status; tensors here are on the host, which is device -1."""
    import torch
    freq = torch.ones(32, dtype=torch.float64)
    one = torch.zeros(1, 4, dtype=torch.int32)
    for pos in (one.expand(3, 4), torch.zeros(4, 3, dtype=torch.int32).t(), torch.zeros(9, dtype=torch.int32).as_strided((3, 4), (2, 1))):
        with pytest.raises(ValueError, match="positions"):
            binding.rotary_params({"positions": pos, "freq": freq}, 4, -1)
    for pos in (one, one[0], torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, 9, dtype=torch.int32)[:, 2:6], one.expand(1, 4)):
        r = binding.rotary_params({"positions": pos, "freq": freq}, 4, -1)
        assert r.ld_positions >= 4 and r.n_axes == (pos.shape[0] if pos.dim() == 2 else 1)
    r = binding.rotary_params({"positions": torch.zeros(3, 1, dtype=torch.int32), "freq": freq}, 1, -1)
    assert r.ld_positions == 1 and r.n_axes == 3
