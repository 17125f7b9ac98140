"""Workgroups of 1024 threads with two pieces of a row each: two of them are on a CU at a time while a thread has 64 vector registers at most (norms of
2000 x 14336 bf16 with a residual 44 us, with 66 registers 50).  Read from the compiler's notes in the library, without a GPU."""
import re

from paper_2207_01405_amd import binding
from test_spilled_registers import _number, _spills


def test_two_workgroups_of_1024_threads_fit_a_cu():
    _spills()                                               # (builds the library if it is not there)
    b, of, key = open(binding.LIB_PATH, "rb").read(), {}, b".vgpr_count"
    for m in re.finditer(rb"\.symbol[\xa0-\xbf\xd9\xda][\x00-\xff]{0,2}?(_Z\w+)\.kd", b):
        name = m.group(1).decode()
        if re.search(r"(rmsnorm|gated)_kernelI\w+Li2ELi1024ELi1024E", name):
            of[name] = _number(b, b.index(key, m.end()) + len(key))
    assert len(of) == 12 and not {name: n for name, n in of.items() if n > 64}
