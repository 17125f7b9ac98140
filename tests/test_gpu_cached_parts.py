"""Attention over the cache in more parts than the join takes in one round of 64, against its definition in 64 bits.  That the sizes here give as many parts is
shown in test_cached_form.py (at 256 CUs) and looked at again from the size of the workspace."""
import math

import pytest

from test_gpu_cached_attention import Setup

pytestmark = pytest.mark.gpu


def parts(ivit, s):
    """of a part: the largest score, the sum and the output of every head in 32 bits"""
    n = ivit.ivit_cached_attention_workspace_bytes(s.B, s.H, s.cache, s.pages.shape[1], s.prefix)
    return n // (s.B * s.H * (s.d + 2) * 4)


def many(seed, lens, prefix, d=128, t="bf16", i8=False, room=33024, H=32, G=8, **more):
    """a table with room for `room` keys"""
    return Setup(seed, lens, prefix, H, G, d, t, i8, 64, spare=-(-room // 64) - max(-(-max(n, 0) // 64) for n in lens), **more)


# (keys of the request, of the prefix, room of the table): own keys alone, a prefix and own keys that pass 64 together, the second round's first part alone with keys of
# its own, no keys in the first round's later parts, none at all
SIZES = [(33000, 0, 33024), (33024, 0, 33024), (20001, 20000, 20032), (13056, 9000, 13056), (5, 9000, 13056), (300, 0, 33024), (1, 0, 33024), (0, 0, 33024), (0, 9000, 13056)]


@pytest.mark.parametrize("keys,prefix,room", SIZES)
def test_many_parts(ivit, keys, prefix, room):
    for d, t, i8 in ((128, "bf16", False), (128, "bf16", True), (64, "f16", False), (64, "f16", True)):
        s = many(keys + prefix, [keys], prefix, d, t, i8, room)
        assert parts(ivit, s) > 64
        first = s.call(ivit).clone()
        s.compare("%d parts" % parts(ivit, s))
        import torch
        for _ in range(3):
            assert torch.equal(first, s.call(ivit)), "equal calls"


def test_two_requests_of_different_length(ivit):
    for i8 in (False, True):
        s = many(3, [17000, -1], 0, i8=i8, room=33024, H=8, G=4)
        assert parts(ivit, s) > 64
        s.call(ivit)
        s.compare("one of two")


@pytest.mark.parametrize("at", [10, 16000, 32990])
def test_the_largest_score_in_the_first_or_the_last_round(ivit, at):
    """One key's score stands out by 20 in weight's exponent or by 400, wherever it lies."""
    import torch
    for size in (20.0, 400.0):
        for i8 in (False, True):
            s = many(at, [33000], 0, i8=i8, H=8, G=8)
            assert parts(ivit, s) > 64
            page, slot = int(s.pages[0, at // 64]), at % 64
            q = s.q[0].reshape(8, 128).double()
            k = q * (size * 128 ** 0.5 / (q * q).sum(1, keepdim=True))
            if i8:
                scale = k.abs().amax(1, keepdim=True) / 127
                s.cache["k"][page, :, slot] = (k / scale).round().to(torch.int8)
                s.cache["k_scale"][page, :, slot] = scale[:, 0].float()
            else:
                s.cache["k"][page, :, slot] = k.bfloat16()
            s.call(ivit)
            s.compare("key %d of score %g" % (at, size))


@pytest.mark.parametrize("at", [0, 15000, 32999])
def test_nan_in_any_round(ivit, at):
    import torch
    for i8 in (False, True):
        for name in "kv":
            s = many(5, [33000], 0, i8=i8, H=8, G=4)
            assert parts(ivit, s) > 64
            want = s.call(ivit).clone().reshape(4, -1)
            where = s.cache[name + "_scale" if i8 else name]
            where[int(s.pages[0, at // 64]), 1, at % 64] = math.nan
            got = s.call(ivit).reshape(4, -1)
            assert bool(got[1].isnan().all()) and torch.equal(got[[0, 2, 3]], want[[0, 2, 3]])


def test_replayed_from_a_graph(ivit):
    """The same launches for requests that grow: parts go by the table."""
    import torch
    s = many(6, [33000], 500, H=8, G=4)
    ws = s.workspace(ivit)
    s.call(ivit, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.call(ivit, ws)
    for n in (33000, 1, 0, 16500, 32999):
        s.lens.fill_(n)
        s.lens_ = [n]
        s.o.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        s.compare("replayed at %d" % n)
        got = s.o.clone()
        assert torch.equal(got, s.call(ivit))
