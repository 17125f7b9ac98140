"""Attention of single tokens over a paged cache, with and without a shared prefix, against its definition in 64 bits."""
import random

import pytest

from attention_rows import U, attend64, check, check_mean, dtype, gen, rand

pytestmark = pytest.mark.gpu


class Setup:
    """A cache whose pages lie in any order, page tables and queries; garbage wherever no key is."""

    def __init__(self, seed, lens, prefix, H, G, d, t, i8, page, spare=0, garbage=None, size=1.0, beside=False):
        import torch
        g = gen(seed)
        self.lens_, self.prefix, self.H, self.G, self.d, self.t, self.i8, self.page = lens, prefix, H, G, d, t, i8, page
        self.B, first = len(lens), -(-prefix // page)
        need = [-(-max(n, 0) // page) for n in lens]
        width = max(need + [0]) + spare
        pages = sum(need) + first + 2
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        self.prefix_pages = order[:first].contiguous() if prefix else None
        self.table, i = torch.full((self.B, width + 1), -7, dtype=torch.int32, device="cuda"), first
        for b, n in enumerate(need):
            self.table[b, :n] = order[i:i + n]
            i += n
        self.pages = self.table[:, :width]
        shape = (pages, G, page, d)
        if i8:
            self.cache = {n: torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8) for n in "kv"}
            for n in "kv":
                self.cache[n + "_scale"] = torch.exp(rand(g, *shape[:3])) / 73.0
        elif beside:
            both = rand(g, pages, 2, *shape[1:]).to(dtype(t))
            self.cache = {"k": both[:, 0], "v": both[:, 1]}
        else:
            self.cache = {n: rand(g, *shape).to(dtype(t)) for n in "kv"}
        if garbage is not None:                              # slots that hold no key
            used = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
            for tb, n in [(self.prefix_pages, prefix)] + [(self.pages[b], n) for b, n in enumerate(lens)]:
                if n > 0:
                    at = torch.arange(n, device="cuda")
                    used[tb[at // page].long(), at % page] = True
            for n in "kv":
                at = (~used)[:, None, :, None].expand(shape)
                if i8:
                    self.cache[n + "_scale"][(~used)[:, None, :].expand(shape[:3])] = garbage
                else:
                    self.cache[n][at] = garbage
        self.q = (rand(g, self.B, H * d) * size).to(dtype(t))
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.wide = torch.full((self.B, H * d + 8), 5.0, device="cuda", dtype=dtype(t))
        self.o = self.wide[:, :H * d]

    def workspace(self, ivit):
        import torch
        n = ivit.ivit_cached_attention_workspace_bytes(self.B, self.H, self.cache, self.pages.shape[1], self.prefix)
        assert n > 0
        return torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)         # NaN wherever it is read before it is written

    def call(self, ivit, ws=None, **more):
        return ivit.ivit_cached_attention(self.q, self.o, self.cache, self.pages, self.lens, self.workspace(ivit) if ws is None else ws,
                                          prefix_pages=self.prefix_pages, prefix_len=self.prefix, **more)

    def keys(self, b, h):
        import torch
        out = []
        for n in "kv":
            c = self.cache[n][:, h].double()
            if self.i8:
                c = c * self.cache[n + "_scale"][:, h].double()[..., None]
            parts = []
            for table, count in ((self.prefix_pages, self.prefix), (self.pages[b], max(self.lens_[b], 0))):
                if count:
                    at = table[:-(-count // self.page)].long().clamp(0, c.shape[0] - 1)
                    parts.append(c[at].reshape(-1, self.d)[:count])
            out.append(torch.cat(parts) if parts else c[:0, 0])
        return out

    def compare(self, what, scale=None, mean=False):
        import torch
        d, group = self.d, self.H // self.G
        what += " lens %s prefix %d %d/%d x %d %s i8 %s page %d" % (str(self.lens_)[:40], self.prefix, self.H, self.G, d, self.t, self.i8, self.page)
        assert bool((self.wide[:, self.H * d:] == 5).all()), what
        sums = [[], [], []]
        for b, n in enumerate(self.lens_):
            if n < 0:
                assert bool((self.o[b] == 5).all()), what + ": a padded row"
                continue
            for h in range(self.G):
                k, v = self.keys(b, h)
                cols = slice(h * group * d, (h + 1) * group * d)
                want, pv, err, spread = attend64(self.q[b, cols].double().reshape(group, d), k, v, d ** -0.5 if scale is None else scale)
                got = self.o[b, cols].reshape(group, d)
                check(got, want, pv, err, k.shape[0], self.t, float(v.abs().max()) if k.shape[0] else 0.0, "%s: request %d, head %d" % (what, b, h),
                      scaled=4 * U)
                for s, x in zip(sums, (got, want, spread)):
                    s.append(x)
        if mean:
            check_mean(*(torch.cat(s) for s in sums), self.t, what)


LENS = [[1], [0], [15], [16], [17], [31], [32], [33], [127], [128], [129], [1000], [5, 0, 300], [1, 2, 3, 700, -1, 64], [-1], [2500, 3]]


@pytest.mark.parametrize("lens", LENS, ids=[str(x) for x in LENS])
def test_lengths(ivit, lens):
    for i, (H, G, d, t) in enumerate(((1, 1, 64, "bf16"), (8, 2, 128, "f16"), (6, 3, 128, "bf16"), (16, 2, 64, "f16"))):
        for i8 in (False, True):
            for prefix in (0, 1, 77, 640):
                s = Setup(31 * i + prefix, lens, prefix, H, G, d, t, i8, (16, 32, 64, 256)[(i + prefix) % 4], spare=i)
                s.call(ivit)
                s.compare("")


@pytest.mark.parametrize("H,G", [(40, 1), (64, 2), (33, 1), (32, 32), (70, 2)])
def test_groups_wider_than_a_tile(ivit, H, G):
    for i8 in (False, True):
        s = Setup(H, [100, 31, 260], 50, H, G, 64, "bf16", i8, 32)
        s.call(ivit)
        s.compare("")


@pytest.mark.parametrize("seed", range(10))
def test_drawn(ivit, seed):
    r = random.Random(seed)
    G = r.choice((1, 2, 3, 8))
    s = Setup(seed, [r.choice((0, -1, r.randint(1, 50), r.randint(1, 1500))) for _ in range(r.choice((1, 3, 20)))], r.choice((0, r.randint(1, 3000))),
              G * r.choice((1, 2, 4, 7)), G, r.choice((64, 128)), r.choice(("f16", "bf16")), r.random() < 0.5, r.choice((16, 32, 64, 128, 1024)),
              spare=r.choice((0, 3)), size=r.choice((1.0, 5.0)), beside=r.random() < 0.5)
    scale = r.choice((None, 0.05))
    s.call(ivit, scale=scale)
    s.compare("", scale=scale)


@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_long(ivit, t):
    for i8 in (False, True):
        for d in (64, 128):
            s = Setup(5, [9000, 4000, 1], 5000, 16, 4, d, t, i8, 64)
            s.call(ivit)
            s.compare("long", mean=not i8)


# more than 64 query rows of a head: workgroups of 128 rows that share tiles of 64 keys of the prefix
@pytest.mark.parametrize("B,H,G", [(65, 1, 1), (33, 4, 2), (17, 8, 2), (40, 32, 4), (130, 6, 6), (3, 200, 2)])
@pytest.mark.parametrize("i8", [False, True])
def test_prefix_of_many_rows(ivit, B, H, G, i8):
    import torch
    for d, t, page in ((64, "bf16", 16), (128, "f16", 32), (128, "bf16", 256)):
        for prefix in (1, 63, 64, 65, 200, 1024, 3000):
            if prefix > 200 and H * B > 600 and d == 64:
                continue
            lens = [(7 * b) % 90 - 1 for b in range(B)]
            s = Setup(prefix + B, lens, prefix, H, G, d, t, i8, page, garbage=float("nan"))
            first = s.call(ivit).clone()
            if prefix in (65, 1024):
                s.compare("wide")
            else:                                           # a few requests stand for the others
                for b in (0, 1, B // 2, B - 1):
                    k, v = s.keys(b, 0)
                    if lens[b] < 0:
                        assert bool((s.o[b] == 5).all())
                        continue
                    group = H // G
                    want, pv, err, _ = attend64(s.q[b, :group * d].double().reshape(group, d), k, v, d ** -0.5)
                    check(s.o[b, :group * d].reshape(group, d), want, pv, err, k.shape[0], t, float(v.abs().max()), "request %d of %d behind %d" % (b, B, prefix),
                          scaled=4 * U)
            for _ in range(3):
                assert torch.equal(first, s.call(ivit)), "equal calls"


def test_prefix_alone(ivit):
    """No keys of their own, and no pages for any: the prefix is all."""
    import torch
    for B, H, G in ((2, 4, 2), (70, 2, 1), (300, 4, 2)):
        for i8 in (False, True):
            for prefix in (5, 500):
                s = Setup(B, [0] * (B - 1) + [-1], prefix, H, G, 128, "bf16", i8, 32)
                s.call(ivit)
                s.compare("no keys of their own")
                assert s.pages.shape[1] == 0


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_slots_without_keys_have_no_part(ivit, bad):
    for t in ("f16", "bf16"):
        for i8 in (False, True):
            for prefix in (0, 41):
                s = Setup(8, [1, 0, 70, 33], prefix, 4, 2, 128, t, i8, 16, garbage=bad)
                s.call(ivit)
                s.compare(str(bad))


def test_lengths_beyond_the_table_and_pages_outside_the_cache(ivit):
    import torch
    s = Setup(4, [64, 32], 0, 2, 1, 64, "bf16", False, 32)
    s.lens = torch.tensor([2 ** 31 - 1, 32], dtype=torch.int32, device="cuda")
    s.call(ivit)
    s.compare("long")
    s = Setup(4, [64, 64], 40, 2, 1, 64, "bf16", False, 32)
    s.pages[0, 1], s.pages[1, 0], s.prefix_pages[1] = 2 ** 31 - 1, -1, 1 << 20
    s.call(ivit)
    s.compare("pages")


def test_scales_of_very_different_size(ivit):
    import torch
    for t in ("f16", "bf16"):
        for power in (-30, -9, 5):
            s = Setup(6, [300, 64], 100, 4, 2, 64, t, True, 32)
            s.cache["v_scale"] *= 2.0 ** power if t == "bf16" else 2.0 ** max(power, -9)
            s.cache["v_scale"][:, :, 3::7] *= 2.0 ** -9
            s.call(ivit)
            s.compare("power %d" % power)
        s.cache["v_scale"].zero_()
        s.call(ivit)
        assert not bool(s.o.any())


def test_equal_calls_give_equal_bits(ivit):
    import torch
    s = Setup(9, [700, 1, 900], 3000, 8, 2, 128, "bf16", False, 64)
    first = s.call(ivit).clone()
    assert torch.equal(first, s.call(ivit))


def test_errors(ivit):
    import torch
    s = Setup(9, [10], 0, 2, 1, 64, "bf16", False, 32)
    with pytest.raises(ivit.IvitError) as e:
        s.call(ivit, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == ivit.IVIT_ERR_WORKSPACE
    with pytest.raises(ValueError):
        s.prefix = 5
        s.call(ivit)


@pytest.mark.parametrize("B,H,G", [(70, 1, 1), (70, 4, 2), (300, 2, 2), (3, 100, 1)])
def test_requests_without_keys_among_many(ivit, B, H, G):
    """One part of every request, no prefix: a row without keys is zeros, a padded one is left."""
    for i8 in (False, True):
        s = Setup(B, [(0, 5, -1, 60)[b % 4] for b in range(B)], 0, H, G, 64, "bf16", i8, 32)
        s.call(ivit)
        s.compare("without keys")


@pytest.mark.parametrize("prefix", [0, 40, 1000])
def test_keys_that_count_and_are_not_finite(ivit, prefix):
    """NaN among the keys, the values or the scales of a request is NaN in its row, whatever parts it is in, and in no other."""
    import torch
    nan = float("nan")
    for lens, where in (([5, 3000, 40], 0), ([5, 3000, 40], 2999), ([1, 700, 1], 3), ([1, 1, 1], 0)):
        for i8 in (False, True):
            for name in "kv":
                s = Setup(12, lens, prefix, 4, 2, 64, "bf16", i8, 16)
                want = s.call(ivit).clone()
                at = int(s.pages[1, where // 16])
                if i8:
                    s.cache[name + "_scale"][at, :, where % 16] = nan
                else:
                    s.cache[name][at, :, where % 16] = nan
                s.call(ivit)
                assert bool(s.o[1].isnan().all()), "%s prefix %d at %d %s i8 %s" % (lens, prefix, where, name, i8)
                assert torch.equal(s.o[[0, 2]], want[[0, 2]])
                if not i8 and name == "k":                  # all of a request's own scores NaN
                    s.cache["k"][s.pages[1, :-(-lens[1] // 16)].long()] = nan
                    s.call(ivit)
                    assert bool(s.o[1].isnan().all()) and torch.equal(s.o[[0, 2]], want[[0, 2]])


def test_queries_of_very_different_size(ivit):
    """bfloat16 queries over an int8 cache, whose products are float16: from below the normal numbers to near the end of the range."""
    import torch
    for power in (-130, -126, -60, 20, 100, 126):
        s = Setup(3, [60, 33], 20, 4, 2, 128, "bf16", True, 16)
        s.q = (s.q.double() * 2.0 ** power).bfloat16()
        s.call(ivit, scale=128 ** -0.5 * 2.0 ** -power if -126 <= -power <= 126 else 1.0)
        s.compare("power %d" % power, scale=128 ** -0.5 * 2.0 ** -power if -126 <= -power <= 126 else 1.0)
    s = Setup(3, [60, 33], 20, 4, 2, 128, "bf16", True, 16)
    s.q.zero_()
    s.call(ivit)
    s.compare("zeros")


@pytest.mark.parametrize("B,prefix", [(1, 0), (3, 40), (70, 40), (70, 1000)])
def test_infinite_values(ivit, B, prefix):
    """A value that counts and is infinite makes its element of the rows that see it so, and no other; the last key of all too."""
    import torch
    inf = float("inf")
    for d, t in ((64, "bf16"), (128, "f16")):
        for i8 in (False, True):
            for n, where in ((5, 4), (33, 32), (333, 332), (333, 100), (prefix, prefix - 1), (prefix, prefix // 2)):
                if not n:
                    continue
                shared = n == prefix and prefix > 0
                s = Setup(13, [7 if shared else n] * B, prefix, 4, 2, d, t, i8, 16)
                table = s.prefix_pages if shared else s.pages[0]
                at = (int(table[where // 16]), 1, where % 16)
                if i8:
                    s.cache["v"][at] = torch.where(s.cache["v"][at] == 0, 1, s.cache["v"][at]).to(torch.int8)
                want = s.call(ivit).clone()
                if i8:
                    sign = s.cache["v"][at].float().sign()
                    s.cache["v_scale"][at] = inf
                else:
                    sign = torch.where(torch.arange(d, device="cuda") % 3 == 0, -1.0, 1.0)
                    s.cache["v"][at] = (sign * inf).to(s.q.dtype)
                s.call(ivit)
                got, old = s.o.reshape(B, 2, 2 * d), want.reshape(B, 2, 2 * d)
                hit = slice(0, B if shared else 1)
                what = "%d x %d %s i8 %s prefix %d: key %d of %d" % (B, d, t, i8, prefix, where, n)
                assert torch.equal(got[hit, 1].float(), (sign * inf).repeat(2).expand(got[hit, 1].shape)), what
                assert torch.equal(got[:, 0], old[:, 0]) and (shared or torch.equal(got[1:], old[1:])), what
