"""The operators of attention over float rows together, as a model of quantised layers uses them; their forms; streams, graphs, far offsets, the trace."""
import math

import pytest

from attention_rows import attend64, check, dtype, gen, rand
from test_gpu_prompt_attention import compare, run, starts

pytestmark = pytest.mark.gpu

H, G, D, C, PAGE = 4, 2, 64, 256, 16


class Layer:
    """Attention's half of a block: norm, qkv layer, rotary positions, cache, attention, projection with the residual."""

    def __init__(self, ivit, seed, t, i8, requests, most):
        import torch
        g = gen(seed)
        self.ivit, self.t, self.i8, self.B = ivit, t, i8, requests
        self.w_qkv, self.s_qkv = self.weights(g, (H + 2 * G) * D, C)
        self.w_out, self.s_out = self.weights(g, C, H * D)
        self.gamma = 1.0 + 0.1 * rand(g, C)
        self.freq = 10000.0 ** (-torch.arange(D // 2, device="cuda", dtype=torch.float64) / (D // 2))
        width = -(-most // PAGE)
        pages = requests * width + 3
        self.table = torch.randperm(pages, generator=g, device="cuda")[:requests * width].to(torch.int32).reshape(requests, width)
        shape = (pages, G, PAGE, D)
        if i8:
            self.cache = {n: torch.zeros(shape, dtype=torch.int8, device="cuda") for n in "kv"}
            self.cache.update({n + "_scale": torch.full(shape[:3], math.nan, device="cuda") for n in "kv"})
        else:
            self.cache = {n: torch.full(shape, math.nan, dtype=dtype(t), device="cuda") for n in "kv"}
        size = ivit.ivit_cached_attention_workspace_bytes(requests, H, self.cache, width, most)
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    @staticmethod
    def weights(g, n, k):
        import torch
        w = rand(g, n, k) * k ** -0.5
        s = w.abs().amax(1) / 127
        return (w / s[:, None]).round().to(torch.int8), s

    def qkv(self, x):
        import torch
        n = x.shape[0]
        q, s = torch.empty(n, C, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        self.ivit.ivit_rmsnorm_quant(x, self.gamma, q, s, 1e-6)
        rows = torch.empty(n, (H + 2 * G) * D, dtype=dtype(self.t), device="cuda")
        return self.ivit.ivit_linear_scaled(q, s, self.w_qkv, self.s_qkv, rows)

    def project(self, o, x):
        import torch
        n = x.shape[0]
        q, s = torch.empty(n, H * D, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        self.ivit.ivit_gated_quant(o, q, s, act="none", gated=False)
        return self.ivit.ivit_linear_scaled(q, s, self.w_out, self.s_out, torch.empty_like(x), residual=x)

    def slots(self, request, position):
        """Of tokens by request and position, on the device."""
        return self.table[request, position // PAGE] * PAGE + (position % PAGE).to(self.table.dtype)

    def prompt(self, x, lengths):
        import torch
        rows = self.qkv(x)
        q, k, v = rows[:, :H * D], rows[:, H * D:(H + G) * D], rows[:, (H + G) * D:]
        position = torch.cat([torch.arange(n, device="cuda") for n in lengths])
        request = torch.cat([torch.full((n,), i, device="cuda") for i, n in enumerate(lengths)])
        turn = {"positions": position.to(torch.int32), "freq": self.freq}
        self.ivit.ivit_rotary(rows[:, :(H + G) * D], rows[:, :(H + G) * D], D, turn)
        self.ivit.ivit_cache_append(k, v, self.slots(request, position), self.cache)
        o = torch.empty(x.shape[0], H * D, dtype=rows.dtype, device="cuda")
        self.ivit.ivit_prompt_attention(q, k, v, o, D, starts(lengths))
        return self.project(o, x), rows, o

    def token(self, x, lens, prefix=0):
        """One more token of every request; lens: those in the cache behind the prefix, on the device."""
        import torch
        rows = self.qkv(x)
        position = (lens + prefix).long()
        q = torch.empty(self.B, H * D, dtype=rows.dtype, device="cuda")
        self.ivit.ivit_cache_append(rows[:, H * D:(H + G) * D], rows[:, (H + G) * D:], self.slots(torch.arange(self.B, device="cuda"), position), self.cache,
                                    rotary={"positions": position.to(torch.int32), "freq": self.freq}, q=rows[:, :H * D], q_out=q)
        o = torch.empty_like(q)
        first = prefix // PAGE
        self.ivit.ivit_cached_attention(q, o, self.cache, self.table[:, first:], lens + 1, self.ws, prefix_pages=self.table[0, :first].contiguous(), prefix_len=prefix)
        return self.project(o, x), q, o

    def keys(self, b, n, h):
        import torch
        at = self.table[b, :-(-n // PAGE)].long()
        out = []
        for name in "kv":
            c = self.cache[name][at, h].double()
            if self.i8:
                c = c * self.cache[name + "_scale"][at, h].double()[..., None]
            out.append(c.reshape(-1, D)[:n])
        return out

    def check_token(self, q, o, lengths, what):
        for b, n in enumerate(lengths):
            for h in range(H):
                k, v = self.keys(b, n, h * G // H)
                cols = slice(h * D, h * D + D)
                want, pv, err, _ = attend64(q[b:b + 1, cols].double(), k, v, D ** -0.5)
                check(o[b:b + 1, cols], want, pv, err, n, self.t, float(v.abs().max()), "%s: request %d head %d" % (what, b, h), scaled=2.0 ** -22)


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("i8", [False, True])
def test_prompts_and_then_token_by_token(ivit, t, i8):
    import torch
    lengths, steps = [37, 5, 64], 20
    layer = Layer(ivit, 3, t, i8, len(lengths), 128)
    g = gen(4)
    x = rand(g, sum(lengths), C).to(dtype(t))
    y, rows, o = layer.prompt(x, lengths)
    compare(o, rows[:, :H * D], rows[:, H * D:(H + G) * D], rows[:, (H + G) * D:], lengths, lengths, H, G, D, True, D ** -0.5, t, "prompt")
    assert bool(y.isfinite().all())
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    for s in range(steps):
        x = rand(g, len(lengths), C).to(dtype(t))
        y, q, o = layer.token(x, lens + s)
        layer.check_token(q, o, [n + s + 1 for n in lengths], "step %d" % s)
        assert bool(y.isfinite().all())
    if not i8:                  # a prompt a token longer than those in the cache: its last rows are what the step gave
        whole = [rand(g, n, (H + 2 * G) * D).to(dtype(t)) for n in (41, 90)]
        cache = Layer(ivit, 5, t, False, 2, 96)
        for b, r in enumerate(whole):
            at = torch.arange(r.shape[0], device="cuda")
            ivit.ivit_cache_append(r[:, H * D:(H + G) * D], r[:, (H + G) * D:], cache.slots(torch.full_like(at, b), at), cache.cache)
        r = torch.cat(whole)
        full = torch.empty(r.shape[0], H * D, dtype=r.dtype, device="cuda")
        ivit.ivit_prompt_attention(r[:, :H * D], r[:, H * D:(H + G) * D], r[:, (H + G) * D:], full, D, starts([41, 90]))
        last = torch.stack([w[-1, :H * D] for w in whole])
        o = torch.empty_like(last)
        ivit.ivit_cached_attention(last, o, cache.cache, cache.table, torch.tensor([41, 90], dtype=torch.int32, device="cuda"), cache.ws)
        # both within their bound of one value; that of sums over at most 90 keys of values below 5: three half steps of 5
        assert float((o.double() - full[[40, 130]].double()).abs().max()) <= 6 * 5 * torch.finfo(dtype(t)).eps / 2


@pytest.mark.parametrize("i8", [False, True])
def test_a_shared_prefix_gives_what_its_copies_give(ivit, i8):
    import torch
    t, B, prefix = "bf16", 5, 64
    layer = Layer(ivit, 9, t, i8, B, 128)
    layer.table[:, :prefix // PAGE] = layer.table[0, :prefix // PAGE].clone()             # the prefix's pages in every table
    g = gen(10)
    x = rand(g, prefix, C).to(dtype(t))
    layer.prompt(x, [prefix])
    lens = torch.tensor([0, 3, 16, 17, 40], dtype=torch.int32, device="cuda")
    for b, n in enumerate(lens.tolist()):
        if n:
            r = layer.qkv(rand(g, n, C).to(dtype(t)))
            at = torch.arange(prefix, prefix + n, device="cuda")
            ivit.ivit_cache_append(r[:, H * D:(H + G) * D], r[:, (H + G) * D:], layer.slots(torch.full_like(at, b), at), layer.cache)
    x = rand(g, B, C).to(dtype(t))
    _, q, o = layer.token(x, lens, prefix)
    layer.check_token(q, o, [prefix + n + 1 for n in lens.tolist()], "prefix")
    alone = torch.empty_like(o)
    ivit.ivit_cached_attention(q, alone, layer.cache, layer.table, lens + 1 + prefix, layer.ws)
    layer.check_token(q, alone, [prefix + n + 1 for n in lens.tolist()], "alone")


@pytest.mark.parametrize("i8", [False, True])
def test_steps_from_a_graph(ivit, i8):
    """A step captured once and replayed for 12 tokens, with eager work of the same layer between the replays, against eager steps bit for bit."""
    import torch
    t, lengths = "bf16", [20, 33, 1]
    pair = [Layer(ivit, 3, t, i8, 3, 96) for _ in range(2)]
    g = gen(8)
    x = rand(g, sum(lengths), C).to(dtype(t))
    for layer in pair:
        layer.prompt(x, lengths)
    stream = torch.cuda.Stream()
    static_x = torch.zeros(3, C, dtype=dtype(t), device="cuda")
    static_lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        static_y, static_q, static_o = pair[0].token(static_x, static_lens)
    for s in range(12):
        x = rand(g, 3, C).to(dtype(t))
        static_x.copy_(x)
        static_lens.copy_(torch.tensor(lengths, device="cuda") + s)
        graph.replay()
        y, q, o = pair[1].token(x, torch.tensor(lengths, dtype=torch.int32, device="cuda") + s)
        if s % 3 == 0:
            torch.cuda.synchronize()
        assert torch.equal(static_q, q) and torch.equal(static_o, o) and torch.equal(static_y, y), "step %d" % s
    for n, c in pair[0].cache.items():
        d = pair[1].cache[n]
        assert torch.equal(c.nan_to_num(7), d.nan_to_num(7)) if c.dtype != torch.int8 else torch.equal(c, d), n


def test_prompts_from_a_graph_and_on_two_streams(ivit):
    import torch
    t, lengths = "bf16", [50, 90]
    layers = [Layer(ivit, 3 + i, t, False, 2, 96) for i in range(2)]
    g = gen(1)
    x = rand(g, 140, C).to(dtype(t))
    want = [layer.prompt(x, lengths)[0].clone() for layer in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    got = []
    for _ in range(3):
        for layer, s in zip(layers, streams):
            with torch.cuda.stream(s):
                got.append(layer.prompt(x, lengths)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[i % 2]) for i, a in enumerate(got))
    # one call of its own on a given stream
    q, k, v = (rand(g, 140, n * D).bfloat16() for n in (H, G, G))
    o, p, st = torch.empty_like(q), torch.empty_like(q), starts(lengths)
    ivit.ivit_prompt_attention(q, k, v, o, D, st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        ivit.ivit_prompt_attention(q, k, v, p, D, st)
    for s in range(3):
        p.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, p)
        st.copy_(starts([50 + s, 90 - s]))                            # (the lengths are read when the graph runs)
        ivit.ivit_prompt_attention(q, k, v, o, D, st)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, p)
        st.copy_(starts(lengths))
        ivit.ivit_prompt_attention(q, k, v, o, D, st)
    ivit.ivit_prompt_attention(q, k, v, p.zero_(), D, st, stream=torch.cuda.current_stream())
    assert torch.equal(o, p)


# few workgroups, as many as CUs or fewer, more: the keys shared by four groups of wavefronts, by two, not at all
FORMS = [(1, 40, 2), (1, 200, 8), (3, 300, 20), (3, 170, 60), (2, 700, 96), (1, 129, 256)]


@pytest.mark.parametrize("seqs,n,heads", FORMS)
def test_forms_of_prompt_attention(ivit, seqs, n, heads):
    for d, t in ((64, "bf16"), (128, "bf16"), (128, "f16")):
        for causal in (True, False):
            run(ivit, n, [n] * seqs, [n] * seqs, heads, heads // 2, d, causal, t)
            run(ivit, n, [n] * seqs, [n + 333] * seqs, heads, heads // 2, d, causal, t)
            run(ivit, n, [n - 39 * i for i in range(seqs)], [n // 2] * seqs, heads, heads // 2, d, causal, t)


@pytest.mark.parametrize("heads", [2, 60, 256])
def test_what_is_left_out_has_no_part_in_any_form(ivit, heads):
    import torch
    for d in (64, 128):
        g = gen(heads)
        n, first = 200, 70
        q, k, v = (rand(g, n, heads * d).bfloat16() for _ in range(3))
        clean = k.clone(), v.clone()
        k[first::9], v[first::5] = math.nan, math.inf
        v[first::7] = math.nan
        o = torch.empty_like(q)
        ivit.ivit_prompt_attention(q, k, v, o, d, starts([n]))
        compare(o[:first], q[:first], clean[0][:first], clean[1][:first], [first], [first], heads, heads, d, True, d ** -0.5, "bf16", "%d heads of %d" % (heads, d))
        assert not bool(o[first:].reshape(n - first, -1).isfinite().all(1).any())


def test_offsets_that_pass_32_bits(ivit):
    import torch
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    g = gen(2)
    # rows 2 MB apart, 6 GB in all
    n, ld = 3000, 1 << 20
    big = torch.empty(n * ld, dtype=torch.bfloat16, device="cuda").as_strided((n, ld), (ld, 1))
    q, k, v, o = (big[:, 1000 * i:1000 * i + 64] for i in range(4))
    for x in (q, k, v):
        x.copy_(rand(g, n, 64))
    ivit.ivit_prompt_attention(q, k, v, o, 64, starts([n]))
    small = [x.contiguous() for x in (q, k, v)]
    p = torch.empty_like(small[0])
    ivit.ivit_prompt_attention(*small, p, 64, starts([n]))
    assert torch.equal(o, p)
    r = {"positions": torch.arange(n, dtype=torch.int32, device="cuda"), "freq": 1.0 / (1.0 + torch.arange(32, device="cuda", dtype=torch.float64))}
    ivit.ivit_rotary(q, o, 64, r)
    assert torch.equal(o, ivit.ivit_rotary(small[0], p, 64, r))
    del big, q, k, v, o
    # a cache of 5 GB each, of which the last pages are used, and pages of an 80 KB stride
    for pages, stride in ((40000, 64 * 8 * 128), (65000, 40960)):
        heads = stride // (64 * 128)
        caches = [torch.empty(pages * stride, dtype=torch.bfloat16, device="cuda").as_strided((pages, heads, 64, 128), (stride, 64 * 128, 128, 1)) for _ in range(2)]
        near = [torch.empty((8, heads, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        rows = rand(g, 500, 2 * heads * 128).bfloat16()
        k, v = rows[:, :heads * 128], rows[:, heads * 128:]
        at = torch.arange(500, device="cuda", dtype=torch.int32)
        ivit.ivit_cache_append(k, v, at + (pages - 8) * 64, dict(zip("kv", caches)))
        ivit.ivit_cache_append(k, v, at, dict(zip("kv", near)))
        for a, b in zip(caches, near):
            assert torch.equal(a[-8:-1], b[:7])
        q = rand(g, 2, heads * 2 * 128).bfloat16()
        out = []
        for c, first in ((caches, pages - 8), (near, 0)):
            c = dict(zip("kv", c))
            table = (torch.arange(8, device="cuda", dtype=torch.int32) + first).reshape(1, 8).expand(2, 8).contiguous()
            ws = torch.empty(ivit.ivit_cached_attention_workspace_bytes(2, heads * 2, c, 8, 70), dtype=torch.uint8, device="cuda")
            out.append(ivit.ivit_cached_attention(q, torch.empty_like(q), c, table, torch.tensor([500, 90], dtype=torch.int32, device="cuda"), ws,
                                                  prefix_pages=table[0, 2:4].contiguous(), prefix_len=70))
        assert torch.equal(*out)
        del caches, near


def test_trace(ivit):
    import torch
    layer = Layer(ivit, 3, "bf16", False, 2, 96)
    g = gen(1)
    ivit.ivit_trace_begin(100)
    layer.prompt(rand(g, 60, C).bfloat16(), [20, 40])
    layer.token(rand(g, 2, C).bfloat16(), torch.tensor([20, 40], dtype=torch.int32, device="cuda"), 16)
    rec = ivit.ivit_trace_end(100)
    assert [ivit.KIND_NAMES[r[1]] for r in rec] == ["rmsnorm", "gemm_scaled", "rotary", "cache_append", "prompt_attention", "gated", "gemm_scaled",
                                                    "rmsnorm", "gemm_scaled", "cache_append", "cached_attention", "cached_attention_join", "gated", "gemm_scaled"]
    assert all(r[0] > 0 and r[3] > 0 for r in rec)


def test_empty_calls(ivit):
    import torch
    z = torch.zeros(0, 128, device="cuda").bfloat16()
    x = rand(gen(1), 4, 128).bfloat16()
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    c = {"k": torch.zeros(2, 2, 16, 64, device="cuda").bfloat16(), "v": torch.zeros(2, 2, 16, 64, device="cuda").bfloat16()}
    ivit.ivit_rotary(z, z, 64, {"positions": none, "freq": torch.ones(32, device="cuda", dtype=torch.float64)})
    ivit.ivit_cache_append(z, z, none, c)
    ivit.ivit_prompt_attention(z, z, z, z, 64, torch.zeros(1, dtype=torch.int32, device="cuda"))
    ivit.ivit_prompt_attention(z, z, z, z, 64, torch.zeros(3, dtype=torch.int32, device="cuda"))
    o = torch.full_like(x, 5.0)
    ivit.ivit_prompt_attention(x, z, z, o, 64, starts([4]), starts([0]))
    assert not bool(o.any())
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    ivit.ivit_cached_attention(z, z, c, torch.zeros(0, 3, dtype=torch.int32, device="cuda"), none, ws)
    o.fill_(5.0)
    ivit.ivit_cached_attention(x, o, c, torch.zeros(4, 0, dtype=torch.int32, device="cuda"), torch.tensor([0, 3, -1, 0], dtype=torch.int32, device="cuda"), ws)
    assert not bool(o[[0, 1, 3]].any()) and bool((o[2] == 5).all())
