"""Performance cases of attention over float rows, of its cache and of rotary positions.

  rotary  rotary positions with one or several axes on the heads of float rows                    (ivit_rotary)
  append  keys, rotated on the way, and values into a paged cache, queries rotated beside them     (ivit_cache_append)
  prompt  attention over whole prompts: packed sequences, grouped heads, causal or not             (ivit_prompt_attention)
  cached  one token per request over the paged cache, with a prefix that the batch shares          (ivit_cached_attention)

The plain forms below are elementary torch operations in 32 bits, angles in 64.  int8 caches are returned as the values they stand for
(q times its scale, in bfloat16), beside the scales.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one token of a served model, queries and keys of one layer: all latency
        {"name": "rotary_1x40x128", "op": "rotary", "rows": 1, "heads": 40, "d": 128, "rot": 128, "axes": 1, "adjacent": False, "type": "bf16"},
        # queries and keys of DeiT-S by row and column of the patch, 128 images of 197 tokens
        {"name": "rotary_25216x12x64_hw", "op": "rotary", "rows": 25216, "heads": 12, "d": 64, "rot": 64, "axes": 2, "adjacent": False, "type": "bf16"},
        # a video of odd length, three axes, adjacent pairs, part of each head turned, a stream in 32 bits
        {"name": "rotary_5003x17x80_thw_f32", "op": "rotary", "rows": 5003, "heads": 17, "d": 80, "rot": 60, "axes": 3, "adjacent": True, "type": "f32"},
        # a step of 64 requests, one token each
        {"name": "append_64_i8", "op": "append", "rows": 64, "heads": 32, "kv": 8, "d": 128, "rot": 128, "axes": 1, "adjacent": False, "type": "bf16",
         "page": 64, "cache": "i8"},
        # a long prompt on its way into the cache
        {"name": "append_16384", "op": "append", "rows": 16384, "heads": 32, "kv": 8, "d": 128, "rot": 128, "axes": 1, "adjacent": False, "type": "bf16",
         "page": 64, "cache": "same"},
        # eight images of DeiT-S, every token sees every other
        {"name": "prompt_8x197_all", "op": "prompt", "seqs": 8, "queries": 197, "past": 0, "ragged": 0, "heads": 6, "kv": 6, "d": 64, "causal": False,
         "type": "bf16"},
        # a served batch of prompts of different lengths
        {"name": "prompt_17_ragged_f16", "op": "prompt", "seqs": 17, "queries": 1500, "past": 0, "ragged": 5, "heads": 32, "kv": 8, "d": 128,
         "causal": True, "type": "f16"},
        # part of a long prompt after the part before it
        {"name": "prompt_500_after_7500", "op": "prompt", "seqs": 1, "queries": 500, "past": 7500, "ragged": 0, "heads": 32, "kv": 4, "d": 128,
         "causal": True, "type": "bf16"},
        # one long prompt: the matrix cores
        {"name": "prompt_8192", "op": "prompt", "seqs": 1, "queries": 8192, "past": 0, "ragged": 0, "heads": 32, "kv": 8, "d": 128, "causal": True,
         "type": "bf16"},
        # one request in the middle of its answer: all latency
        {"name": "cached_1x1000", "op": "cached", "requests": 1, "prefix": 0, "own": 1000, "ragged": 0, "heads": 32, "kv": 8, "d": 128, "page": 64,
         "type": "bf16", "cache": "same"},
        # requests behind one long instruction
        {"name": "cached_64_prefix_8000", "op": "cached", "requests": 64, "prefix": 8000, "own": 600, "ragged": 3, "heads": 32, "kv": 8, "d": 128, "page": 64,
         "type": "bf16", "cache": "same"},
        # long answers over an int8 cache: bytes
        {"name": "cached_48x16384_i8", "op": "cached", "requests": 48, "prefix": 1024, "own": 16384, "ragged": 7, "heads": 32, "kv": 8, "d": 128, "page": 128,
         "type": "bf16", "cache": "i8"},
    ]


def _log(rng, lo, hi):
    """A whole number of lo .. hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rotary", "append", "prompt", "prompt", "cached", "cached"))
    d = rng.choice((64, 128, 128))
    kv = _log(rng, 1, 16)
    heads = kv * rng.choice((1, 2, 4, 5, 8))
    t = rng.choice(("f16", "bf16", "bf16"))
    if op == "rotary":
        d = 2 * _log(rng, 4, 128)
        rot = d if rng.random() < 0.6 else 2 * rng.randint(1, d // 2)
        heads, rows = _log(rng, 1, 64), _log(rng, 1, 50000)
        rows = max(1, min(rows, (1 << 25) // (heads * d)))
        return {"op": op, "rows": rows, "heads": heads, "d": d, "rot": rot, "axes": rng.choice((1, 2, 3)), "adjacent": rng.random() < 0.4,
                "type": rng.choice(("f32", "f16", "bf16"))}
    if op == "append":
        rows = max(1, min(_log(rng, 1, 30000), (1 << 26) // ((heads + 2 * kv) * d)))
        return {"op": op, "rows": rows, "heads": heads, "kv": kv, "d": d, "rot": rng.choice((d, d, d // 2)), "axes": rng.choice((1, 1, 3)),
                "adjacent": rng.random() < 0.3, "type": t, "page": rng.choice((16, 32, 64, 128, 256)), "cache": rng.choice(("same", "i8"))}
    if op == "prompt":
        seqs, queries, past = _log(rng, 1, 40), _log(rng, 1, 8192), rng.choice((0, 0, _log(rng, 1, 8192)))
        queries = max(1, min(queries, 32768 // seqs))
        past = min(past, 32768 // seqs)
        while seqs * queries * (queries + past) * heads * d > 2.0 ** 37:
            queries, past = max(1, queries * 3 // 4), past * 3 // 4
        return {"op": op, "seqs": seqs, "queries": queries, "past": past, "ragged": rng.randint(0, 99), "heads": heads, "kv": kv, "d": d,
                "causal": rng.random() < 0.7, "type": t}
    requests, prefix, length = _log(rng, 1, 200), rng.choice((0, _log(rng, 1, 16384))), _log(rng, 1, 32768)
    length = max(1, min(length, (1 << 28) // (requests * kv * d)))
    prefix = min(prefix, (1 << 28) // (requests * heads * d) * 64)
    return {"op": op, "requests": requests, "prefix": prefix, "own": length, "ragged": rng.randint(0, 99), "heads": heads, "kv": kv, "d": d,
            "page": rng.choice((16, 32, 64, 128, 256)), "type": t, "cache": rng.choice(("same", "i8"))}


def _lengths(n, longest, ragged):
    """Lengths of n sequences: all the longest, or from nothing to the longest."""
    if not ragged:
        return [longest] * n
    r = random.Random(ragged)
    return [longest] + [r.randint(0, longest) for _ in range(n - 1)]


def _prompt_lengths(case):
    """(queries, keys) of each sequence"""
    nq = _lengths(case["seqs"], case["queries"], case["ragged"])
    return nq, [n + p for n, p in zip(nq, _lengths(case["seqs"], case["past"], case["ragged"]))]


def _int8_rows(v):
    """float rows -> (int8 rows, the scale of each)"""
    s = v.abs().amax(-1).clamp_min(1e-20) / 127.0
    return (v / s[..., None]).round_().to(torch.int8), s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def whole(low, high, shape):
        return torch.randint(low, high, shape, generator=g, device="cuda", dtype=torch.int32)

    def rows(n, heads):
        """[n, heads * d] of the case's type: channels of different size"""
        return (normal(n, heads * case["d"]) * torch.exp(0.3 * normal(heads * case["d"]))).to(TYPES[case["type"]])

    def starts(lengths):
        return torch.tensor([0] + lengths).cumsum(0).to(torch.int32).cuda()

    s, op, d = dict(case), case["op"], case["d"]
    if op in ("rotary", "append"):
        half, n = case["rot"] // 2, case["rows"]
        s["freq"] = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        s["axis"] = None if case["axes"] == 1 else (torch.arange(half, device="cuda") * case["axes"] // half).to(torch.int32)
        if case["axes"] == 1:           # tokens of one long text or of requests at different places of theirs
            s["positions"] = (torch.arange(n, device="cuda", dtype=torch.int32) + whole(0, 100000, (1,))) if n > 256 else whole(0, 100000, (n,))
        else:                           # tokens of images and videos
            s["positions"] = torch.stack([whole(0, (2000, 64, 64)[a], (n,)) for a in range(case["axes"])])
    if op == "rotary":
        s["x"] = rows(n, case["heads"])
        s["y"] = torch.empty_like(s["x"])
    elif op == "append":
        kv, page, i8 = case["kv"], case["page"], case["cache"] == "i8"
        s["qkv"] = rows(n, case["heads"] + 2 * kv)
        s["q_out"] = torch.zeros((n, case["heads"] * d), dtype=s["qkv"].dtype, device="cuda")
        used = -(-n // page)
        pages = used + used // 4 + 1
        at = torch.randperm(pages, generator=g, device="cuda")[:used].to(torch.int32)
        t = torch.arange(n, device="cuda")
        s["slots"] = at[t // page] * page + (t % page).to(torch.int32)
        if n > 50:                      # a batch padded behind its last token
            s["slots"][-(n // 50):] = -1
        shape = (pages, kv, page, d)
        if i8:
            (k, ks), (v, vs) = _int8_rows(normal(*shape)), _int8_rows(normal(*shape))
            s["cache"] = {"k": k, "v": v, "k_scale": ks, "v_scale": vs}
            s["values"] = [torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        else:
            s["cache"] = {"k": normal(*shape).to(s["qkv"].dtype), "v": normal(*shape).to(s["qkv"].dtype)}
    elif op == "prompt":
        nq, nk = _prompt_lengths(case)
        s["nq"], s["nk"] = nq, nk
        s["q"], s["k"], s["v"] = rows(sum(nq), case["heads"]), rows(sum(nk), case["kv"]), rows(sum(nk), case["kv"])
        s["o"] = torch.zeros_like(s["q"])
        s["q_start"], s["k_start"] = starts(nq), starts(nk)
    else:
        B, kv, page, i8 = case["requests"], case["kv"], case["page"], case["cache"] == "i8"
        s["lengths"] = _lengths(B, case["own"], case["ragged"])
        width, first = -(-case["own"] // page), -(-case["prefix"] // page)
        s["q"] = rows(B, case["heads"])
        s["o"] = torch.zeros_like(s["q"])
        s["lens"] = torch.tensor(s["lengths"], dtype=torch.int32).cuda()
        need = [-(-n // page) for n in s["lengths"]]
        at = torch.randperm(sum(need) + first, generator=g, device="cuda").to(torch.int32)
        s["prefix_pages"] = at[sum(need):].contiguous()
        table, i = torch.zeros((B, width), dtype=torch.int32, device="cuda"), 0
        for b, n in enumerate(need):
            table[b, :n] = at[i:i + n]
            i += n
        s["pages"] = table
        shape = (sum(need) + first, kv, page, d)
        if i8:
            (k, ks), (v, vs) = _int8_rows(normal(*shape)), _int8_rows(normal(*shape))
            s["cache"] = {"k": k, "v": v, "k_scale": ks, "v_scale": vs}
        else:
            s["cache"] = {"k": normal(*shape).to(s["q"].dtype), "v": normal(*shape).to(s["q"].dtype)}
        if own:
            from paper_2207_01405_amd import binding
            size = binding.ivit_cached_attention_workspace_bytes(B, case["heads"], s["cache"], width, case["prefix"])
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


def _run_own(s):
    from paper_2207_01405_amd import binding
    op, d = s["op"], s["d"]
    if op in ("rotary", "append"):
        rotary = {"positions": s["positions"], "freq": s["freq"], "axis": s["axis"], "adjacent": s["adjacent"]}
    if op == "rotary":
        return {"y": binding.ivit_rotary(s["x"], s["y"], d, rotary)}
    if op == "append":
        H, kv, qkv, c = s["heads"] * d, s["kv"] * d, s["qkv"], s["cache"]
        binding.ivit_cache_append(qkv[:, H:H + kv], qkv[:, H + kv:], s["slots"], c, rotary=rotary, q=qkv[:, :H], q_out=s["q_out"])
        if "k_scale" not in c:
            return {"q": s["q_out"], "k": c["k"], "v": c["v"], "k_scale": None, "v_scale": None}
        k, v = (torch.mul(c[n], c[n + "_scale"][..., None], out=out) for n, out in zip("kv", s["values"]))
        return {"q": s["q_out"], "k": k, "v": v, "k_scale": c["k_scale"], "v_scale": c["v_scale"]}
    if op == "prompt":
        return {"o": binding.ivit_prompt_attention(s["q"], s["k"], s["v"], s["o"], d, s["q_start"], s["k_start"], causal=s["causal"])}
    return {"o": binding.ivit_cached_attention(s["q"], s["o"], s["cache"], s["pages"], s["lens"], s["workspace"], prefix_pages=s["prefix_pages"],
                                               prefix_len=s["prefix"])}


def _turned(s, x):
    """x [rows, heads * d] with the pairs of its heads turned, in 32 bits"""
    half, n = s["rot"] // 2, s["rows"]
    p = s["positions"].reshape(s["axes"], n).double()
    p = p[0][:, None].expand(n, half) if s["axis"] is None else p[s["axis"].long()].t()
    angle = p * s["freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    x = x.float().reshape(n, -1, s["d"])
    y = x.clone()
    if s["adjacent"]:
        first, second = slice(0, s["rot"], 2), slice(1, s["rot"], 2)
    else:
        first, second = slice(0, half), slice(half, s["rot"])
    y[..., first] = x[..., first] * cos - x[..., second] * sin
    y[..., second] = x[..., second] * cos + x[..., first] * sin
    return y


def _quantised(v):
    scale = v.abs().amax(-1) / 127.0
    q = torch.round(v / torch.where(scale > 0, scale, torch.ones_like(scale))[..., None])
    return q.to(torch.int8), scale


def _attend(q, k, v, hidden=None):
    """q [heads, n, d], k and v [heads, m, d] in 32 bits -> (sum of weights times values, sum of weights, largest score); hidden [n, m]: keys left out"""
    score = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(q.shape[2])
    if hidden is not None:
        score.masked_fill_(hidden, -math.inf)
    top = score.amax(2, keepdim=True)
    weight = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    return torch.matmul(weight, v), weight.sum(2, keepdim=True), top


def run(s):
    if own:
        return _run_own(s)
    op, d = s["op"], s["d"]
    if op == "rotary":
        return {"y": _turned(s, s["x"]).reshape(s["rows"], -1).to(s["x"].dtype)}
    if op == "append":
        H, kv, page, qkv, c = s["heads"], s["kv"], s["page"], s["qkv"], s["cache"]
        x = _turned(s, qkv[:, :(H + kv) * d])
        k, v = x[:, H:], qkv[:, (H + kv) * d:].float().reshape(-1, kv, d)
        there = torch.nonzero(s["slots"] >= 0)[:, 0]
        at = s["slots"][there].long()
        at, offset = at // page, at % page
        s["q_out"][there] = x[there, :H].reshape(-1, H * d).to(qkv.dtype)
        for name, rows in (("k", k[there]), ("v", v[there])):
            if "k_scale" in c:
                c[name][at, :, offset], c[name + "_scale"][at, :, offset] = _quantised(rows)
            else:
                c[name][at, :, offset] = rows.to(qkv.dtype)
        if "k_scale" not in c:
            return {"q": s["q_out"], "k": c["k"], "v": c["v"], "k_scale": None, "v_scale": None}
        k, v = ((c[n].float() * c[n + "_scale"][..., None]).to(torch.bfloat16) for n in "kv")
        return {"q": s["q_out"], "k": k, "v": v, "k_scale": c["k_scale"], "v_scale": c["v_scale"]}
    group = s["heads"] // s["kv"]
    if op == "prompt":
        o, i, j = torch.zeros_like(s["o"]), 0, 0
        for nq, nk in zip(s["nq"], s["nk"]):
            if nq:
                q = s["q"][i:i + nq].float().reshape(nq, s["kv"], group * d)
                k, v = (s[n][j:j + nk].float().reshape(nk, s["kv"], d) for n in "kv")
                hidden = None
                if s["causal"]:
                    hidden = torch.arange(nk, device="cuda") > torch.arange(nq, device="cuda")[:, None] + (nk - nq)
                step = max(1, (1 << 28) // (nq * nk * group))
                for h in range(0, s["kv"], step):
                    e = min(s["kv"], h + step)
                    qh = q[:, h:e].reshape(nq, -1, d).transpose(0, 1).contiguous()
                    kh, vh = (x[:, h:e].transpose(0, 1).repeat_interleave(group, 0) for x in (k, v))
                    value, total, _ = _attend(qh, kh, vh, hidden)
                    value = torch.where(total > 0, value / total, torch.zeros_like(value))
                    o[i:i + nq, h * group * d:e * group * d] = value.transpose(0, 1).reshape(nq, -1).to(o.dtype)
            i, j = i + nq, j + nk
        return {"o": o}
    c, B, kv = s["cache"], s["requests"], s["kv"]

    def keys(pages, n):
        """The first n keys and values of these pages: [kv, n, d] each"""
        at = pages[:-(-n // s["page"])].long()
        both = (c[x][at].float() if "k_scale" not in c else c[x][at].float() * c[x + "_scale"][at][..., None] for x in "kv")
        return [x.transpose(0, 1).reshape(kv, -1, d)[:, :n].contiguous() for x in both]

    q = s["q"].float().reshape(B, kv, group, d).transpose(0, 1).contiguous()
    o = torch.zeros_like(q)
    if s["prefix"]:
        k, v = keys(s["prefix_pages"], s["prefix"])
        parts = [_attend(q.reshape(kv, B * group, d)[:, r:r + 512], k, v) for r in range(0, B * group, 512)]
        shared = [torch.cat([p[i] for p in parts], 1).reshape(kv, B, group, -1) for i in range(3)]
    for b, n in enumerate(s["lengths"]):
        parts = [tuple(x[:, b] for x in shared)] if s["prefix"] else []
        if n:
            k, v = keys(s["pages"][b], n)
            parts.append(_attend(q[:, b], k, v))
        if parts:
            top = torch.stack([p[2] for p in parts]).amax(0)
            value = sum(p[0] * torch.exp(p[2] - top) for p in parts)
            o[:, b] = value / sum(p[1] * torch.exp(p[2] - top) for p in parts)
    return {"o": o.transpose(0, 1).reshape(B, -1).to(s["q"].dtype)}


def work(case):
    """Each input read once, each output written once; a multiply-add is two operations."""
    op, d = case["op"], float(case["d"])
    e = {"f32": 4.0, "f16": 2.0, "bf16": 2.0}[case["type"]]
    if op == "rotary":
        x = case["rows"] * case["heads"] * d
        return {"bytes": 2.0 * e * x + 4.0 * case["rows"] * case["axes"], "flops": 3.0 * x * case["rot"] / d}
    if op == "append":
        n, q, kv = float(case["rows"]), case["heads"] * d, case["kv"] * d
        stored = kv + 4.0 * case["kv"] if case["cache"] == "i8" else e * kv
        return {"bytes": n * (e * (2.0 * q + 2.0 * kv) + 2.0 * stored + 4.0 * (1 + case["axes"])), "flops": 3.0 * n * (q + kv) * case["rot"] / d}
    if op == "prompt":
        nq, nk = _prompt_lengths(case)
        if case["causal"]:              # query i of n sees i + 1 + past keys
            pairs = sum(n * (m - n) + n * (n + 1) / 2.0 for n, m in zip(nq, nk))
        else:
            pairs = float(sum(n * m for n, m in zip(nq, nk)))
        return {"bytes": e * d * (2.0 * case["heads"] * sum(nq) + 2.0 * case["kv"] * sum(nk)), "flops": 4.0 * d * case["heads"] * pairs}
    lengths = _lengths(case["requests"], case["own"], case["ragged"])
    row = d + 4.0 if case["cache"] == "i8" else e * d
    return {"bytes": 2.0 * row * case["kv"] * (case["prefix"] + sum(lengths)) + 2.0 * e * d * case["heads"] * case["requests"],
            "flops": 4.0 * d * case["heads"] * (float(case["requests"]) * case["prefix"] + sum(lengths))}


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    f64, d, op = torch.float64, case["d"], case["op"]

    def rotated(x):
        """Pairs as complex numbers times exp(i phi)"""
        n, half = case["rows"], case["rot"] // 2
        z = x.to(f64).view(n, -1, d)
        where = s["positions"].view(case["axes"], n).to(f64)
        which = torch.zeros(half, dtype=torch.int64, device="cuda") if s["axis"] is None else s["axis"].long()
        phi = torch.stack([where[a] for a in which.tolist()], dim=1) * s["freq"]
        turn = torch.polar(torch.ones_like(phi), phi).unsqueeze(1)
        head, rest = z[..., :case["rot"]], z[..., case["rot"]:]
        if case["adjacent"]:
            pairs = torch.view_as_complex(head.reshape(n, -1, half, 2).contiguous()) * turn
            head = torch.view_as_real(pairs).flatten(-2)
        else:
            pairs = torch.complex(head[..., :half].contiguous(), head[..., half:].contiguous()) * turn
            head = torch.cat([pairs.real, pairs.imag], dim=-1)
        return torch.cat([head, rest], dim=-1)

    if op == "rotary":
        return {"y": rotated(s["x"]).flatten(1)}
    if op == "append":
        q, k, v = s["qkv"].split([case["heads"] * d, case["kv"] * d, case["kv"] * d], dim=1)
        new = {"k": rotated(k), "v": v.to(f64).view(-1, case["kv"], d)}
        q_out, q = s["q_out"].to(f64), rotated(q).flatten(1)
        slots = s["slots"].tolist()
        real = torch.tensor([i for i, slot in enumerate(slots) if slot >= 0], dtype=torch.int64, device="cuda")
        flat = torch.tensor([slot for slot in slots if slot >= 0], dtype=torch.int64, device="cuda")
        q_out[real] = q[real]
        out = {"q": q_out}
        for name in ("k", "v"):
            pool = s["cache"][name].to(f64)
            pages, kv, page, _ = pool.shape
            rows, scales = new[name][real], None
            if case["cache"] == "i8":
                scales = s["cache"][name + "_scale"].to(f64)
                pool = pool * scales.unsqueeze(-1)
                peak = rows.abs().max(dim=-1, keepdim=True).values
                rows = torch.round(rows * 127.0 / peak.clamp_min(1e-300)) * peak / 127.0
                by_token = scales.transpose(1, 2).reshape(pages * page, kv)
                by_token[flat] = peak.squeeze(-1) / 127.0
                scales = by_token.view(pages, page, kv).transpose(1, 2).contiguous()
            by_token = pool.transpose(1, 2).reshape(pages * page, kv, d)
            by_token[flat] = rows
            out[name] = by_token.view(pages, page, kv, d).transpose(1, 2).contiguous()
            out[name + "_scale"] = scales
        return out

    group = case["heads"] // case["kv"]
    if op == "prompt":
        o = torch.zeros(s["o"].shape, dtype=f64, device="cuda")
        q_at = [0]
        k_at = [0]
        for n, m in zip(s["nq"], s["nk"]):
            q_at.append(q_at[-1] + n)
            k_at.append(k_at[-1] + m)
        for n, (qa, ka, kb) in enumerate(zip(q_at, k_at, k_at[1:])):
            count, m = s["nq"][n], kb - ka
            if count == 0 or m == 0:
                continue
            for h in range(case["heads"]):
                mine = slice((h // group) * d, (h // group) * d + d)
                K, V = s["k"][ka:kb, mine].to(f64), s["v"][ka:kb, mine].to(f64)
                Kt = K.t().contiguous()
                for a in range(0, count, 4096):
                    b = min(count, a + 4096)
                    logits = torch.mm(s["q"][qa + a:qa + b, h * d:(h + 1) * d].to(f64), Kt) * d ** -0.5
                    if case["causal"]:
                        last = torch.arange(a, b, device="cuda") + m - count
                        logits[torch.arange(m, device="cuda").unsqueeze(0) > last.unsqueeze(1)] = -1e300
                    o[qa + a:qa + b, h * d:(h + 1) * d] = torch.mm(torch.softmax(logits, dim=1), V)
        return {"o": o}
    pool = [s["cache"][n].to(f64) if case["cache"] == "same" else s["cache"][n].to(f64) * s["cache"][n + "_scale"].to(f64).unsqueeze(-1) for n in "kv"]
    o = torch.zeros(s["o"].shape, dtype=f64, device="cuda")
    lead = s["prefix_pages"].long()
    for b, length in enumerate(s["lengths"]):
        tail = s["pages"][b].long()
        for h in range(case["kv"]):
            K, V = (torch.cat([x[lead, h].reshape(-1, d)[:case["prefix"]], x[tail, h].reshape(-1, d)[:length]]) for x in pool)
            if K.shape[0]:
                cols = slice(h * group * d, (h + 1) * group * d)
                logits = torch.mm(s["q"][b, cols].to(f64).view(group, d), K.t().contiguous()) * d ** -0.5
                o[b, cols] = torch.mm(torch.softmax(logits, dim=1), V).flatten()
    return {"o": o}
