"""Performance cases of the operators around int8 Dense layers whose scales are taken per token at run time.

  norm    root-mean-square norm with the residual's addition, int8 rows with a scale each    (ivit_rmsnorm_quant)
  dense   int8 Dense layer with scales, bias, activation and residual in its epilogue         (ivit_linear_scaled)
  gate    activation of an MLP's hidden rows, gated or not, int8 rows with a scale each       (ivit_gated_quant)

The plain forms below are elementary torch operations in 32 bits.  int8 results are returned as the values they stand for
(q times its scale, in bfloat16), beside the scales.
"""
import math

import torch

own = False

EPS = 1e-6
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one token of a served model between two layers: all latency
        {"name": "norm_1x4096", "op": "norm", "rows": 1, "cols": 4096, "type": "bf16", "residual": True, "out": "i8"},
        # DeiT-S, 128 images of 197 tokens
        {"name": "norm_25216x384", "op": "norm", "rows": 25216, "cols": 384, "type": "bf16", "residual": True, "out": "i8"},
        # the norm before a head: no addition, the stream's own type out; a width that no vector divides
        {"name": "norm_5003x2049_f16", "op": "norm", "rows": 5003, "cols": 2049, "type": "f16", "residual": False, "out": "same"},
        # long prompts of a wide model
        {"name": "norm_16384x4096", "op": "norm", "rows": 16384, "cols": 4096, "type": "bf16", "residual": True, "out": "i8"},
        # one token: the weights are read for it alone
        {"name": "dense_1x4096x4096", "op": "dense", "rows": 1, "n": 4096, "k": 4096, "type": "bf16", "act": "none", "bias": False,
         "residual": True, "x_scales": "rows"},
        # a batch of sixteen single tokens through a wide MLP layer
        {"name": "dense_16x11008x4096_silu", "op": "dense", "rows": 16, "n": 11008, "k": 4096, "type": "bf16", "act": "silu", "bias": False,
         "residual": False, "x_scales": "rows"},
        # first MLP layer of DeiT-S, eight images
        {"name": "dense_1576x1536x384_gelu", "op": "dense", "rows": 1576, "n": 1536, "k": 384, "type": "bf16", "act": "gelu", "bias": True,
         "residual": False, "x_scales": "rows"},
        # sizes that no tile divides, a residual stream in 32 bits
        {"name": "dense_1001x777x1040_f32", "op": "dense", "rows": 1001, "n": 777, "k": 1040, "type": "f32", "act": "gelu_tanh", "bias": True,
         "residual": True, "x_scales": "rows"},
        # QKV layer of DeiT-S, 128 images, one scale for x; int8 out at a fixed step, as the integer attention takes it
        {"name": "dense_25216x1152x384_i8", "op": "dense", "rows": 25216, "n": 1152, "k": 384, "type": "i8", "act": "none", "bias": True,
         "residual": False, "x_scales": "one"},
        # a wide layer over long prompts: the matrix cores
        {"name": "dense_8192x8192x4096", "op": "dense", "rows": 8192, "n": 8192, "k": 4096, "type": "bf16", "act": "none", "bias": True,
         "residual": True, "x_scales": "rows"},
        # MLP of DeiT-S, one image
        {"name": "gate_197x1536_gelu", "op": "gate", "rows": 197, "cols": 1536, "type": "bf16", "act": "gelu", "gated": False},
        # gated MLP of a wide model, long prompts
        {"name": "gate_8192x14336_silu", "op": "gate", "rows": 8192, "cols": 14336, "type": "bf16", "act": "silu", "gated": True},
    ]


def _log(rng, lo, hi):
    """A whole number of lo .. hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh", "gelu_sigmoid")


def draw(rng):
    op = rng.choice(("norm", "dense", "dense", "gate"))
    if op == "norm":
        rows, cols = _log(rng, 1, 50000), _log(rng, 48, 16384)
        rows = max(1, min(rows, (1 << 25) // cols))
        return {"op": op, "rows": rows, "cols": cols, "type": rng.choice(("f32", "f16", "bf16", "bf16")), "residual": rng.random() < 0.7,
                "out": rng.choice(("i8", "i8", "i8", "same"))}
    if op == "gate":
        rows, cols = _log(rng, 1, 50000), _log(rng, 48, 28672)
        rows = max(1, min(rows, (1 << 25) // cols))
        return {"op": op, "rows": rows, "cols": cols, "type": rng.choice(("f32", "f16", "bf16", "bf16")), "act": rng.choice(ACTS[1:]),
                "gated": rng.random() < 0.6}
    M, N, K = _log(rng, 1, 30000), _log(rng, 10, 16384), 16 * _log(rng, 4, 768)
    M = max(1, min(M, (1 << 25) // N, (1 << 25) // K, int(2.5e11 / (N * K))))
    t = rng.choice(("f32", "f16", "bf16", "bf16", "i8"))
    return {"op": op, "rows": M, "n": N, "k": K, "type": t, "act": rng.choice(ACTS), "bias": rng.random() < 0.7,
            "residual": t != "i8" and rng.random() < 0.5, "x_scales": rng.choice(("rows", "rows", "one"))}


def _int8_rows(v):
    """float rows -> (int8 rows, the scale of each)"""
    s = v.abs().amax(1).clamp_min(1e-20) / 127.0
    return (v / s[:, None]).round_().to(torch.int8), s


def case_step(case):
    """The step of an int8 result: four deviations of the sums at the ends of its range."""
    return 4.0 * 0.02 * math.sqrt(case["k"]) / 127.0


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def buffer(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    s, op, rows = dict(case), case["op"], case["rows"]
    if op == "norm":
        C, t = case["cols"], TYPES[case["type"]]
        dev = torch.exp(0.4 * normal(C))            # of the channels: most near 1, some several times that
        s["x"] = (normal(rows, C) * dev).to(t)
        s["r"] = (normal(rows, C) * dev).to(t) if case["residual"] else None
        s["gamma"] = 1.0 + 0.1 * normal(C)
        s["sum"] = buffer((rows, C), t) if case["residual"] else None
        s["y"] = buffer((rows, C), torch.int8 if case["out"] == "i8" else t)
        s["scale"] = buffer((rows,), torch.float32) if case["out"] == "i8" else None
        s["value"] = buffer((rows, C), torch.bfloat16) if case["out"] == "i8" else None
    elif op == "gate":
        C, t = case["cols"], TYPES[case["type"]]
        s["x"] = (1.5 * normal(rows, 2 * C if case["gated"] else C)).to(t)
        s["y"], s["scale"] = buffer((rows, C), torch.int8), buffer((rows,), torch.float32)
        s["value"] = buffer((rows, C), torch.bfloat16)
    else:
        N, K, i8 = case["n"], case["k"], case["type"] == "i8"
        v = normal(rows, K)
        if case["x_scales"] == "rows":
            s["x"], s["x_scale"] = _int8_rows(v * torch.exp(0.3 * normal(rows, 1)))
        else:
            s["x"], s["x_scale"] = (v * 32.0).round_().clamp_(-127, 127).to(torch.int8), torch.full((1,), 1.0 / 32.0, device="cuda")
        s["w"], s["w_scale"] = _int8_rows(0.02 * normal(N, K))
        s["bias"] = 0.1 * normal(N) if case["bias"] else None
        s["step"] = case_step(case) if i8 else None
        t = torch.int8 if i8 else TYPES[case["type"]]
        s["r"] = normal(rows, N).to(t) if case["residual"] else None
        s["y"] = buffer((rows, N), t)
        s["value"] = buffer((rows, N), torch.bfloat16) if i8 else None
    return s


def _act(v, act):
    if act == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "gelu_sigmoid":
        return v / (1.0 + torch.exp(-1.702 * v))
    return v


def _quantised(v):
    """Rows of 32-bit values -> (the values that their int8 forms stand for, the scales)"""
    scale = v.abs().amax(1) / 127.0
    q = torch.round(v / torch.where(scale > 0, scale, torch.ones_like(scale))[:, None])
    return (q * scale[:, None]).to(torch.bfloat16), scale


def _run_own(s):
    from paper_2207_01405_amd import binding
    op = s["op"]
    if op == "norm":
        binding.ivit_rmsnorm_quant(s["x"], s["gamma"], s["y"], s["scale"], EPS, residual=s["r"], sum_out=s["sum"])
        y = s["y"] if s["scale"] is None else torch.mul(s["y"], s["scale"][:, None], out=s["value"])
        return {"sum": s["sum"], "y": y, "scale": s["scale"]}
    if op == "gate":
        binding.ivit_gated_quant(s["x"], s["y"], s["scale"], act=s["act"], gated=s["gated"])
        return {"y": torch.mul(s["y"], s["scale"][:, None], out=s["value"]), "scale": s["scale"]}
    binding.ivit_linear_scaled(s["x"], s["x_scale"], s["w"], s["w_scale"], s["y"], bias=s["bias"], act=s["act"], residual=s["r"],
                               y_step=s["step"])
    return {"y": s["y"] if s["step"] is None else torch.mul(s["y"], s["step"], out=s["value"])}


def run(s):
    if own:
        return _run_own(s)
    op = s["op"]
    if op == "norm":
        h = s["x"].float()
        if s["r"] is not None:
            h = h + s["r"].float()
        total = None if s["r"] is None else h.to(s["x"].dtype)
        n = h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * s["gamma"]
        if s["out"] != "i8":
            return {"sum": total, "y": n.to(s["x"].dtype), "scale": None}
        y, scale = _quantised(n)
        return {"sum": total, "y": y, "scale": scale}
    if op == "gate":
        x, C = s["x"].float(), s["cols"]
        v = _act(x[:, :C], s["act"])
        if s["gated"]:
            v = v * x[:, C:]
        y, scale = _quantised(v)
        return {"y": y, "scale": scale}
    v = (s["x"].float() @ s["w"].float().t()) * s["x_scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        v = v + s["bias"]
    v = _act(v, s["act"])
    if s["step"] is not None:
        return {"y": (torch.round(v / s["step"]).clamp(-127, 127) * s["step"]).to(torch.bfloat16)}
    if s["r"] is not None:
        v = v + s["r"].float()
    return {"y": v.to(s["y"].dtype)}


def work(case):
    """Each input read once, each output written once; a multiply-add is two operations."""
    e = {"f32": 4.0, "f16": 2.0, "bf16": 2.0, "i8": 1.0}[case["type"]]
    rows = float(case["rows"])
    if case["op"] == "norm":
        C, r = float(case["cols"]), case["residual"]
        out = rows * C + 4.0 * rows if case["out"] == "i8" else e * rows * C
        return {"bytes": e * rows * C * (3 if r else 1) + out + 4.0 * C, "flops": (7.0 if r else 6.0) * rows * C}
    if case["op"] == "gate":
        C = float(case["cols"])
        return {"bytes": e * rows * C * (2 if case["gated"] else 1) + rows * C + 4.0 * rows, "flops": 10.0 * rows * C}
    N, K = float(case["n"]), float(case["k"])
    params = N * K + 4.0 * N * (2 if case["bias"] else 1) + 4.0 * (rows if case["x_scales"] == "rows" else 1.0)
    return {"bytes": rows * K + params + e * rows * N * (2 if case["residual"] else 1), "flops": 2.0 * rows * N * K}


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    f64 = torch.float64

    def activation(z):
        kind = case["act"]
        if kind == "none":
            return z
        if kind == "relu":
            return z.clamp_min(0.0)
        if kind == "gelu":
            return z * torch.special.ndtr(z)
        slope = {"silu": z, "gelu_sigmoid": 1.702 * z}.get(kind)
        if slope is None:                       # (1 + tanh a) / 2 = sigma(2 a)
            slope = 2.0 * (2.0 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)
        return z * torch.sigmoid(slope)

    def as_int8(z):
        top = z.abs().max(dim=1, keepdim=True).values
        levels = torch.round(z * 127.0 / top.clamp_min(1e-300))
        return levels * top / 127.0, top.squeeze(1) / 127.0

    if case["op"] == "norm":
        z = s["x"].to(f64)
        if case["residual"]:
            z = z + s["r"].to(f64)
        n = s["gamma"].to(f64) * z * (z.square().sum(1, keepdim=True) / case["cols"] + EPS).rsqrt()
        y, scale = as_int8(n) if case["out"] == "i8" else (n, None)
        return {"sum": z if case["residual"] else None, "y": y, "scale": scale}
    if case["op"] == "gate":
        halves = s["x"].to(f64).split(case["cols"], dim=1)
        z = activation(halves[0])
        y, scale = as_int8(z * halves[1] if case["gated"] else z)
        return {"y": y, "scale": scale}
    z = torch.mm(s["x"].to(f64), s["w"].to(f64).t().contiguous())
    z *= s["x_scale"].to(f64).reshape(-1, 1) * s["w_scale"].to(f64).reshape(1, -1)
    if case["bias"]:
        z += s["bias"].to(f64)
    z = activation(z)
    if case["type"] == "i8":
        return {"y": torch.round(z / case_step(case)).clamp(-127.0, 127.0) * case_step(case)}
    return {"y": z + s["r"].to(f64) if case["residual"] else z}
