"""Performance cases of the 8-bit layers: what a user calls who runs drafts with 8-bit linear layers.

Three operators, at the layer shapes of the networks the library runs (the 1.3B- and 14B-shaped transformers and
the small ones of the tests) and at generic ragged ones:

* *quant*: rows of activations or weights to 8-bit integers with one scale a row;
* *linear*: the matrix product of 8-bit rows and 8-bit weights with a scale for each token and each output channel,
  and the epilogues of the library's linear layers (bias, GELU, gated residual with the cache copy);
* *norm*: the seam between two blocks, h = alpha x + gate norm(y), then the next block's modulated norm of h, as
  activations or as the 8-bit rows the next product reads.

8-bit outputs come back as the values they stand for, integer times the row's scale in fp32, with the scales.  A code
is the nearest integer to value / scale, so values next to a border between two codes decide it: where a case has
8-bit outputs the plain forms compute in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-6
TINY = 2.0 ** -126          # smallest row scale: the scale of a row of zeros
ACT = {"bf16": torch.bfloat16, "fp32": torch.float32}
# (hidden, MLP width) of the networks, and the text width of the larger ones
NETS = {"tiny": (64, 256), "mid": (256, 704), "wan1.3b": (1536, 8960), "wan14b": (5120, 13824)}


def listed():
    return [
        # the smallest call: one token's activations before an 8-bit layer, all launch latency
        quant_case("quant one token bf16", "bf16", 1, 1536),
        # GELU outputs of a pool of 16 candidates before the MLP down-projection
        quant_case("quant mlp hidden pool16 bf16", "bf16", 24960, 8960),
        # MLP up weights of a 14B-shaped block, quantised once when a model is loaded
        quant_case("quant weights 14b fp32", "fp32", 13824, 5120),
        # one token through the MLP up-projection: the weights are read once, nothing else counts
        linear_case("linear one token gelu bf16", "bf16", 1, 8960, 1536, "gelu"),
        # odd sizes on every axis (rows that start on no 16-byte boundary), fp32 activations
        linear_case("linear odd fp32", "fp32", 389, 701, 253, "store"),
        # one candidate's QKV projection
        linear_case("linear qkv one bf16", "bf16", 1560, 4608, 1536, "store"),
        # one candidate's MLP down-projection: few tiles, long sums, gated residual and cache copy
        linear_case("linear mlp down one bf16", "bf16", 1560, 1536, 8960, "residual"),
        # the widest layer of the draft: MLP up-projection of 16 candidates
        linear_case("linear mlp up pool16 bf16", "bf16", 24960, 8960, 1536, "gelu"),
        # MLP down-projection of a 14B-shaped block, 4 candidates of 4096 tokens
        linear_case("linear mlp down 14b bf16", "bf16", 16384, 5120, 13824, "residual"),
        # one token between two blocks
        norm_case("norm one token to 8 bits bf16", "bf16", 1, 1536, "rms", "layer", "i8"),
        # the pool's residual stream between attention and MLP, out as the 8-bit rows of the next product
        norm_case("norm pool16 to 8 bits bf16", "bf16", 24960, 1536, "rms", "layer", "i8"),
        # 14B-shaped stream without a norm after the block, out as activations
        norm_case("norm 14b bf16", "bf16", 16384, 5120, "none", "rms", "act"),
    ]


def quant_case(name, dtype, m, k):
    return {"name": name, "kind": "quant", "dtype": dtype, "m": m, "k": k}


def linear_case(name, dtype, m, n, k, epilogue):
    return {"name": name, "kind": "linear", "dtype": dtype, "m": m, "n": n, "k": k, "epilogue": epilogue}


def norm_case(name, dtype, m, d, post, pre, out):
    """post, pre: the norms after and before a block; out: "act" or "i8"."""
    return {"name": name, "kind": "norm", "dtype": dtype, "m": m, "d": d, "post": post, "pre": pre, "out": out}


# ------------------------------------------------------------------------------------------ drawn cases
def log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


MOST_FLOPS = 2.3e12                    # below the largest listed product
MOST_VALUES = {"quant": 2.2e8, "norm": 8e7}


def draw(rng):
    while True:
        kind = rng.choices(["linear", "quant", "norm"], [5, 2, 3])[0]
        dtype = rng.choices(["bf16", "fp32"], [3, 1])[0]
        if kind == "linear":
            d, f = NETS[rng.choices(list(NETS), [1, 2, 3, 2])[0]]
            n, k = rng.choice([(d, d), (f, d), (d, f)])
            if rng.random() < 0.35:            # generic sizes, odd ones among them
                n, k = log_int(rng, 5, 12000), log_int(rng, 9, 12000)
            case = linear_case("", dtype, log_int(rng, 1, 26000), n, k,
                               rng.choice(["store", "gelu", "store_f32", "residual"]))
            fits = 2.0 * case["m"] * n * k <= MOST_FLOPS
        elif kind == "quant":
            k = rng.choice([rng.choice([s for net in NETS.values() for s in net]), log_int(rng, 1, 40000)])
            case = quant_case("", dtype, log_int(rng, 1, 26000), k)
            fits = case["m"] * k <= MOST_VALUES[kind]
        else:
            d = rng.choice([rng.choice([net[0] for net in NETS.values()]), log_int(rng, 1, 6144)])
            case = norm_case("", dtype, log_int(rng, 1, 26000), d, rng.choice(["none", "layer", "rms"]),
                             rng.choice(["layer", "rms"]), rng.choice(["act", "i8"]))
            fits = case["m"] * d <= MOST_VALUES[kind]
        if fits:
            case.pop("name")
            return case


# -------------------------------------------------------------------------------------------- inputs
def normal(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device="cuda") * std


def codes(gen, rows, k):
    """8-bit rows of normal values with a few wide channels, every row's largest at 127, and a scale a row."""
    x = normal(gen, rows, k) * torch.exp(normal(gen, k, std=0.4))
    x *= 127.0 / x.abs().amax(1, keepdim=True)
    return x.round_().to(torch.int8), torch.exp(normal(gen, rows, std=0.2))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    act = ACT[case["dtype"]]
    m = case["m"]
    s = dict(case)
    if case["kind"] == "quant":
        s["x"] = (normal(gen, m, case["k"]) * torch.exp(normal(gen, m, 1, std=0.5))).to(act)
        s["q"] = torch.empty(m, case["k"], dtype=torch.int8, device="cuda")
        s["scale"] = torch.empty(m, device="cuda")
    elif case["kind"] == "linear":
        n, k = case["n"], case["k"]
        s["a"], s["sa"] = codes(gen, m, k)
        s["w"], s["sw"] = codes(gen, n, k)
        s["sa"] *= 3.0 / 127          # rows of unit variance
        s["sw"] *= 4.0 * 0.02 / 127   # weights of standard deviation 0.02
        s["bias"] = normal(gen, n, std=0.02)
        residual = case["epilogue"] == "residual"
        s["gate"] = normal(gen, n, std=0.5) if residual else None
        s["h"] = normal(gen, m, n) if residual else None
        s["y"] = torch.empty(m, n, dtype=act if case["epilogue"] in ("store", "gelu") else torch.float32, device="cuda")
        s["cache"] = torch.empty(m, n, device="cuda") if residual else None
    else:
        d = case["d"]
        s["x"] = normal(gen, m, d) + normal(gen, d, std=0.5)
        s["branch"] = normal(gen, m, d, std=0.7).to(act)
        s["alpha"] = 0.75
        s["gain"] = 1.0 + normal(gen, d, std=0.1)
        s["gate"] = normal(gen, d, std=0.5)
        s["shift"], s["scale"] = normal(gen, d, std=0.3), normal(gen, d, std=0.3)
        s["h"] = torch.empty(m, d, device="cuda")
        if case["out"] == "i8":
            s["q"] = torch.empty(m, d, dtype=torch.int8, device="cuda")
            s["qs"] = torch.empty(m, device="cuda")
        else:
            s["act"] = torch.empty(m, d, dtype=act, device="cuda")
    return s


# ------------------------------------------------------------------------------------------ plain forms
def plain_codes(v):
    """Rows of 64-bit values to the values their 8-bit codes stand for, and the scales (fp32)."""
    scale = (v.abs().amax(1) / 127).float().clamp_min(TINY)
    q = torch.round(v / scale.double()[:, None])
    return q.float() * scale[:, None], scale


def plain_norm(v, kind):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    return v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)


def plain_quant(s):
    values, scale = plain_codes(s["x"].double())
    return {"values": values, "scale": scale}


def plain_linear(s):
    v = (s["a"].float() @ s["w"].float().t()) * s["sw"] * s["sa"][:, None] + s["bias"]
    if s["epilogue"] == "residual":
        h = s["h"] + s["gate"] * v
        return {"h": h, "cache": h.clone()}
    if s["epilogue"] == "gelu":
        v = 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    return {"y": v.to(s["y"].dtype)}


def plain_seam(s):
    wide = torch.float64 if s["out"] == "i8" else torch.float32
    u = plain_norm(s["branch"].to(wide), s["post"]) * s["gain"].to(wide)
    h = (s["alpha"] * s["x"].to(wide) + s["gate"].to(wide) * u).float()
    a = plain_norm(h.to(wide), s["pre"]) * (1 + s["scale"].to(wide)) + s["shift"].to(wide)
    if s["out"] == "i8":
        values, scale = plain_codes(a)
        return {"h": h, "values": values, "scale": scale}
    return {"h": h, "a": a.to(s["act"].dtype)}


# -------------------------------------------------------------------------------------- the library's calls
def own_quant(s):
    from paper_2607_04461_amd import flashbon as fb
    code = fb.BF16 if s["dtype"] == "bf16" else fb.FP32
    fb.flashbon_op_quant_rows(code, s["m"], s["k"], s["x"], s["q"], s["scale"])
    return {"values": s["q"] * s["scale"][:, None], "scale": s["scale"]}


def own_linear(s):
    from paper_2607_04461_amd import flashbon as fb
    code = fb.BF16 if s["dtype"] == "bf16" else fb.FP32
    epi = {"store": fb.EPI_STORE, "gelu": fb.EPI_GELU, "store_f32": fb.EPI_STORE_F32, "residual": fb.EPI_RESIDUAL}[s["epilogue"]]
    fb.flashbon_op_linear_i8(code, s["m"], s["n"], s["k"], s["a"], s["sa"], s["w"], s["sw"], s["bias"], epi, s["y"],
                             gate=s["gate"], residual_in=s["h"], cache_out=s["cache"])
    return {"h": s["y"], "cache": s["cache"]} if s["epilogue"] == "residual" else {"y": s["y"]}


def own_seam(s):
    from paper_2607_04461_amd import flashbon as fb
    code = fb.BF16 if s["dtype"] == "bf16" else fb.FP32
    kinds = {"none": fb.NORM_NONE, "layer": fb.NORM_LAYER, "rms": fb.NORM_RMS}
    i8 = s["out"] == "i8"
    fb.flashbon_op_norm_residual(code, s["m"], s["d"], EPS, s["x"], s["branch"], alpha=s["alpha"],
                                 post_norm=kinds[s["post"]], post_gain=s["gain"], gate=s["gate"], x_out=s["h"],
                                 pre_norm=kinds[s["pre"]], shift=s["shift"], scale=s["scale"],
                                 out=None if i8 else s["act"], q=s["q"] if i8 else None, q_scale=s["qs"] if i8 else None)
    if i8:
        return {"h": s["h"], "values": s["q"] * s["qs"][:, None], "scale": s["qs"]}
    return {"h": s["h"], "a": s["act"]}


def run(state):
    if own:
        return {"quant": own_quant, "linear": own_linear, "norm": own_seam}[state["kind"]](state)
    return {"quant": plain_quant, "linear": plain_linear, "norm": plain_seam}[state["kind"]](state)


# ---------------------------------------------------------------------------------------------- the work
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    m = case["m"]
    if case["kind"] == "quant":     # activations in, the values (fp32) and scales out
        return {"bytes": m * case["k"] * (e + 4) + 4 * m, "flops": 3 * m * case["k"]}
    if case["kind"] == "linear":
        n, k = case["n"], case["k"]
        out = {"store": e, "gelu": e, "store_f32": 4, "residual": 12}[case["epilogue"]]
        return {"bytes": m * k + n * k + 4 * (m + 3 * n) + m * n * out, "flops": 2 * m * n * k}
    out = 4 if case["out"] == "i8" else e
    return {"bytes": m * case["d"] * (4 + e + 4 + out) + 16 * case["d"] + 4 * m, "flops": 20 * m * case["d"]}


# ------------------------------------------------------------------- the definitions, in 64 bits throughout
def exact_codes(v):
    top = torch.maximum(v.max(1).values, -v.min(1).values)
    scale = torch.maximum(top / 127, torch.full_like(top, TINY)).to(torch.float32).to(torch.float64)
    ratio = v / scale.unsqueeze(1)
    low = torch.floor(ratio)
    up = ratio - low
    q = torch.where((up > 0.5) | ((up == 0.5) & (torch.remainder(low, 2) == 1)), low + 1, low)
    return q.mul_(scale.unsqueeze(1)), scale


def exact_rows(v, kind):
    if kind == "none":
        return v
    var, mean = torch.var_mean(v, 1, unbiased=False, keepdim=True)
    if kind == "layer":
        return (v - mean) / torch.sqrt(var + EPS)
    return v / torch.sqrt(var + mean ** 2 + EPS)


def exact(case, seed):
    s = prepare(case, seed)
    f64 = lambda name: s[name].to(torch.float64)  # noqa: E731
    if case["kind"] == "quant":
        values, scale = exact_codes(f64("x"))
        return {"values": values, "scale": scale}
    if case["kind"] == "linear":
        parts = []                              # blocks of rows: whole numbers, exact in 64 bits
        weight = f64("w").t().contiguous()
        for rows in f64("a").split(4096):
            parts.append(rows @ weight)
        v = torch.cat(parts).mul_(f64("sa").unsqueeze(1)).mul_(f64("sw")).add_(f64("bias"))
        if case["epilogue"] == "residual":
            h = torch.addcmul(f64("h"), f64("gate").expand_as(v), v)
            return {"h": h, "cache": h}
        if case["epilogue"] == "gelu":          # x sigmoid(2 u) = x (1 + tanh u) / 2
            v = v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
        return {"y": v}
    h = s["alpha"] * f64("x") + f64("gate") * (exact_rows(f64("branch"), case["post"]) * f64("gain"))
    # the next norm reads the stream as it is stored, in fp32
    a = exact_rows(h.to(torch.float32).to(torch.float64), case["pre"])
    a = a + a * f64("scale") + f64("shift")
    if case["out"] == "i8":
        values, scale = exact_codes(a)
        return {"h": h, "values": values, "scale": scale}
    return {"h": h, "a": a}
