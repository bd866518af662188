"""Performance cases of the cross-attention branch with a prompt and an adapter per candidate, and of its gradients.

Three operators, each with its gradient, at the layer shapes of the networks the library runs (the 1.3B- and
14B-shaped transformers and the small ones of the tests) and at generic ragged ones:

* *norm*: LayerNorm of the residual stream, affine or modulated by a vector pair for each group of rows (a candidate's
  tokens at its own timestep), with the rows' statistics; the gradient adds the residual stream's own;
* *cross*: attention of image tokens to encoder states of another length, each candidate to its prompt, each prompt of
  its own length, key heads shared by groups of query heads; with the log-sum-exp that the gradient starts from;
* *adapters*: low-rank adapters beside a shared projection, one per candidate or none, added to the projection's output.

Gradients take what the forward call left (statistics, output and log-sum-exp, the inner product u) as inputs.
"""
import math

import torch

own = False

EPS = 1e-6
ACT = {"bf16": torch.bfloat16, "fp32": torch.float32}
# (hidden, MLP width, heads) of the networks
NETS = {"tiny": (64, 256, 4), "mid": (256, 704, 2), "wan1.3b": (1536, 8960, 12), "wan14b": (5120, 13824, 40)}


def listed():
    return [
        # the smallest call: one token before a projection, all launch latency
        norm_case("norm one token bf16", "bf16", 1, 1536, 1, True, False),
        # residual stream of a 14B-shaped pool of 4, each candidate at a timestep of its own
        norm_case("norm 14b pool4 bf16", "bf16", 16384, 5120, 4096, True, False),
        # training step over 16 candidates: rows' gradients and the modulations' of every candidate
        norm_case("norm grad pool16 bf16", "bf16", 24960, 1536, 1560, True, True),
        # odd sizes on every axis, one affine weight for all rows
        norm_case("norm grad odd fp32", "fp32", 1037, 701, 1037, False, True),
        # one query to long encoder states: few rows, all of K and V to read
        cross_case("cross one query bf16", "bf16", 1, 40, 40, 128, 1, 4096, 1, 4001, False),
        # the draft pool with four prompts of different lengths
        cross_case("cross pool16 bf16", "bf16", 16, 12, 12, 128, 1560, 512, 4, 77, False),
        # odd sizes, four query heads to a key head, one prompt empty
        cross_case("cross grad odd fp32", "fp32", 3, 8, 2, 64, 389, 77, 2, 0, True),
        # training step of a 14B-shaped pool of 4, two prompts
        cross_case("cross grad 14b pool4 bf16", "bf16", 4, 40, 40, 128, 4096, 512, 2, 300, True),
        # one token of each of 64 requests, 16 adapters and none
        adapters_case("adapters one token each bf16", "bf16", 64, 1536, 1536, 32, 1, 16, True, "store", False),
        # query projection of the draft pool, four adapters and none
        adapters_case("adapters pool16 bf16", "bf16", 24960, 1536, 1536, 32, 1560, 4, True, "store", False),
        # training step of one adapter over 16 candidates
        adapters_case("adapters grad pool16 bf16", "bf16", 24960, 1536, 1536, 32, 1560, 1, False, "store", True),
        # odd numbers of rows, three small adapters, gradient rows added in fp32
        adapters_case("adapters grad odd fp32", "fp32", 389, 712, 264, 8, 37, 3, True, "f32", True),
    ]


def norm_case(name, dtype, m, d, per, modulated, grad):
    """per: rows that share a weight and a bias."""
    return {"name": name, "kind": "norm", "dtype": dtype, "m": m, "d": d, "per": per, "modulated": modulated, "grad": grad}


def cross_case(name, dtype, batch, heads, kv_heads, dh, tq, tk, prompts, shortest, grad):
    """Prompt lengths run from tk down to shortest."""
    return {"name": name, "kind": "cross", "dtype": dtype, "batch": batch, "heads": heads, "kv_heads": kv_heads, "dh": dh,
            "tq": tq, "tk": tk, "prompts": prompts, "shortest": shortest, "grad": grad}


def adapters_case(name, dtype, m, n, k, rank, per, count, none, out, grad):
    """per: rows of a request; none: whether some requests have no adapter; out: "store" (the act type) or "f32"."""
    return {"name": name, "kind": "adapters", "dtype": dtype, "m": m, "n": n, "k": k, "rank": rank, "per": per,
            "count": count, "none": none, "out": out, "grad": grad}


def lengths(case):
    c = case["prompts"]
    return [case["tk"] - (case["tk"] - case["shortest"]) * i // max(1, c - 1) if c > 1 else case["shortest"] for i in range(c)]


def prompt_of(case):
    return [b * case["prompts"] // case["batch"] for b in range(case["batch"])]


def adapter_of(case):
    groups, kinds = -(-case["m"] // case["per"]), case["count"] + (1 if case["none"] else 0)
    return [g % kinds if g % kinds < case["count"] else -1 for g in range(groups)]


def adapted_rows(case):
    per, m = case["per"], case["m"]
    return sum(min(per, m - g * per) for g, a in enumerate(adapter_of(case)) if a >= 0)


# ------------------------------------------------------------------------------------------ drawn cases
def log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


MOST_VALUES = 8e7                      # of a norm, below the largest listed one
MOST_FLOPS = {"bf16": 4.2e11, "fp32": 2.6e10}


def draw(rng):
    while True:
        kind = rng.choices(["norm", "cross", "adapters"], [2, 3, 3])[0]
        dtype = rng.choices(["bf16", "fp32"], [3, 1])[0]
        grad = rng.random() < 0.5
        d, f, heads = NETS[rng.choices(list(NETS), [1, 2, 3, 2])[0]]
        if kind == "norm":
            m = log_int(rng, 1, 26000)
            width = rng.choice([d, log_int(rng, 1, 6144)])
            case = norm_case("", dtype, m, width, rng.choice([m, log_int(rng, 1, m)]), rng.random() < 0.6, grad)
            fits = m * width <= MOST_VALUES
        elif kind == "cross":
            dh = d // heads
            if rng.random() < 0.4:             # generic heads
                dh, heads = rng.choice([8, 16, 32, 64, 128]), rng.choice([1, 2, 3, 6, 8, 12, 16, 24])
            shared = rng.choice([s for s in (1, 1, 2, 3, 4, 8) if heads % s == 0])
            tk = log_int(rng, 1, 4096 if rng.random() < 0.3 else 512)
            batch = log_int(rng, 1, 16)
            prompts = rng.randint(1, min(4, batch))
            case = cross_case("", dtype, batch, heads, heads // shared, dh, log_int(rng, 1, 4096), tk, prompts,
                              rng.randint(0, tk), grad)
            fits = work(case)["flops"] <= MOST_FLOPS[dtype]
            fits = fits and batch * heads * case["tq"] * tk <= 4e8 and case["shortest"] + (prompts > 1) > 0
        else:
            n, k = rng.choice([(d, d), (f, d), (d, f)])
            if rng.random() < 0.35:            # generic sizes
                n, k = 8 * log_int(rng, 1, 1200), 8 * log_int(rng, 1, 1200)
            m = log_int(rng, 1, 26000)
            # single tokens, or candidates
            per = 1 if m <= 256 and rng.random() < 0.5 else log_int(rng, max(1, m // 16), m)
            case = adapters_case("", dtype, m, n, k, rng.choice([8, 16, 32, 64, 128]), per, rng.randint(1, 16),
                                 rng.random() < 0.5, rng.choice(["store", "f32"]), grad)
            fits = m * (n + k) <= MOST_VALUES and work(case)["flops"] <= MOST_FLOPS[dtype] / 8
        if fits:
            case.pop("name")
            return case


# -------------------------------------------------------------------------------------------- inputs
def normal(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device="cuda") * std


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"norm": prepare_norm, "cross": prepare_cross, "adapters": prepare_adapters}[case["kind"]](case, gen)


def prepare_norm(case, gen):
    s, m, d, act = dict(case), case["m"], case["d"], ACT[case["dtype"]]
    groups = -(-m // case["per"])
    s["x"] = normal(gen, m, d) * torch.exp(normal(gen, m, 1, std=0.3)) + normal(gen, d, std=0.5)
    s["weight"] = normal(gen, groups, d, std=0.3) + (0.0 if case["modulated"] else 1.0)
    s["bias"] = normal(gen, groups, d, std=0.3)
    s["mean"], s["rstd"] = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    if case["grad"]:
        wide = s["x"].double()
        var, mean = torch.var_mean(wide, 1, unbiased=False)
        s["mean"].copy_(mean)
        s["rstd"].copy_(torch.rsqrt(var + EPS))
        s["dy"] = normal(gen, m, d).to(act)
        s["res"] = normal(gen, m, d)
        s["dx"] = torch.empty(m, d, device="cuda")
        s["dweight"], s["dbias"] = torch.empty(groups, d, device="cuda"), torch.empty(groups, d, device="cuda")
        s["ws"] = torch.empty(0, dtype=torch.uint8, device="cuda")
    else:
        s["y"] = torch.empty(m, d, dtype=act, device="cuda")
    return s


def prepare_cross(case, gen):
    s, act, dh = dict(case), ACT[case["dtype"]], case["dh"]
    b, tq, tk, c = case["batch"], case["tq"], case["tk"], case["prompts"]
    wide, narrow = case["heads"] * dh, case["kv_heads"] * dh
    # normalised queries and keys: scores of a spread around one
    s["q"] = normal(gen, b, tq, wide).to(act)
    s["kv"] = normal(gen, c, tk, 2 * narrow).to(act)          # keys, then values, in each row
    s["len"], s["index"] = ints(lengths(case)), ints(prompt_of(case))
    s["out"] = torch.empty(b, tq, wide, dtype=act, device="cuda")
    s["lse"] = torch.empty(b, case["heads"], tq, device="cuda")
    s["ws"] = torch.empty(0, dtype=torch.uint8, device="cuda")
    if case["grad"]:
        forward = plain_cross(s)
        s["out"], s["lse"] = forward["out"], forward["lse"]
        s["dout"] = normal(gen, b, tq, wide).to(act)
        s["dq"], s["dkv"] = torch.empty_like(s["q"]), torch.empty_like(s["kv"])
    return s


def prepare_adapters(case, gen):
    s, act = dict(case), ACT[case["dtype"]]
    m, n, k, r, a = case["m"], case["n"], case["k"], case["rank"], case["count"]
    store = act if case["out"] == "store" else torch.float32
    s["down"] = normal(gen, a, r, k, std=k ** -0.5).to(act)
    s["up"] = normal(gen, a, n, r, std=0.3 * r ** -0.5).to(act)
    s["scales"] = torch.exp(normal(gen, a, std=0.3))
    s["index"] = ints(adapter_of(case))
    s["x"] = normal(gen, m, k).to(act)
    s["u"] = torch.empty(m, r, device="cuda")
    if case["grad"]:
        s["dy"] = normal(gen, m, n).to(act)
        s["u"] = plain_adapters(s)["u"]
        s["base"], s["dx"] = normal(gen, m, k).to(store), torch.empty(m, k, dtype=store, device="cuda")
        s["ddown"], s["dup"] = torch.empty(a, r, k, device="cuda"), torch.empty(a, n, r, device="cuda")
        s["ws"] = torch.empty(0, dtype=torch.uint8, device="cuda")
    else:
        s["base"], s["y"] = normal(gen, m, n).to(store), torch.empty(m, n, dtype=store, device="cuda")
    return s


# ------------------------------------------------------------------------------------------ plain forms
def rows_of(v, s):
    """A vector for each group of rows to one for each row."""
    return v.repeat_interleave(s["per"], 0)[:s["m"]]


def plain_norm(s):
    x = s["x"]
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
    factor = s["weight"] + 1 if s["modulated"] else s["weight"]
    y = c * rstd * rows_of(factor, s) + rows_of(s["bias"], s)
    return {"y": y.to(s["y"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}


def plain_norm_grad(s):
    m, per = s["m"], s["per"]
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xhat = (s["x"] - s["mean"][:, None]) * rstd
    g = dy * rows_of(s["weight"] + 1 if s["modulated"] else s["weight"], s)
    dx = s["res"] + rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    short = -m % per                                          # rows missing from the last group
    grouped = lambda v: torch.cat([v, v.new_zeros(short, s["d"])]).view(-1, per, s["d"]).sum(1)  # noqa: E731
    return {"dx": dx, "dweight": grouped(dy * xhat), "dbias": grouped(dy)}


def split_heads(x, dh):
    """[b][t][h dh] to [b][h][t][dh] in 32 bits."""
    return x.float().view(x.shape[0], x.shape[1], -1, dh).transpose(1, 2).contiguous()


def join_heads(x):
    return x.transpose(1, 2).flatten(2)


def keys_values(s):
    """Keys and values of each candidate and query head, zero past the prompt's end, and which of them count."""
    dh, shared, index = s["dh"], s["heads"] // s["kv_heads"], s["index"].long()
    live = (torch.arange(s["tk"], device="cuda") < s["len"][:, None])
    k, v = s["kv"].masked_fill(~live[:, :, None], 0).chunk(2, 2)
    k, v = (split_heads(t, dh)[index].repeat_interleave(shared, 1) for t in (k, v))
    return k, v, live[index][:, None, None, :]


def plain_cross(s):
    k, v, live = keys_values(s)
    scores = (split_heads(s["q"], s["dh"]) @ k.transpose(2, 3).contiguous()) / math.sqrt(s["dh"])
    scores = scores.masked_fill(~live, -math.inf)
    top = scores.amax(3, keepdim=True).clamp_min(-3e38)
    p = torch.exp(scores - top)
    total = p.sum(3, keepdim=True)
    out = (p @ v) / torch.where(total > 0, total, 1.0)
    return {"out": join_heads(out).to(s["q"].dtype), "lse": torch.where(total > 0, top + torch.log(total), -math.inf)[..., 0]}


def plain_cross_grad(s):
    dh, scale, act = s["dh"], 1 / math.sqrt(s["dh"]), s["q"].dtype
    k, v, live = keys_values(s)
    q, dout, out = (split_heads(s[name], dh) for name in ("q", "dout", "out"))
    scores = (q @ k.transpose(2, 3).contiguous()) * scale
    p = torch.where(live, torch.exp(scores - s["lse"][..., None]), 0.0)
    dp = dout @ v.transpose(2, 3).contiguous()
    ds = p * (dp - (dout * out).sum(3, keepdim=True)) * scale
    dq = ds @ k
    dk, dv = ds.transpose(2, 3).contiguous() @ q, p.transpose(2, 3).contiguous() @ dout
    # over the query heads of a key head, then over the candidates of a prompt
    chosen = (torch.arange(s["prompts"], device="cuda")[:, None] == s["index"]).float()
    dk, dv = (t.unflatten(1, (s["kv_heads"], -1)).sum(2) for t in (dk, dv))
    dk, dv = ((chosen @ t.flatten(1)).view(s["prompts"], *t.shape[1:]) for t in (dk, dv))
    return {"dq": join_heads(dq).to(act), "dkv": torch.cat([join_heads(dk), join_heads(dv)], 2).to(act)}


def requests(x, s):
    """Rows to [groups][per][width] in 32 bits, the last group filled up with zeros."""
    return torch.cat([x.float(), x.new_zeros(-s["m"] % s["per"], x.shape[1], dtype=torch.float32)]).view(-1, s["per"], x.shape[1])


def chosen_adapters(s):
    """down, up and scale of each request, zeros where it has none."""
    index, has = s["index"].long().clamp_min(0), (s["index"] >= 0).float()[:, None, None]
    return s["down"].float()[index] * has, s["up"].float()[index] * has, s["scales"][index][:, None, None]


def plain_adapters(s):
    down, up, scale = chosen_adapters(s)
    u = requests(s["x"], s) @ down.transpose(1, 2).contiguous()
    if "base" not in s:
        return {"u": u.flatten(0, 1)[:s["m"]].contiguous()}
    y = s["base"].float() + ((u @ up.transpose(1, 2).contiguous()) * scale).flatten(0, 1)[:s["m"]]
    return {"y": y.to(s["y"].dtype), "u": u.flatten(0, 1)[:s["m"]]}


def plain_adapters_grad(s):
    down, up, scale = chosen_adapters(s)
    dy, x, u = requests(s["dy"], s), requests(s["x"], s), requests(s["u"], s)
    du = (dy @ up) * scale
    dx = s["base"].float() + (du @ down).flatten(0, 1)[:s["m"]]
    ddown = du.transpose(1, 2).contiguous() @ x
    dup = (dy.transpose(1, 2).contiguous() @ u) * scale
    chosen = (torch.arange(s["count"], device="cuda")[:, None] == s["index"]).float()
    ddown, dup = ((chosen @ t.flatten(1)).view(s["count"], *t.shape[1:]) for t in (ddown, dup))
    return {"dx": dx.to(s["dx"].dtype), "ddown": ddown, "dup": dup}


# -------------------------------------------------------------------------------------- the library's calls
def workspace(s, need):
    """The program's workspace, made on the first pass and kept."""
    if s["ws"].numel() < need:
        s["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return s["ws"]


def own_norm(s):
    from paper_2607_04461_amd import flashbon as fb
    code = fb.BF16 if s["dtype"] == "bf16" else fb.FP32
    if s["grad"]:
        ws = workspace(s, fb.flashbon_op_layer_norm_grad_workspace(s["m"], s["d"], s["per"]))
        fb.flashbon_op_layer_norm_grad(code, s["m"], s["d"], s["x"], s["mean"], s["rstd"], s["dy"], s["dx"], weight=s["weight"],
                                       rows_per_group=s["per"], modulated=s["modulated"], residual=s["res"],
                                       dweight=s["dweight"], dbias=s["dbias"], workspace=ws)
        return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    fb.flashbon_op_layer_norm(code, s["m"], s["d"], EPS, s["x"], s["y"], weight=s["weight"], bias=s["bias"],
                              rows_per_group=s["per"], modulated=s["modulated"], mean=s["mean"], rstd=s["rstd"])
    return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}


def own_cross(s):
    from paper_2607_04461_amd import flashbon as fb
    code = fb.BF16 if s["dtype"] == "bf16" else fb.FP32
    sizes = (code, s["batch"], s["heads"], s["kv_heads"], s["dh"], s["tq"], s["tk"])
    wide, narrow = s["heads"] * s["dh"], s["kv_heads"] * s["dh"]
    q_strides, kv_strides = (s["tq"] * wide, wide), (s["tk"] * 2 * narrow, 2 * narrow)
    k, v = s["kv"][:, :, :narrow], s["kv"][:, :, narrow:]
    if s["grad"]:
        ws = workspace(s, fb.flashbon_op_cross_attention_grad_workspace(*sizes, s["prompts"]))
        fb.flashbon_op_cross_attention_grad(*sizes, s["q"], *q_strides, k, v, *kv_strides, s["index"], s["prompts"], s["len"],
                                            s["out"], *q_strides, s["lse"], s["dout"], s["dq"], s["dkv"][:, :, :narrow],
                                            s["dkv"][:, :, narrow:], workspace=ws)
        return {"dq": s["dq"], "dkv": s["dkv"]}
    ws = workspace(s, fb.flashbon_op_cross_attention_workspace(*sizes))
    fb.flashbon_op_cross_attention(*sizes, s["q"], *q_strides, k, v, *kv_strides, s["index"], s["prompts"], s["len"],
                                   s["out"], *q_strides, lse=s["lse"], workspace=ws)
    return {"out": s["out"], "lse": s["lse"]}


def own_adapters(s):
    from paper_2607_04461_amd import flashbon as fb
    code = fb.BF16 if s["dtype"] == "bf16" else fb.FP32
    epilogue = fb.EPI_STORE if s["out"] == "store" else fb.EPI_STORE_F32
    sizes = (code, s["m"], s["n"], s["k"], s["rank"], s["count"])
    if s["grad"]:
        ws = workspace(s, fb.flashbon_op_adapters_grad_workspace(*sizes, s["per"]))
        fb.flashbon_op_adapters_grad(*sizes, s["x"], s["down"], s["up"], s["scales"], s["index"], s["per"], s["u"], s["dy"],
                                     epilogue, s["base"], s["dx"], s["ddown"], s["dup"], workspace=ws)
        return {"dx": s["dx"], "ddown": s["ddown"], "dup": s["dup"]}
    fb.flashbon_op_adapters(*sizes, s["x"], s["down"], s["up"], s["scales"], s["index"], s["per"], epilogue, s["base"],
                            s["y"], s["u"])
    return {"y": s["y"], "u": s["u"]}


def run(state):
    if own:
        return {"norm": own_norm, "cross": own_cross, "adapters": own_adapters}[state["kind"]](state)
    plain = {"norm": plain_norm_grad, "cross": plain_cross_grad, "adapters": plain_adapters_grad} if state["grad"] else \
        {"norm": plain_norm, "cross": plain_cross, "adapters": plain_adapters}
    return plain[state["kind"]](state)


# ---------------------------------------------------------------------------------------------- the work
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "norm":
        m, d = case["m"], case["d"]
        vectors = 4 * d * -(-m // case["per"])
        if case["grad"]:       # x, dy, the stream's gradient in; dx out; weight in, its gradient and the bias's out
            return {"bytes": m * d * (4 + e + 4 + 4) + 3 * vectors + 8 * m, "flops": 15 * m * d}
        return {"bytes": m * d * (4 + e) + 2 * vectors + 8 * m, "flops": 8 * m * d}
    if case["kind"] == "cross":
        b, h, dh, tq = case["batch"], case["heads"], case["dh"], case["tq"]
        keys = lengths(case)
        pairs = h * tq * sum(keys[c] for c in prompt_of(case))
        rows, used = b * tq * h * dh * e, 2 * sum(keys) * case["kv_heads"] * dh * e
        if case["grad"]:       # q, out, dout in, dq out; keys and values in, their gradients out (whole buffers)
            whole = 2 * case["prompts"] * case["tk"] * case["kv_heads"] * dh * e
            return {"bytes": 4 * rows + used + whole + 4 * b * h * tq, "flops": 10 * pairs * dh}
        return {"bytes": 2 * rows + used + 4 * b * h * tq, "flops": 4 * pairs * dh}
    m, n, k, r = case["m"], case["n"], case["k"], case["rank"]
    o = e if case["out"] == "store" else 4
    rows, weights = adapted_rows(case), min(case["count"], len(adapter_of(case))) * r * (n + k)
    if case["grad"]:           # x, dy, u in for adapted rows; base in and dx out for all
        return {"bytes": rows * ((n + k) * e + 4 * r) + 2 * m * k * o + weights * (e + 4), "flops": 4 * rows * r * (n + k)}
    return {"bytes": rows * k * e + 2 * m * n * o + 4 * m * r + weights * e, "flops": 2 * rows * r * (n + k)}


# ------------------------------------------------------------------- the definitions, in 64 bits throughout
def exact(case, seed):
    s = prepare(case, seed)
    s.update({name: t.to(torch.float64) for name, t in s.items() if torch.is_tensor(t) and t.is_floating_point()})
    return {"norm": exact_norm, "cross": exact_cross, "adapters": exact_adapters}[case["kind"]](case, s)


def exact_norm(case, s):
    m, per, x = case["m"], case["per"], s["x"]
    group = torch.arange(m, device="cuda") // per
    weight = s["weight"][group]
    weight = weight + 1.0 if case["modulated"] else weight
    if not case["grad"]:
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = (var + EPS) ** -0.5
        y = torch.addcmul(s["bias"][group], (x - mean.unsqueeze(1)).mul_(rstd.unsqueeze(1)), weight)
        return {"y": y, "mean": mean, "rstd": rstd}
    dy, d, rstd = s["dy"], case["d"], s["rstd"].unsqueeze(1)
    xhat = (x - s["mean"].unsqueeze(1)).mul_(rstd)
    g = dy * weight
    along = torch.linalg.vecdot(g, xhat).unsqueeze(1)
    dx = s["res"] + (d * g - g.sum(1, keepdim=True) - xhat * along) * (rstd / d)
    zero = torch.zeros_like(s["weight"])
    return {"dx": dx, "dweight": zero.index_add(0, group, dy * xhat), "dbias": zero.index_add(0, group, dy)}


def exact_cross(case, s):
    dh, heads, kvh = case["dh"], case["heads"], case["kv_heads"]
    keys, narrow, shared = lengths(case), kvh * dh, heads // kvh
    grad = case["grad"]
    out, lse = torch.zeros_like(s["q"]), torch.full_like(s["lse"], -math.inf)
    dq, dkv = torch.zeros_like(s["q"]), torch.zeros_like(s["kv"])
    for b, c in enumerate(prompt_of(case)):
        n = keys[c]
        if n == 0:
            continue
        for h in range(heads):
            at, kat = slice(h * dh, h * dh + dh), slice(h // shared * dh, h // shared * dh + dh)
            vat = slice(narrow + kat.start, narrow + kat.stop)
            q, k, v = s["q"][b, :, at], s["kv"][c, :n, kat], s["kv"][c, :n, vat]
            scores = q.mm(k.t()).div_(dh ** 0.5)
            if not grad:
                lse[b, h] = torch.logsumexp(scores, 1)
                out[b, :, at] = torch.softmax(scores, 1).mm(v)
                continue
            p = scores.sub_(s["lse"][b, h].unsqueeze(1)).exp_()
            do = s["dout"][b, :, at]
            ds = p * (do.mm(v.t()) - torch.linalg.vecdot(do, s["out"][b, :, at]).unsqueeze(1)) / dh ** 0.5
            dq[b, :, at] = ds.mm(k)
            dkv[c, :n, kat] += ds.t().mm(q)
            dkv[c, :n, vat] += p.t().mm(do)
    return {"dq": dq, "dkv": dkv} if grad else {"out": out, "lse": lse}


def exact_adapters(case, s):
    row = torch.tensor(adapter_of(case), device="cuda")[torch.arange(case["m"], device="cuda") // case["per"]]
    grad = case["grad"]
    result = s["base"].clone()
    u = torch.zeros_like(s["u"])
    ddown, dup = torch.zeros_like(s["down"]), torch.zeros_like(s["up"])
    for a in range(case["count"]):
        at = torch.nonzero(row == a).flatten()
        down, up, scale, x = s["down"][a], s["up"][a], s["scales"][a], s["x"][at]
        if grad:
            dy = s["dy"][at]
            du = scale * dy.mm(up)
            result[at] += du.mm(down)
            ddown[a], dup[a] = du.t().mm(x), scale * dy.t().mm(s["u"][at])
        else:
            u[at] = x.mm(down.t())
            result[at] += scale * u[at].mm(up.t())
    return {"dx": result, "ddown": ddown, "dup": dup} if grad else {"y": result, "u": u}
