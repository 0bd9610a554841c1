"""The operators of one mixture-of-experts sublayer, as cases to be measured.

A decode step of a model whose experts this library keeps compressed runs, after attention, three operators around the
decoder: the residual's addition with the root-mean-square norm (zipmoe_add_rmsnorm, bf16 rows or 8-bit rows with
scales), the router (zipmoe_route: projection, softmax, top-k) and the routed SwiGLU experts on weights that are already
recovered and resident in device memory (zipmoe_expert_ffn).  Every case is one call of one of them.

`own` false: elementary torch operations in 32 bits.  `own` true: the calls that a program makes of the library."""
import math

import torch

own = False

E4M3_MAX = 448.0


def listed():
    return [
        # one new token of one request in the 2048-wide model: latency alone counts
        {"name": "norm_token", "op": "norm", "rows": 1, "cols": 2048, "pitch": 2048, "residual": "bf16", "quant": 0},
        # a decode batch whose normed rows go to an 8-bit projection, one scale per row
        {"name": "norm_batch_8bit", "op": "norm", "rows": 64, "cols": 4096, "pitch": 4096, "residual": "bf16", "quant": 4096},
        # a long prompt through the 4096-wide model: pure bandwidth
        {"name": "norm_prompt", "op": "norm", "rows": 8192, "cols": 4096, "pitch": 4096, "residual": "bf16", "quant": 0},
        # rows that are slices of a wider buffer, fp32 residual stream, scales of 128 columns, odd number of rows
        {"name": "norm_odd_8bit", "op": "norm", "rows": 1531, "cols": 1408, "pitch": 2816, "residual": "f32", "quant": 128},
        # one token's router over 64 experts
        {"name": "route_token", "op": "route", "tokens": 1, "hidden": 2048, "experts": 64, "k": 6, "masked": 0},
        # a batch of odd size over 60 experts of which three are switched off by the bias
        {"name": "route_odd", "op": "route", "tokens": 777, "hidden": 2048, "experts": 60, "k": 4, "masked": 3},
        # a long prompt
        {"name": "route_prompt", "op": "route", "tokens": 8192, "hidden": 2048, "experts": 64, "k": 6, "masked": 0},
        # one token through six of 64 small experts: the smallest useful call of the expert layer
        {"name": "experts_token", "op": "experts", "tokens": 1, "hidden": 2048, "inter": 1408, "experts": 64, "active": 6, "k": 6},
        # one token through two of eight large experts
        {"name": "experts_large_token", "op": "experts", "tokens": 1, "hidden": 4096, "inter": 14336, "experts": 8, "active": 2, "k": 2},
        # an odd batch over most of 60 small experts whose intermediate size fills no whole tile
        {"name": "experts_odd", "op": "experts", "tokens": 37, "hidden": 2048, "inter": 1416, "experts": 60, "active": 55, "k": 4},
        # a decode batch over all eight large experts
        {"name": "experts_batch", "op": "experts", "tokens": 64, "hidden": 4096, "inter": 14336, "experts": 8, "active": 8, "k": 2},
        # the largest batch that one call takes
        {"name": "experts_large_batch", "op": "experts", "tokens": 256, "hidden": 4096, "inter": 14336, "experts": 8, "active": 8, "k": 2},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "route", "experts"])
    if op == "norm":
        cols = rng.choice([_log(rng, 64, 14336), 8 * _log(rng, 8, 1792), rng.choice([1408, 2048, 4096, 14336])])
        rows = _log(rng, 1, min(8192, 8192 * 4096 // cols))
        pitch = cols + rng.choice([0, 0, 8, rng.randint(1, 64)])
        return {"op": op, "rows": rows, "cols": cols, "pitch": pitch, "residual": rng.choice(["bf16", "f32", "none"]),
                "quant": rng.choice([0, 0, cols, 128])}
    if op == "route":
        experts = rng.choice([8, 16, 60, 64, 128, 256, rng.randint(4, 256)])
        hidden = 8 * _log(rng, 32, 512)
        return {"op": op, "tokens": _log(rng, 1, 8192), "hidden": hidden, "experts": experts,
                "k": rng.randint(1, min(8, experts // 2)), "masked": rng.choice([0, 0, rng.randint(1, experts // 2)])}
    tokens = _log(rng, 1, 256)
    experts = _log(rng, 4, 64)
    hidden = 8 * _log(rng, 64, 512)
    inter = 8 * _log(rng, 64, min(1792, 8 * 4096 * 14336 // (8 * experts * hidden)))
    k = rng.randint(1, min(8, experts))
    active = rng.randint(k, min(experts, tokens * k))
    return {"op": op, "tokens": tokens, "hidden": hidden, "inter": inter, "experts": experts, "active": active, "k": k}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _norm_inputs(c, seed):
    g = _generator(seed)
    shape = (c["rows"], c["pitch"])
    x = torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)[:, :c["cols"]]
    residual = None
    if c["residual"] != "none":
        # the residual stream: a few channels are far larger than the others
        residual = torch.randn(shape, generator=g, device="cuda") * 3
        residual[:, :: 97] *= 20
        residual = residual[:, :c["cols"]] if c["residual"] == "f32" else residual.to(torch.bfloat16)[:, :c["cols"]]
    weight = (1 + 0.2 * torch.randn(c["cols"], generator=g, device="cuda")).to(torch.bfloat16)
    return x, residual, weight


def _route_inputs(c, seed):
    # Activations in steps of 1/16, gate weights in steps of 2^-10 and a bias in steps of 2^-14: every product and every
    # partial sum is a whole number of steps below 2^24, so the logits do not depend on the order of the sums, and the
    # chosen experts can be compared as whole numbers.
    g = _generator(seed)
    x = (torch.randn(c["tokens"], c["hidden"], generator=g, device="cuda").clamp(-5, 5) * 16).round() / 16
    gate = (torch.randn(c["experts"], c["hidden"], generator=g, device="cuda").clamp(-5, 5) * 20).round() / 1024
    bias = (torch.randn(c["experts"], generator=g, device="cuda") * 0.1 * 16384).round() / 16384
    if c["masked"]:
        off = torch.randperm(c["experts"], generator=g, device="cuda")[:c["masked"]]
        bias[off] = -math.inf
    return x.to(torch.bfloat16), gate.to(torch.bfloat16), bias


def _expert_inputs(c, seed):
    g = _generator(seed)
    T, H, I, E, A, k = (c[n] for n in ("tokens", "hidden", "inter", "experts", "active", "k"))
    x = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)

    def weights(rows, cols):
        # N(0, s) with one input channel in a thousand at twenty times that, as large models' matrices have
        gain = torch.full((cols,), 0.8 / math.sqrt(cols), device="cuda")
        gain[torch.randperm(cols, generator=g, device="cuda")[:max(1, cols // 1000)]] *= 20
        return torch.stack([(torch.randn(rows, cols, generator=g, device="cuda") * gain).to(torch.bfloat16) for _ in range(E)])

    w1, w3, w2 = weights(I, H), weights(I, H), weights(H, I)
    # exactly `active` experts have tokens: the first tokens take each of them in turn, the others draw k of them without
    # replacement, popularity falling as 1 / rank^1.2
    experts = torch.randperm(E, generator=g, device="cuda")[:A]
    gumbel = -torch.log(-torch.log(torch.rand(T, A, generator=g, device="cuda").clamp(1e-6, 1 - 1e-6)))
    picks = (gumbel - 1.2 * torch.log(torch.arange(1, A + 1, device="cuda"))).topk(k, dim=1).indices
    first = min(T, -(-A // k))
    picks[:first] = (torch.arange(first * k, device="cuda") % A).view(first, k)
    ids = experts[picks].to(torch.int32)
    wts = torch.softmax(torch.randn(T, k, generator=g, device="cuda"), dim=1)
    return x, w1, w3, w2, ids, wts


def prepare(case, seed):
    s = {"case": case}
    if case["op"] == "norm":
        s["x"], s["residual"], s["weight"] = _norm_inputs(case, seed)
        if own:
            from paper_2601_21198_b200 import binding as zb
            s["norm"] = zb.RmsNorm(s["weight"], 1e-6)
            rows, cols, q = case["rows"], case["cols"], case["quant"]
            s["residual_out"] = None if s["residual"] is None else torch.empty(rows, cols, dtype=s["residual"].dtype, device="cuda")
            if q:
                s["out_q"] = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device="cuda")
                s["scales"] = torch.empty(rows, -(-cols // q), device="cuda")
            else:
                s["out"] = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    elif case["op"] == "route":
        s["x"], s["gate"], s["bias"] = _route_inputs(case, seed)
        if own:
            from paper_2601_21198_b200 import binding as zb
            s["router"] = zb.Router(s["gate"], case["k"], bias=s["bias"])
            s["ids"] = torch.empty(case["tokens"], case["k"], dtype=torch.int32, device="cuda")
            s["weights"] = torch.empty(case["tokens"], case["k"], device="cuda")
            s["logits"] = torch.empty(case["tokens"], case["experts"], device="cuda")
    else:
        s["x"], s["w1"], s["w3"], s["w2"], s["ids"], s["weights"] = _expert_inputs(case, seed)
        if own:
            from paper_2601_21198_b200 import binding as zb
            tensors = [w[e] for e in range(case["experts"]) for w in (s["w1"], s["w3"], s["w2"])]
            s["experts"] = zb.ResidentExperts(tensors, case["hidden"], case["inter"])
            s["out"] = torch.empty_like(s["x"])
    return s


def run(s):
    case = s["case"]
    if case["op"] == "norm":
        return _run_norm(s, case["quant"])
    if case["op"] == "route":
        return _run_route(s, case["k"])
    return _run_experts(s)


def _run_norm(s, quant):
    if own:
        if quant:
            s["norm"].add_norm_8bit(s["x"], s["residual"], s["residual_out"], s["out_q"], s["scales"], group=quant)
            out = {"q": s["out_q"], "scales": s["scales"]}
        else:
            s["norm"].add_norm(s["x"], s["residual"], s["residual_out"], s["out"])
            out = {"out": s["out"]}
        if s["residual"] is not None:
            out["residual"] = s["residual_out"]
        return out
    h = s["x"].float()
    out = {}
    if s["residual"] is not None:
        h = h + s["residual"].float()
        out["residual"] = h.to(s["residual"].dtype)
    y = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + 1e-6) * s["weight"].float()
    if not quant:
        out["out"] = y.to(torch.bfloat16)
        return out
    rows, cols = y.shape
    groups = -(-cols // quant)
    y = torch.nn.functional.pad(y, (0, groups * quant - cols)).view(rows, groups, quant)
    scales = y.abs().amax(dim=2) / E4M3_MAX
    q = y / torch.where(scales > 0, scales, 1).unsqueeze(2)
    out["q"] = q.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(rows, groups * quant)[:, :cols]
    out["scales"] = scales
    return out


def _run_route(s, k):
    if own:
        s["router"].route(s["x"], s["ids"], s["weights"], s["logits"])
        return {"ids": s["ids"], "weights": s["weights"], "logits": s["logits"]}
    logits = s["x"].float() @ s["gate"].float().t() + s["bias"]
    value, order = torch.sort(logits, dim=1, descending=True, stable=True)   # ties: the lowest index first
    value, ids = value[:, :k], order[:, :k].to(torch.int32)
    there = value > -math.inf
    p = torch.exp(value - value[:, :1]) * there
    return {"ids": torch.where(there, ids, -1), "weights": p / p.sum(dim=1, keepdim=True), "logits": logits}


def _run_experts(s):
    if own:
        return s["experts"].ffn(s["x"], s["ids"], s["weights"], s["out"])
    active = torch.unique(s["ids"]).long()
    x = s["x"].float()
    g = x @ s["w1"][active].float().transpose(1, 2)          # [A, T, I]
    h = g / (1 + torch.exp(-g)) * (x @ s["w3"][active].float().transpose(1, 2))
    y = h @ s["w2"][active].float().transpose(1, 2)          # [A, T, H]
    share = ((s["ids"].long().unsqueeze(0) == active.view(-1, 1, 1)) * s["weights"]).sum(dim=2)   # [A, T]
    return (share.unsqueeze(2) * y).sum(dim=0).to(torch.bfloat16)


def work(c):
    if c["op"] == "norm":
        n, rows = c["rows"] * c["cols"], c["rows"]
        residual = {"bf16": 4, "f32": 8, "none": 0}[c["residual"]]
        out = n + 4 * rows * -(-c["cols"] // c["quant"]) if c["quant"] else 2 * n
        return {"bytes": 2 * n + residual * n + 2 * c["cols"] + out, "flops": 6 * n}
    if c["op"] == "route":
        T, H, E, k = c["tokens"], c["hidden"], c["experts"], c["k"]
        return {"bytes": 2 * (T + E) * H + 4 * E + 8 * T * k + 4 * T * E, "flops": 2 * T * H * E}
    T, H, I, k = c["tokens"], c["hidden"], c["inter"], c["k"]
    return {"bytes": c["active"] * 3 * H * I * 2 + 4 * T * H + 8 * T * k, "flops": 6 * T * k * H * I}


def exact(case, seed):
    """What run() returns, from the formulas in 64 bits."""
    if case["op"] == "norm":
        x, residual, weight = _norm_inputs(case, seed)
        rows, cols, group = case["rows"], case["cols"], case["quant"]
        out = {}
        h = x.double()
        if residual is not None:
            h = h.add(residual.double())
            out["residual"] = h
        rms = torch.sqrt(torch.einsum("rc,rc->r", h, h) / cols + 1e-6)
        y = h / rms[:, None] * weight.double()
        if group:
            scales = torch.stack([part.abs().max(dim=1).values for part in torch.split(y, group, dim=1)], dim=1) / E4M3_MAX
            out["q"] = None          # a value of eight bits: no real number is it
            out["scales"] = scales
        else:
            out["out"] = y
        return out
    if case["op"] == "route":
        x, gate, bias = _route_inputs(case, seed)
        k = case["k"]
        logits = torch.einsum("th,eh->te", x.double(), gate.double()) + bias.double()
        best = torch.topk(logits, k, dim=1).values
        return {"ids": None, "weights": torch.softmax(best, dim=1), "logits": logits}
    x, w1, w3, w2, ids, wts = _expert_inputs(case, seed)
    y = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if t.numel() == 0:
            continue
        xe = x[t].double()
        h = torch.nn.functional.silu(xe @ w1[e].double().t()) * (xe @ w3[e].double().t())
        y.index_add_(0, t, wts[t, j].double()[:, None] * (h @ w2[e].double().t()))
    return y
