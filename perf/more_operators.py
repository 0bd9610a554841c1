"""The expert products of a prompt and products in 8-bit integers, as cases to be measured.

Beside a decode step (whose operators are measured elsewhere) a mixture-of-experts layer takes prompts: the tokens' choices
are grouped by expert (group_tokens), every expert's tokens go through W1 and W3 and the gated activation (GroupedMatrix of
pairs), the result goes through W2 and each token's choices are added with their weights (GroupedMatrix, combine_rows).  The
dense projections around the experts can run in 8-bit integers with a scale per token and per output channel (Int8Linear).
Every case is a pass through one of these four; the products of either kind begin with the choices' lists in both forms, since
a layer makes them anew for every prompt.

`own` false: elementary torch operations in 32 bits.  `own` true: the calls that a program makes of the library."""
import math

import torch

own = False


def listed():
    return [
        # the choices of a decode batch over eight experts: the smallest call, latency alone counts
        {"name": "group_batch", "op": "group", "tokens": 64, "k": 2, "experts": 8, "active": 8, "masked": 0},
        # the choices of a long prompt over 64 experts, some of them dropped (-1)
        {"name": "group_prompt", "op": "group", "tokens": 8192, "k": 6, "experts": 64, "active": 64, "masked": 500},
        # one new token through W1 and W3 of six of 64 small experts
        {"name": "gate_up_token", "op": "gate_up", "tokens": 1, "k": 6, "experts": 64, "active": 6, "masked": 0, "hidden": 2048, "inter": 1408},
        # a short prompt of odd length through 60 experts whose intermediate size fills no whole tile, some choices dropped
        {"name": "gate_up_odd", "op": "gate_up", "tokens": 777, "k": 4, "experts": 60, "active": 55, "masked": 101, "hidden": 2048, "inter": 1416},
        # a long prompt through 64 small experts
        {"name": "gate_up_prompt", "op": "gate_up", "tokens": 8192, "k": 6, "experts": 64, "active": 64, "masked": 0, "hidden": 2048, "inter": 1408},
        # a prompt through eight large experts: the most work of all cases
        {"name": "gate_up_large", "op": "gate_up", "tokens": 4096, "k": 2, "experts": 8, "active": 8, "masked": 0, "hidden": 4096, "inter": 14336},
        # one token's two choices through W2 of eight large experts, and their weighted sum
        {"name": "down_token", "op": "down", "tokens": 1, "k": 2, "experts": 8, "active": 2, "masked": 0, "hidden": 4096, "inter": 14336},
        # the second half of gate_up_odd
        {"name": "down_odd", "op": "down", "tokens": 777, "k": 4, "experts": 60, "active": 55, "masked": 101, "hidden": 2048, "inter": 1416},
        # the second half of gate_up_prompt
        {"name": "down_prompt", "op": "down", "tokens": 8192, "k": 6, "experts": 64, "active": 64, "masked": 0, "hidden": 2048, "inter": 1408},
        # one token through a dense projection in 8 bits: the weights' bytes
        {"name": "int8_token", "op": "int8", "tokens": 1, "cols": 4096, "rows": 14336},
        # an odd number of tokens through a projection of odd sizes
        {"name": "int8_odd", "op": "int8", "tokens": 1531, "cols": 1424, "rows": 2051},
        # a long prompt through a wide projection
        {"name": "int8_prompt", "op": "int8", "tokens": 8192, "cols": 4096, "rows": 14336},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["group", "gate_up", "down", "int8"])
    if op == "int8":
        cols, rows = 16 * _log(rng, 16, 896), _log(rng, 100, 14336)
        return {"op": op, "tokens": _log(rng, 1, min(8192, 8192 * 4096 * 14336 // (cols * rows))), "cols": cols, "rows": rows}
    experts = _log(rng, 4, 64)
    k = rng.randint(1, min(8, experts))
    tokens = _log(rng, 1, 49152 // k)
    c = {"op": op, "tokens": tokens, "k": k, "experts": experts, "active": rng.randint(k, min(experts, tokens * k))}
    if op != "group":
        c["hidden"] = 8 * _log(rng, 32, 512)
        c["inter"] = 8 * _log(rng, 32, min(1792, 4096 * 14336 * 8 // (8 * c["hidden"] * max(experts, 8))))
        # no more products than the largest listed case has
        c["tokens"] = tokens = max(-(-c["active"] // k), min(tokens, 8192 * 4096 * 14336 // (k * c["hidden"] * c["inter"])))
    spare = tokens * k - _first(c) * k
    c["masked"] = rng.choice([0, rng.randint(0, spare // 2)])
    return c


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _first(c):
    """How many tokens take the active experts in turn, so that each of them has one at least."""
    return min(c["tokens"], -(-c["active"] // c["k"]))


def _routing(c, g):
    """ids [T, k] int32: every token's choices are distinct; popularity falls with an expert's rank (the most popular of 64
    has about five times the mean); `masked` of the choices are dropped."""
    T, k, A = c["tokens"], c["k"], c["active"]
    experts = torch.randperm(c["experts"], generator=g, device="cuda")[:A]
    gumbel = -torch.log(-torch.log(torch.rand(T, A, generator=g, device="cuda").clamp(1e-6, 1 - 1e-6)))
    picks = (gumbel - 0.6 * torch.log(torch.arange(1, A + 1, device="cuda"))).topk(k, dim=1).indices
    first = _first(c)
    picks[:first] = (torch.arange(first * k, device="cuda") % A).view(first, k)
    ids = experts[picks].to(torch.int32)
    if c["masked"]:
        spare = torch.randperm(T * k - first * k, generator=g, device="cuda")[:c["masked"]] + first * k
        ids.view(-1)[spare] = -1
    return ids


def _matrices(g, E, rows, cols):
    """N(0, s) with one input channel in a thousand at twenty times that, as large models' matrices have."""
    gain = torch.full((cols,), 0.8 / math.sqrt(cols), device="cuda")
    gain[torch.randperm(cols, generator=g, device="cuda")[:max(1, cols // 1000)]] *= 20
    w = torch.empty(E, rows, cols, dtype=torch.bfloat16, device="cuda")
    for e in range(E):
        w[e] = torch.randn(rows, cols, generator=g, device="cuda") * gain
    return w


def _inputs(c, seed):
    g = _generator(seed)
    if c["op"] == "int8":
        x = torch.randn(c["tokens"], c["cols"], generator=g, device="cuda")
        x[:, ::97] *= 6       # activations have a few wide channels
        w = torch.randint(-127, 128, (c["rows"], c["cols"]), generator=g, device="cuda", dtype=torch.int8)
        scales = torch.rand(c["rows"], generator=g, device="cuda") * 2e-4 + 1e-4
        return {"x": x.to(torch.bfloat16), "w": w, "scales": scales}
    ids = _routing(c, g)
    if c["op"] == "group":
        return {"ids": ids}
    T, k, H, I, E = (c[n] for n in ("tokens", "k", "hidden", "inter", "experts"))
    if c["op"] == "gate_up":
        x = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
        return {"ids": ids, "x": x, "w1": _matrices(g, E, I, H), "w3": _matrices(g, E, I, H)}
    h = torch.randn(T * k, I, generator=g, device="cuda") * torch.rand(T * k, I, generator=g, device="cuda")
    weights = torch.softmax(torch.randn(T, k, generator=g, device="cuda"), dim=1)
    return {"ids": ids, "h": h.to(torch.bfloat16), "w2": _matrices(g, E, H, I), "weights": weights}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] != "int8":
        # the most tokens of an expert: what a padded batch of products is sized by
        s["most"] = int(torch.bincount(s["ids"][s["ids"] >= 0].long()).max())
    if own:
        from paper_2601_21198_b200 import binding as zb
        if case["op"] == "int8":
            s["linear"] = zb.Int8Linear(s["w"], s["scales"])
            s["out"] = torch.empty(case["tokens"], case["rows"], dtype=torch.bfloat16, device="cuda")
            return s
        T, k = case["tokens"], case["k"]
        if case["op"] == "group":
            s["offsets"] = torch.empty(case["experts"] + 1, dtype=torch.int32, device="cuda")
            s["order"] = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")   # (those behind the last group stay)
            s["place"] = torch.empty(T, k, dtype=torch.int32, device="cuda")
            return s
        if case["op"] == "gate_up":
            s["gate_up"] = zb.GroupedMatrix(list(s["w1"]), up=list(s["w3"]))
            s["h"] = torch.zeros(T * k, case["inter"], dtype=torch.bfloat16, device="cuda")   # (rows behind the last group stay)
        else:
            s["down"] = zb.GroupedMatrix(list(s["w2"]))
            s["y"] = torch.empty(T * k, case["hidden"], dtype=torch.float32, device="cuda")
            s["out"] = torch.empty(T, case["hidden"], dtype=torch.bfloat16, device="cuda")
    return s


def run(s):
    op = s["case"]["op"]
    if op == "int8":
        return s["linear"].product(s["x"], out=s["out"]) if own else _plain_int8(s["x"], s["w"], s["scales"])
    if op == "group":
        if not own:
            return _plain_group(s["ids"], s["case"]["experts"])
        from paper_2601_21198_b200 import binding as zb
        zb.group_tokens(s["ids"], s["case"]["experts"], offsets=s["offsets"], order=s["order"], place=s["place"])
        return {"offsets": s["offsets"], "order": s["order"], "place": s["place"]}
    if op == "gate_up":
        if own:
            from paper_2601_21198_b200 import binding as zb
            groups = zb.group_tokens(s["ids"], s["case"]["experts"])
            return s["gate_up"].product(s["x"], groups, gather=True, out=s["h"])
        return _plain_gate_up(s["x"], s["ids"], s["w1"], s["w3"], s["most"])
    if own:
        from paper_2601_21198_b200 import binding as zb
        groups = zb.group_tokens(s["ids"], s["case"]["experts"])
        s["down"].product(s["h"], groups, out=s["y"])
        return zb.combine_rows(s["y"], groups, s["weights"], out=s["out"])
    return _plain_down(s["h"], s["ids"], s["w2"], s["weights"], s["most"])


def _plain_int8(x, w, scales):
    x = x.float()
    top = x.abs().amax(dim=1, keepdim=True)
    q = torch.where(top > 0, (x * 127 / torch.where(top > 0, top, 1)).round(), 0)
    return ((q @ w.float().t()) * (top / 127) * scales).to(torch.bfloat16)


def _plain_group(ids, E):
    flat = ids.reshape(-1)
    there = flat >= 0
    order = torch.sort(torch.where(there, flat, E), stable=True).indices
    counts = (flat[:, None] == torch.arange(E, device=ids.device)).sum(dim=0)
    offsets = torch.nn.functional.pad(torch.cumsum(counts, 0), (1, 0))
    rank = torch.empty_like(order)
    rank[order] = torch.arange(order.numel(), device=ids.device)
    order = torch.where(torch.arange(order.numel(), device=ids.device) < offsets[-1], order, -1)
    return {"offsets": offsets.to(torch.int32), "order": order.to(torch.int32), "place": torch.where(there, rank, -1).to(torch.int32).view(ids.shape)}


def _padded(ids, most):
    """The active experts; for each of them `most` choices (some stand in for none); where each grouped row is among those, and
    which rows there are."""
    flat = ids.reshape(-1)
    active = torch.unique(flat[flat >= 0])
    counts = (flat[:, None] == active).sum(dim=0)
    begin = torch.cumsum(counts, 0) - counts
    order = torch.sort(torch.where(flat >= 0, flat, flat.max() + 1), stable=True).indices
    at = (begin[:, None] + torch.arange(most, device=ids.device)).clamp(max=flat.numel() - 1)
    row = torch.arange(flat.numel(), device=ids.device)
    group = ((row[:, None] >= begin).sum(dim=1) - 1).clamp(min=0)
    within = (row - begin[group]).clamp(max=most - 1)
    return active.long(), order, at, group, within, row < counts.sum()


def _plain_gate_up(x, ids, w1, w3, most):
    active, order, at, group, within, there = _padded(ids, most)
    xe = x[order[at] // ids.shape[1]].float()                      # [A, most, H]
    g = xe @ w1[active].float().transpose(1, 2)
    h = g / (1 + torch.exp(-g)) * (xe @ w3[active].float().transpose(1, 2))
    return (h[group, within] * there[:, None]).to(torch.bfloat16)


def _plain_down(h, ids, w2, weights, most):
    active, order, at, group, within, there = _padded(ids, most)
    y = h[at].float() @ w2[active].float().transpose(1, 2)         # [A, most, H]
    y = y[group, within]                                           # grouped rows
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=ids.device)
    share = weights * (ids >= 0)
    return (share.unsqueeze(2) * y[place].view(*ids.shape, -1)).sum(dim=1).to(torch.bfloat16)


def work(c):
    if c["op"] == "int8":
        T, K, N = c["tokens"], c["cols"], c["rows"]
        return {"bytes": 2 * T * K + N * K + 4 * N + 2 * T * N, "flops": 2 * T * K * N + 3 * T * K}
    T, k = c["tokens"], c["k"]
    if c["op"] == "group":
        return {"bytes": 12 * T * k + 4 * (c["experts"] + 1), "flops": 2 * T * k}
    rows, H, I = T * k - c["masked"], c["hidden"], c["inter"]
    if c["op"] == "gate_up":
        return {"bytes": c["active"] * 4 * H * I + 2 * T * H + 4 * T * k + 2 * rows * I, "flops": 4 * rows * H * I}
    return {"bytes": c["active"] * 2 * H * I + 2 * rows * I + 8 * T * k + 2 * T * H, "flops": 2 * rows * H * I + 2 * rows * H}


def exact(case, seed):
    """What run() returns, from the formulas in 64 bits, expert by expert."""
    s = _inputs(case, seed)
    if case["op"] == "group":
        return None           # whole numbers: nothing in them is rounded
    if case["op"] == "int8":
        x = s["x"].double()
        top = x.abs().max(dim=1).values
        q = torch.round(torch.nan_to_num(x * 127 / top[:, None]))      # (rows of zeros)
        total = torch.einsum("tk,nk->tn", q, s["w"].double())
        return total * torch.outer(top / 127, s["scales"].double())
    ids, k = s["ids"], case["k"]
    flat = ids.view(-1)
    if case["op"] == "gate_up":
        out = torch.zeros(flat.numel(), case["inter"], dtype=torch.float64, device="cuda")
    else:
        out = torch.zeros(case["tokens"], case["hidden"], dtype=torch.float64, device="cuda")
    begin = 0
    for e in range(case["experts"]):
        choice = torch.nonzero(flat == e)[:, 0]
        end = begin + choice.numel()
        if begin == end:
            continue
        if case["op"] == "gate_up":
            x = s["x"][torch.div(choice, k, rounding_mode="floor")].double()
            out[begin:end] = torch.nn.functional.silu(x @ s["w1"][e].double().t()) * (x @ s["w3"][e].double().t())
        else:
            y = s["h"][begin:end].double() @ s["w2"][e].double().t()
            out.index_add_(0, torch.div(choice, k, rounding_mode="floor"), y * s["weights"].view(-1)[choice].double()[:, None])
        begin = end
    return out
