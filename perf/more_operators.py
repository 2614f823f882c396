"""Operators around the products by expert, as cases to be measured: the plain form of each in elementary torch operations, and the calls
that a user makes of the library.

  route    which experts a token goes to, and with which weights.  Scores are the softmax or the sigmoid of a token's logits; the choice is by
           score plus a bias (for balance), first among groups of experts (by the sum of their best one or two), then among the experts of the
           groups that were kept; ties go to the lower index.  Weights are the chosen scores, without the bias, over their sum where that is
           asked for, times a constant.  Experts whose logit is -inf cannot be chosen; a choice that there is not has id -1 and weight 0.
           Backward: the gradient of the logits from that of the weights.
  order    the chosen rows sorted by expert, in the order of the tokens within each: offsets of the experts' rows and the row of each choice
  rows     "out": a token's row to the row of each of its choices, in the type it has or quantised to 8-bit integers with a scale for each
           row; "back": the rows of a token's choices times their weights, added up, and a residual; "grad": the gradients of "back"
  product  C[i][j] = SA[i] SB[j] sum_k A[i][k] B[j][k] in 8-bit integers, a scale for each token and each channel; with experts, the rows of A
           sorted by expert, times their expert's matrix.  Rows outside of all experts stay as they are in C.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "i8": 1}
LEAST = 2.0 ** -126  # scale of a row of zeros


def listed():
    return [
        # one token: latency
        {"name": "route_1x256", "op": "route", "backward": False, "tokens": 1, "masked": 0, "experts": 256, "chosen": 8, "type": "f32", "scores": "sigmoid", "bias": True,
         "groups": 8, "kept": 4, "best": 2, "renormalise": True, "scale": 2.5},
        # a padded batch of prompts, experts that are no power of two, plain softmax weights
        {"name": "route_1500x60", "op": "route", "backward": False, "tokens": 1500, "masked": 37, "experts": 60, "chosen": 6, "type": "bf16", "scores": "softmax", "bias": False,
         "groups": 1, "kept": 1, "best": 1, "renormalise": False, "scale": 1.0},
        # a training step's batch, groups of experts on several machines, a bias for balance
        {"name": "route_16384x256", "op": "route", "backward": False, "tokens": 16384, "masked": 0, "experts": 256, "chosen": 8, "type": "f32", "scores": "sigmoid", "bias": True,
         "groups": 8, "kept": 4, "best": 2, "renormalise": True, "scale": 2.5},
        # the same step's way back, all experts of a row involved
        {"name": "route_grad_16384x128", "op": "route", "backward": True, "tokens": 16384, "masked": 100, "experts": 128, "chosen": 8, "type": "bf16", "scores": "softmax",
         "bias": False, "groups": 1, "kept": 1, "best": 1, "renormalise": False, "scale": 1.0},
        # two tokens that each go to eight experts
        {"name": "order_2x8", "op": "order", "tokens": 2, "masked": 0, "experts": 32, "chosen": 8},
        # a training step's batch
        {"name": "order_16384x8", "op": "order", "tokens": 16384, "masked": 100, "experts": 256, "chosen": 8},
        # prompts to their experts, quantised on the way
        {"name": "rows_out_i8_4096x2048", "op": "rows", "way": "out", "tokens": 4096, "masked": 0, "experts": 64, "chosen": 8, "cols": 2048, "type": "bf16", "out": "i8",
         "residual": False},
        # a few tokens back from theirs, with what the layer adds them to
        {"name": "rows_back_7x4096", "op": "rows", "way": "back", "tokens": 7, "masked": 0, "experts": 32, "chosen": 8, "cols": 4096, "type": "bf16", "out": "bf16",
         "residual": True},
        # a training step's way back, rows that are no whole 16 bytes
        {"name": "rows_grad_3000x2050", "op": "rows", "way": "grad", "tokens": 3000, "masked": 11, "experts": 16, "chosen": 6, "cols": 2050, "type": "bf16", "out": "bf16",
         "residual": False},
        # a few requests that each decode one token: the weights are what is read
        {"name": "product_4x4096x4096", "op": "product", "experts": 0, "empty": 0, "rows": 4, "tail": 0, "cols": 4096, "depth": 4096, "out": "bf16"},
        # a full batch of prompts: the matrix cores
        {"name": "product_8192x8192x8192", "op": "product", "experts": 0, "empty": 0, "rows": 8192, "tail": 0, "cols": 8192, "depth": 8192, "out": "bf16"},
        # prompts through many experts, a padded batch, an expert without rows
        {"name": "product_experts_16384", "op": "product", "experts": 32, "empty": 1, "rows": 16384, "tail": 384, "cols": 2048, "depth": 4096, "out": "bf16"},
    ]


def _spread(rng, low, high, step=1):
    """An integer whose logarithm is spread evenly, a multiple of `step`."""
    return max(low, int(math.exp(rng.uniform(math.log(low), math.log(high))))) // step * step or step


def draw(rng):
    most = 2.0 * 8192 ** 3
    while True:
        op = rng.choice(["route", "route", "order", "rows", "rows", "product", "product"])
        if op == "product":
            experts = rng.choice([0, _spread(rng, 2, 64)])
            rows = _spread(rng, max(1, experts), 16384)
            case = {"op": op, "experts": experts, "empty": rng.randrange(0, experts // 2 + 1), "rows": rows, "tail": rng.choice([0, 0, rows // 20]) if experts else 0,
                    "cols": _spread(rng, 256, 4096 if experts else 16384, rng.choice([1, 8, 128])), "depth": _spread(rng, 256, 4096 if experts else 16384, rng.choice([16, 128])),
                    "out": rng.choice(["bf16", "f16", "f32"])}
        else:
            tokens = _spread(rng, 1, 16384)
            groups = rng.choice([1, 1, 2, 4, 8]) if op == "route" else 1
            experts = _spread(rng, 4, 512 // groups) * groups
            chosen = min(_spread(rng, 1, 16), experts // groups)
            case = {"op": op, "tokens": tokens, "masked": rng.choice([0, 0, tokens // 30]), "experts": experts, "chosen": chosen}
            if op == "route":
                backward = rng.random() < 0.4
                scores = rng.choice(["softmax", "sigmoid"])
                case |= {"backward": backward, "type": rng.choice(["f32", "bf16", "f16"]), "scores": scores, "bias": not backward and rng.random() < 0.5, "groups": groups,
                         "kept": rng.randrange(1, groups + 1), "best": rng.choice([1, 2]) if groups > 1 else 1, "renormalise": rng.random() < 0.6 and not (backward and chosen == 1),  # constant weights have no gradient
                         "scale": rng.choice([1.0, 2.5])}
            elif op == "rows":
                way, kind = rng.choice(["out", "back", "grad"]), rng.choice(["bf16", "bf16", "f16", "f32"])
                case |= {"way": way, "cols": _spread(rng, 64, 8192, rng.choice([1, 8, 128])), "type": kind, "out": rng.choice(["i8", kind]) if way == "out" else kind,
                         "residual": way == "back" and rng.random() < 0.5}
        w = work(case)
        if w["flops"] <= most and w["bytes"] <= 0.8e9:
            return case


# ---------------------------------------------------------------- inputs

def _counts(case, seed):
    """Rows of each expert: uneven shares, `empty` experts without any, each other at least one where there are enough."""
    rng = random.Random(seed * 1000003 + 17)
    experts, rows = case["experts"], case["rows"] - case["tail"]
    active = sorted(rng.sample(range(experts), experts - case["empty"]))[:max(1, rows)]
    share = [rng.expovariate(1.0) + 0.3 for _ in active]
    counts, left = [0] * experts, rows - len(active)
    for e, s in zip(active, share):
        counts[e] = 1 + int(left * s / sum(share))
    counts[active[-1]] += rows - sum(counts)
    return counts


def _quantise(x, least=1e-12):
    """x [..., rows, cols] in 8-bit integers with a scale for each row."""
    s = x.abs().amax(-1).clamp_min(least) / 127
    return (x / s.unsqueeze(-1)).round().to(torch.int8), s


def _places(ids, experts):
    """The row of each choice among all, sorted by expert and in the order of the tokens; -1 where there is no choice."""
    flat = ids.reshape(-1)
    order = torch.where(flat >= 0, flat, experts).argsort(stable=True)
    place = torch.empty_like(flat)
    place[order] = torch.arange(flat.numel(), dtype=flat.dtype, device=flat.device)
    return torch.where(flat >= 0, place, -1).view(ids.shape)


def _inputs(case, seed):
    device = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device=device) * scale

    op = case["op"]
    if op == "product":
        rows, cols, depth = case["rows"], case["cols"], case["depth"]
        s = {}
        s["a"], s["sa"] = _quantise(normal(rows, depth))
        if case["experts"]:
            counts = _counts(case, seed)
            at = [0]
            for c in counts:
                at.append(at[-1] + c)
            s["offsets"], s["most"] = torch.tensor(at, dtype=torch.int32, device=device), max(counts)
            s["b"], s["sb"] = _quantise(normal(case["experts"], cols, depth, scale=0.03))
        else:
            s["b"], s["sb"] = _quantise(normal(cols, depth, scale=0.03))
        return s
    tokens, experts, chosen = case["tokens"], case["experts"], case["chosen"]
    # experts differ in how much they are liked
    logits = normal(tokens, experts, scale=1.5) + normal(experts, scale=0.5)
    live = torch.arange(tokens, device=device) < tokens - case["masked"]
    if op == "route" and not case["backward"]:
        s = {"logits": logits.masked_fill(~live[:, None], -math.inf).to(TYPES[case["type"]])}
        if case["bias"]:
            s["bias"] = normal(experts, scale=0.1)
        return s
    # padding at the end goes nowhere
    ids = torch.where(live[:, None], logits.argsort(1, descending=True)[:, :chosen], -1).to(torch.int32).contiguous()
    if op == "route":
        return {"logits": logits.to(TYPES[case["type"]]), "ids": ids, "dw": normal(tokens, chosen)}
    if op == "order":
        return {"ids": ids}
    s = {"place": _places(ids, experts)}
    kind, cols = TYPES[case["type"]], case["cols"]
    if case["way"] != "back":
        s["x"] = normal(tokens, cols).to(kind)
    if case["way"] != "out":
        s["c"] = normal(tokens * chosen, cols).to(kind)
        s["w"] = torch.rand(tokens, chosen, generator=g, device=device)
    if case["residual"]:
        s["r"] = normal(tokens, cols).to(kind)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    device = next(v.device for v in s.values() if isinstance(v, torch.Tensor))
    s["case"] = case
    if case["op"] == "product":
        s["y"] = torch.zeros(case["rows"], case["cols"], dtype=TYPES[case["out"]], device=device)  # rows outside of all experts keep what they hold
    else:
        tokens, experts, chosen = case["tokens"], case["experts"], case["chosen"]
        if case["op"] == "route" and case["backward"]:
            s["y"] = torch.empty_like(s["logits"])
        elif case["op"] == "route":
            s["ids"] = torch.empty(tokens, chosen, dtype=torch.int32, device=device)
            s["w"] = torch.empty(tokens, chosen, device=device)
        elif case["op"] == "order":
            s["offsets"] = torch.empty(experts + 1, dtype=torch.int32, device=device)
            s["place"] = torch.empty(tokens, chosen, dtype=torch.int32, device=device)
        elif case["way"] == "back":
            s["y"] = torch.empty(tokens, case["cols"], dtype=TYPES[case["out"]], device=device)
        else:
            s["y"] = torch.zeros(tokens * chosen, case["cols"], dtype=TYPES[case["out"]], device=device)  # rows of no choice keep what they hold
            if case["out"] == "i8":
                s["s"] = torch.zeros(tokens * chosen, device=device)
            if case["way"] == "grad":
                s["dw"] = torch.empty(tokens, chosen, device=device)
    if own:
        s["plan"] = _plan(case)
        if case["op"] == "order":
            s["workspace"] = torch.empty(max(1, s["plan"].workspace_bytes()), dtype=torch.uint8, device=device)
    return s


# ---------------------------------------------------------------- plain forms

def _scores(case, x):
    if case["scores"] == "sigmoid":
        return 1 / (1 + torch.exp(-x))
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _route(s):
    case = s["case"]
    chosen, groups = case["chosen"], case["groups"]
    x = s["logits"].double()  # whom a token goes to must not hang on how an exponential rounds
    there = x > -math.inf
    row = there.any(-1, keepdim=True)
    score = _scores(case, torch.where(row, x, 0.0))
    # scores order as their logits do
    choice = x if not case["bias"] and case["best"] == 1 else score + s["bias"].double() if case["bias"] else score
    choice = torch.where(there, choice, -math.inf)
    if groups > 1:
        each = choice.unflatten(-1, (groups, -1))
        best = each.sort(-1, descending=True).values[..., :case["best"]]
        value = torch.where(best > -math.inf, best, 0.0).sum(-1).masked_fill(~there.unflatten(-1, (groups, -1)).any(-1), -math.inf)
        first = value.sort(dim=-1, descending=True, stable=True).indices[:, :case["kept"]]
        keep = torch.zeros_like(value, dtype=torch.bool).scatter_(1, first, True)
        choice = each.masked_fill(~keep.unsqueeze(-1), -math.inf).flatten(-2)
    ordered, ids = choice.sort(dim=-1, descending=True, stable=True)
    ids, real = ids[:, :chosen], ordered[:, :chosen] > -math.inf
    w = score.gather(1, ids) * real
    if case["renormalise"]:
        w = w / torch.where(real.any(-1, keepdim=True), w.sum(-1, keepdim=True), 1.0)
    return [torch.where(real, ids, -1).to(torch.int32), (w * case["scale"]).float()]


def _route_grad(s):
    case = s["case"]
    x, real = s["logits"].float(), s["ids"] >= 0
    ids = s["ids"].clamp_min(0).long()
    g = s["dw"] * real * case["scale"]
    score = _scores(case, x)
    if case["renormalise"]:
        p = score.gather(1, ids) * real
        total = torch.where(real.any(-1, keepdim=True), p.sum(-1, keepdim=True), 1.0)
        g = (g - (g * (p / total)).sum(-1, keepdim=True)) / total * real
    d = torch.zeros_like(x).scatter_add_(1, ids, g)
    d = score * (d - (d * score).sum(-1, keepdim=True)) if case["scores"] == "softmax" else d * score * (1 - score)
    return d.to(s["logits"].dtype)


def _order(s):
    ids = s["ids"]
    flat = torch.where(ids >= 0, ids, s["case"]["experts"]).reshape(-1)
    ordered, order = flat.sort(dim=0, stable=True)
    place = torch.empty_like(flat)
    place[order] = torch.arange(flat.numel(), dtype=torch.int32, device=flat.device)
    place = torch.where(ids >= 0, place.view(ids.shape), -1)
    offsets = torch.searchsorted(ordered, torch.arange(s["case"]["experts"] + 1, dtype=torch.int32, device=flat.device))
    return [offsets.to(torch.int32), place]


def _to_places(s, values):
    """values [tokens, chosen, ...] at the rows of their choices, zeros elsewhere."""
    place = s["place"]
    rows = place.numel()
    full = torch.zeros(rows + 1, *values.shape[2:], dtype=values.dtype, device=values.device)
    full[torch.where(place >= 0, place, rows).long()] = values  # choices that there are not end up behind the last row
    return full[:-1]


def _rows(s):
    case = s["case"]
    place, way = s["place"], case["way"]
    if way == "out":
        x = s["x"].float()
        if case["out"] == "i8":
            scale = (x.abs().amax(-1) / 127).clamp_min(LEAST)
            q = (x / scale[:, None]).round().to(torch.int8)
            return [_to_places(s, t[:, None].expand(*place.shape, *t.shape[1:])) for t in (q, scale)]
        return _to_places(s, s["x"][:, None].expand(*place.shape, -1))
    real = place >= 0
    c = s["c"].float()[place.clamp_min(0).long()]
    if way == "back":
        y = (torch.where(real, s["w"], 0.0)[..., None] * torch.where(real[..., None], c, 0.0)).sum(1)
        if case["residual"]:
            y = y + s["r"].float()
        return y.to(s["y"].dtype)
    x = s["x"].float()[:, None]
    return [_to_places(s, (s["w"][..., None] * x).to(s["y"].dtype)), (c * x).sum(-1) * real]


def _product(s):
    case = s["case"]
    a, b = s["a"].double(), s["b"].double()  # sums of more than 24 bits
    if not case["experts"]:
        return (a @ b.t() * s["sa"].double()[:, None] * s["sb"].double()).to(s["y"].dtype)
    rows = case["rows"]
    first, last = s["offsets"][:-1].long(), s["offsets"][1:].long()
    at = first[:, None] + torch.arange(s["most"], device=first.device)
    inside, at = at < last[:, None], at.clamp(max=rows - 1)
    c = torch.bmm(a[at], b.transpose(1, 2).contiguous()) * s["sa"].double()[at][..., None] * s["sb"].double()[:, None]
    full = torch.zeros(rows + 1, case["cols"], dtype=s["y"].dtype, device=c.device)
    full[torch.where(inside, at, rows)] = c.to(full.dtype)  # places that are no rows end up behind the last
    return full[:-1]


# ---------------------------------------------------------------- the library's calls

def _plan(case):
    """What a user's program builds once for an operator's sizes: its kernels, loaded on the current device."""
    from paper_2205_13603_amd import binding as B
    if case["op"] == "product":
        rows, cols, depth, experts = case["rows"], case["cols"], case["depth"], case["experts"]
        op = B.grouped_gemm_op(experts, rows, cols, depth, True, "i8", case["out"]) if experts else B.scaled_gemm_op(rows, cols, depth, case["out"], in_dtype="i8")
    else:
        tokens, experts, chosen = case["tokens"], case["experts"], case["chosen"]
        if case["op"] == "order":
            op = B.expert_order_op(experts, tokens, chosen)
        elif case["op"] == "rows":
            sizes = (tokens, chosen, case["cols"], tokens * chosen, case["type"])
            op = {"out": lambda: B.spread_rows_op(*sizes, case["out"]), "back": lambda: B.join_rows_op(*sizes, residual=case["residual"]), "grad": lambda: B.join_grad_op(*sizes)}[case["way"]]()
        elif case["backward"]:
            op = B.route_grad_op(tokens, experts, chosen, case["type"], scores=case["scores"], renormalise=case["renormalise"], scale=case["scale"])
        else:
            op = B.route_op(tokens, experts, chosen, case["type"], scores=case["scores"], bias=case["bias"], groups=case["groups"], kept=case["kept"], best=case["best"],
                            renormalise=case["renormalise"], scale=case["scale"])
    space = op.space()
    variant = B.Variant(op, space, B.default_trace(space))
    variant.prepare()
    return variant


def _call(s):
    from paper_2205_13603_amd import devmem
    case, stream = s["case"], devmem.current_stream()
    op = case["op"]
    if op == "product":
        names, outs = ("a", "b", "offsets", "sa", "sb") if case["experts"] else ("a", "b", "sa", "sb"), ("y",)
    elif op == "order":
        names, outs = ("ids",), ("offsets", "place")
    elif op == "route":
        names, outs = (("logits", "ids", "dw"), ("y",)) if case["backward"] else (("logits", "bias"), ("ids", "w"))
    else:
        names, outs = {"out": (("x", "place"), ("y", "s")), "back": (("c", "place", "w", "r"), ("y",)), "grad": (("x", "place", "w", "c"), ("y", "dw"))}[case["way"]]
    # a tensor that the operator does not have is None
    s["plan"].launch([s[n].data_ptr() if n in s else None for n in names], [s[n].data_ptr() if n in s else None for n in outs], stream=stream,
                     workspace=s["workspace"].data_ptr() if op == "order" else None)
    got = [s[n] for n in outs if n in s]
    return got if len(got) > 1 else got[0]


def run(state):
    if own:
        return _call(state)
    op = state["case"]["op"]
    if op == "route" and state["case"]["backward"]:
        return _route_grad(state)
    return {"route": _route, "order": _order, "rows": _rows, "product": _product}[op](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"] == "product":
        used, active = case["rows"] - case["tail"], max(1, case["experts"] - case["empty"])
        cols, depth = case["cols"], case["depth"]
        moved = used * depth + active * cols * depth + 4 * (used + active * cols) + used * cols * BYTES[case["out"]] + (4 * (case["experts"] + 1) if case["experts"] else 0)
        return {"bytes": moved, "flops": 2.0 * used * cols * depth}
    tokens, experts, chosen = case["tokens"], case["experts"], case["chosen"]
    live = tokens - case["masked"]
    if case["op"] == "order":
        return {"bytes": 8 * tokens * chosen + 4 * (experts + 1), "flops": 0}
    if case["op"] == "route":
        logits = tokens * experts * BYTES[case["type"]]
        if not case["backward"]:  # scores (exponential, sum, quotient), one comparison for each
            return {"bytes": logits + 8 * tokens * chosen + (4 * experts if case["bias"] else 0), "flops": 5 * tokens * experts}
        dense = case["scores"] == "softmax" and not case["renormalise"]  # otherwise the chosen logits are all that is read
        return {"bytes": logits + (logits if dense else live * chosen * BYTES[case["type"]]) + 8 * tokens * chosen, "flops": (8 if dense else 1) * tokens * experts}
    cols, size = case["cols"], BYTES[case["type"]]
    token, row = live * cols * size, live * chosen * cols
    if case["way"] == "out":
        return {"bytes": token + row * BYTES[case["out"]] + 4 * tokens * chosen + (4 * live * chosen if case["out"] == "i8" else 0), "flops": 4 * live * cols if case["out"] == "i8" else 0}
    if case["way"] == "back":
        return {"bytes": row * size + tokens * cols * (BYTES[case["out"]] + (size if case["residual"] else 0)) + 8 * tokens * chosen, "flops": 2 * row}
    return {"bytes": token + 2 * row * size + 12 * tokens * chosen, "flops": 3 * row}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_weights(case, s):
    """Ranks counted pair by pair, a few tokens at a time."""
    experts, chosen, groups = case["experts"], case["chosen"], case["groups"]
    index = torch.arange(experts, device=s["logits"].device)
    out = []
    for x in s["logits"].double().split(max(1, (1 << 25) // experts ** 2)):
        low = x.amax(-1, keepdim=True).clamp_min(-1e300)
        e = (x - low).exp()
        score = e / e.sum(-1, keepdim=True) if case["scores"] == "softmax" else x.sigmoid()
        key = score + s["bias"].double() if case["bias"] else score if case["best"] > 1 else x
        key = key.masked_fill(x == -math.inf, -math.inf)
        if groups > 1:
            size = experts // groups
            value = torch.stack([key[:, i * size:(i + 1) * size].topk(min(case["best"], size)).values.clamp_min(-1e30).sum(-1) for i in range(groups)], 1)
            ahead = (value[:, None] > value[..., None]) | ((value[:, None] == value[..., None]) & (index[:groups] < index[:groups, None]))
            key = key.masked_fill((ahead.sum(-1) >= case["kept"]).repeat_interleave(size, 1), -math.inf)
        rank = ((key[:, None] > key[..., None]) | ((key[:, None] == key[..., None]) & (index < index[:, None]))).sum(-1)
        w = torch.zeros(len(x), chosen, dtype=torch.float64, device=x.device)
        token, expert = torch.nonzero((rank < chosen) & (key > -math.inf), as_tuple=True)
        w[token, rank[token, expert]] = score[token, expert]
        if case["renormalise"]:
            total = w.sum(-1, keepdim=True)
            w = w / torch.where(total > 0, total, 1.0)
        out.append(w * case["scale"])
    return torch.cat(out)


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "order":
        return None
    if op == "product":
        c = torch.zeros(case["rows"], case["cols"], dtype=torch.float64, device=s["a"].device)
        at = s["offsets"].tolist() if case["experts"] else [0, case["rows"]]
        for e in range(len(at) - 1):
            rows = slice(at[e], at[e + 1])
            b, sb = (s["b"][e], s["sb"][e]) if case["experts"] else (s["b"], s["sb"])
            c[rows] = (s["a"][rows].double() * s["sa"][rows].double()[:, None]) @ (b.double() * sb.double()[:, None]).t()
        return c
    if op == "route" and not case["backward"]:
        return [None, _exact_weights(case, s)]
    if op == "route":
        # the jacobian of the weights, row by row of the chosen: d w_j / d l_e
        d = torch.zeros_like(s["logits"], dtype=torch.float64)
        x, real = s["logits"].double(), s["ids"] >= 0
        score = (x - x.logsumexp(-1, keepdim=True)).exp() if case["scores"] == "softmax" else x.sigmoid()
        p = score.gather(1, s["ids"].clamp_min(0).long()) * real
        total = p.sum(-1).clamp_min(1e-300) if case["renormalise"] else torch.ones_like(p[:, 0])
        w = p / total[:, None]
        g = s["dw"].double() * case["scale"]
        for j in range(case["chosen"]):
            on = torch.nn.functional.one_hot(s["ids"][:, j].clamp_min(0).long(), case["experts"]).double() * real[:, j:j + 1]
            if case["scores"] == "softmax" and not case["renormalise"]:
                d += g[:, j:j + 1] * p[:, j:j + 1] * (on - score)
            else:
                slope = torch.ones_like(p) if case["scores"] == "softmax" else 1 - p  # of the logarithm of a score
                d += g[:, j:j + 1] * w[:, j:j + 1] * on * slope[:, j:j + 1]
                if case["renormalise"]:
                    d.scatter_add_(1, s["ids"].clamp_min(0).long(), -g[:, j:j + 1] * w[:, j:j + 1] * w * slope * real)
        return d
    place, way = s["place"].long(), case["way"]
    token, choice = torch.nonzero(place >= 0, as_tuple=True)
    row = place[token, choice]
    if way == "out":
        a = torch.zeros(place.numel(), case["cols"], dtype=torch.float64, device=place.device)
        if case["out"] == "i8":
            scale = torch.zeros(place.numel(), dtype=torch.float64, device=place.device)
            scale[row] = s["x"][token].double().abs().amax(-1) / 127
            return [None, scale]
        a[row] = s["x"][token].double()
        return a
    if way == "back":
        y = s["r"].double() if case["residual"] else torch.zeros(place.shape[0], case["cols"], dtype=torch.float64, device=place.device)
        return y.index_add(0, token, s["c"][row].double() * s["w"][token, choice].double()[:, None])
    dc = torch.zeros(place.numel(), case["cols"], dtype=torch.float64, device=place.device)
    dw = torch.zeros(place.shape, dtype=torch.float64, device=place.device)
    x = s["x"][token].double()
    dc[row] = x * s["w"][token, choice].double()[:, None]
    dw[token, choice] = (x * s["c"][row].double()).sum(-1)
    return [dc, dw]
