"""Operators of large language models that the library offers as kernels of their own, as cases to be measured: the plain form of each
in elementary torch operations, and the calls that a user makes of the library.

  norm     Y, S, H = quantise(rms_norm(X + R) * w): H = X + R rounded to the type of X, Y in 8-bit floats with one scale in S for every
           128 columns of a row (or Y in the type of X, without S; without a residual there is no H)
  scaled   C[i][j] = sum_b SA[i][b] SB[j/128][b] sum_{k in block b} A[i][k] B[j][k], blocks of 128 along k, A and B in 8-bit floats
  grouped  C[t][j] = sum_k A[t][k] B[e(t)][j][k] (or B[e(t)][k][j]): the rows of A lie sorted by expert, offsets on the device say where an
           expert's rows begin; 8-bit floats carry scales as above.  Rows outside of all experts stay as they are in C.
  wgrad    D[e][i][j] = sum_{t of expert e} P[t][i] Q[t][j]: the gradient of the experts' weights, zero for an expert without rows
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "f8": torch.float8_e4m3fn}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "f8": 1}
BLOCK = 128          # columns (k values) that share a scale
LARGEST = 448.0      # of the 8-bit floats
EPS = 1e-6


def listed():
    return [
        # one token through the norm in front of a projection: latency
        {"name": "norm_1x4096", "op": "norm", "rows": 1, "cols": 4096, "type": "bf16", "out": "f8", "residual": True},
        # a batch of prompts, rows that are no whole blocks, no residual (the first layer)
        {"name": "norm_613x5000", "op": "norm", "rows": 613, "cols": 5000, "type": "f16", "out": "f8", "residual": False},
        # a full batch of long prompts: memory bandwidth
        {"name": "norm_16384x8192", "op": "norm", "rows": 16384, "cols": 8192, "type": "bf16", "out": "f8", "residual": True},
        # a few requests that each decode one token: the weights are what is read
        {"name": "scaled_4x4096x4096", "op": "scaled", "rows": 4, "cols": 4096, "depth": 4096, "out": "bf16"},
        # prompts of odd lengths, a projection that is no whole number of blocks either way
        {"name": "scaled_1111x2056x1360", "op": "scaled", "rows": 1111, "cols": 2056, "depth": 1360, "out": "f16"},
        # a full batch of prompts: the matrix cores
        {"name": "scaled_8192x8192x8192", "op": "scaled", "rows": 8192, "cols": 8192, "depth": 8192, "out": "bf16"},
        # two tokens that each go to eight experts
        {"name": "grouped_decode_bf16", "op": "grouped", "experts": 32, "empty": 20, "rows": 16, "tail": 0, "cols": 1024, "depth": 2048, "type": "bf16",
         "out": "bf16", "rows_of_k": True},
        # prompts through many experts, quantised weights
        {"name": "grouped_prefill_f8", "op": "grouped", "experts": 32, "empty": 1, "rows": 16384, "tail": 0, "cols": 2048, "depth": 4096, "type": "f8",
         "out": "bf16", "rows_of_k": True},
        # a training step's forward product over a few large experts
        {"name": "grouped_train_bf16", "op": "grouped", "experts": 8, "empty": 0, "rows": 8192, "tail": 0, "cols": 4096, "depth": 4096, "type": "bf16",
         "out": "bf16", "rows_of_k": True},
        # the gradient of the experts' inputs: the weights as they are, read the other way; a padded batch, experts without rows
        {"name": "grouped_input_grad_f16", "op": "grouped", "experts": 16, "empty": 3, "rows": 4099, "tail": 37, "cols": 1032, "depth": 2048, "type": "f16",
         "out": "f16", "rows_of_k": False},
        # the gradient of large experts' weights, in 32 bits for the optimiser
        {"name": "wgrad_train_bf16", "op": "wgrad", "experts": 8, "empty": 0, "rows": 8192, "tail": 0, "cols": 4096, "depth": 2048, "type": "bf16", "out": "f32"},
        # many small experts of odd sizes, some without rows
        {"name": "wgrad_odd_f16", "op": "wgrad", "experts": 24, "empty": 5, "rows": 1500, "tail": 11, "cols": 1032, "depth": 520, "type": "f16", "out": "f16"},
    ]


def _spread(rng, low, high, step=1):
    """An integer whose logarithm is spread evenly, a multiple of `step`."""
    return max(low, int(math.exp(rng.uniform(math.log(low), math.log(high))))) // step * step or step


def draw(rng):
    most = 2.0 * 8192 ** 3
    while True:
        op = rng.choice(["norm", "scaled", "grouped", "wgrad"])
        if op == "norm":
            kind = rng.choice(["bf16", "bf16", "f16", "f32"])
            case = {"op": op, "rows": _spread(rng, 1, 16384), "cols": _spread(rng, 256, 16384, rng.choice([1, 8, 128])), "type": kind,
                    "out": rng.choice(["f8", "f8", kind]), "residual": rng.random() < 0.7}
        elif op == "scaled":
            case = {"op": op, "rows": _spread(rng, 1, 16384), "cols": _spread(rng, 256, 16384, rng.choice([8, 128])),
                    "depth": _spread(rng, 256, 16384, rng.choice([16, 128])), "out": rng.choice(["bf16", "f16"])}
        else:
            experts = _spread(rng, 2, 64)
            kind = rng.choice(["bf16", "f16", "f8"]) if op == "grouped" else rng.choice(["bf16", "f16"])
            rows = _spread(rng, experts, 16384)
            case = {"op": op, "experts": experts, "empty": rng.randrange(0, experts // 2 + 1), "rows": rows, "tail": rng.choice([0, 0, rows // 20]),
                    "cols": _spread(rng, 256, 4096, rng.choice([8, 128])), "depth": _spread(rng, 256, 4096, rng.choice([16, 128])), "type": kind,
                    "out": {"f8": rng.choice(["bf16", "f16"])}.get(kind, kind)}
            if op == "grouped":
                case["rows_of_k"] = kind == "f8" or rng.random() < 0.6
            else:
                case["out"] = rng.choice([kind, "f32"])
        w = work(case)
        if w["flops"] <= most and w["bytes"] <= 1.0e9:
            return case


# ---------------------------------------------------------------- inputs

def _quantise(x):
    """x [..., rows, cols] in 8-bit floats with a scale for each BLOCK columns of a row."""
    rows, cols = x.shape[-2:]
    blocks = -(-cols // BLOCK)
    padded = torch.nn.functional.pad(x, (0, blocks * BLOCK - cols)).unflatten(-1, (blocks, BLOCK))
    scale = padded.abs().amax(-1).clamp_min(1e-12) / LARGEST
    q = (padded / scale.unsqueeze(-1)).flatten(-2)[..., :cols]
    return q.to(TYPES["f8"]).contiguous(), scale.contiguous()


def _quantise_weights(x):
    """x [..., rows, cols] with a scale for each BLOCK x BLOCK."""
    rows, cols = x.shape[-2:]
    rb, cb = -(-rows // BLOCK), -(-cols // BLOCK)
    padded = torch.nn.functional.pad(x, (0, cb * BLOCK - cols, 0, rb * BLOCK - rows)).unflatten(-1, (cb, BLOCK)).unflatten(-3, (rb, BLOCK))
    scale = padded.abs().amax((-3, -1)).clamp_min(1e-12) / LARGEST  # [..., rb, cb]
    q = (padded / scale[..., :, None, :, None]).flatten(-2).flatten(-3, -2)[..., :rows, :cols]
    return q.to(TYPES["f8"]).contiguous(), scale.contiguous()


def _counts(case, seed):
    """Rows of each expert: uneven shares, `empty` experts without any, each other at least one where there are enough."""
    rng = random.Random(seed * 1000003 + 17)
    experts, rows = case["experts"], case["rows"] - case["tail"]
    active = sorted(rng.sample(range(experts), experts - case["empty"]))
    share = [rng.expovariate(1.0) + 0.3 for _ in active]
    counts, left = [0] * experts, rows - len(active)
    for e, s in zip(active, share):
        counts[e] = 1 + int(left * s / sum(share))
    counts[active[-1]] += rows - sum(counts)
    return counts


def _inputs(case, seed):
    device = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device=device) * scale

    op, rows, cols = case["op"], case["rows"], case["cols"]
    if op == "norm":
        kind = TYPES[case["type"]]
        s = {"x": normal(rows, cols).to(kind), "w": (1 + normal(cols, scale=0.1)).to(kind)}
        if case["residual"]:
            s["r"] = normal(rows, cols, scale=2.0).to(kind)
        return s
    depth = case["depth"]
    if op == "scaled":
        a, sa = _quantise(normal(rows, depth))
        b, sb = _quantise_weights(normal(cols, depth, scale=0.03))
        return {"a": a, "sa": sa, "b": b, "sb": sb}
    counts = _counts(case, seed)
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    s = {"offsets": torch.tensor(at, dtype=torch.int32, device=device), "most": max(counts)}
    if op == "wgrad":
        s["p"] = normal(rows, cols, scale=0.1).to(TYPES[case["type"]])
        s["q"] = normal(rows, depth).to(TYPES[case["type"]])
        return s
    shape = (case["experts"], cols, depth) if case["rows_of_k"] else (case["experts"], depth, cols)
    a, b = normal(rows, depth), normal(*shape, scale=0.03)
    if case["type"] == "f8":
        s["a"], s["sa"] = _quantise(a)
        s["b"], s["sb"] = _quantise_weights(b)
    else:
        s["a"], s["b"] = a.to(TYPES[case["type"]]), b.to(TYPES[case["type"]])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    device = next(v.device for v in s.values() if isinstance(v, torch.Tensor))
    rows, cols = case["rows"], case["cols"]
    out = TYPES[case["out"]]
    if case["op"] == "norm":
        s["y"] = torch.empty(rows, cols, dtype=out, device=device)
        if case["out"] == "f8":
            s["s"] = torch.empty(rows, -(-cols // BLOCK), device=device)
        if case["residual"]:
            s["h"] = torch.empty_like(s["x"])
    elif case["op"] == "scaled":
        s["c"] = torch.empty(rows, cols, dtype=out, device=device)
    elif case["op"] == "grouped":
        s["c"] = torch.zeros(rows, cols, dtype=out, device=device)  # rows outside of all experts keep what they hold
    else:
        s["d"] = torch.empty(case["experts"], cols, case["depth"], dtype=out, device=device)
    if own:
        s["plan"] = _plan(case)
    return s


# ---------------------------------------------------------------- plain forms

def _norm(s):
    case = s["case"]
    x = s["x"].float()
    out = []
    if case["residual"]:
        h = (x + s["r"].float()).to(s["x"].dtype)
        x = h.float()
        out = [h]
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["w"].float()
    if case["out"] != "f8":
        return [y.to(s["x"].dtype)] + out
    rows, cols = y.shape
    blocks = -(-cols // BLOCK)
    y = torch.nn.functional.pad(y, (0, blocks * BLOCK - cols)).view(rows, blocks, BLOCK)
    scale = (y.abs().amax(-1) / LARGEST).clamp_min(2.0 ** -126)
    q = (y / scale.unsqueeze(-1)).view(rows, -1)[:, :cols]
    return [q.to(TYPES["f8"]), scale] + out


def _values(q, scale, each_row):
    """8-bit floats [..., rows, cols] times their scales."""
    rows, cols = q.shape[-2:]
    wide = scale.repeat_interleave(BLOCK, -1)[..., :cols]
    if not each_row:
        wide = wide.repeat_interleave(BLOCK, -2)[..., :rows, :]
    return q.float() * wide


def _scaled(s):
    c = _values(s["a"], s["sa"], True) @ _values(s["b"], s["sb"], False).t()
    return c.to(s["c"].dtype)


def _places(s, rows):
    """Of `most` places for each expert the row that each stands for, and whether it is one of the expert's."""
    first, last = s["offsets"][:-1].long(), s["offsets"][1:].long()
    at = first[:, None] + torch.arange(s["most"], device=first.device)
    inside = at < last[:, None]
    return at.clamp(max=rows - 1), inside


def _grouped(s):
    case = s["case"]
    a, b = s["a"], s["b"]
    if case["type"] == "f8":
        a, b = _values(a, s["sa"], True), _values(b, s["sb"], False)
    if case["rows_of_k"]:
        b = b.transpose(1, 2)
    b = b.to(torch.float32, memory_format=torch.contiguous_format)
    at, inside = _places(s, case["rows"])
    c = torch.bmm(a.float()[at], b)
    full = torch.zeros(case["rows"] + 1, case["cols"], device=c.device)
    full[torch.where(inside, at, case["rows"])] = c  # places that are no rows end up behind the last
    return full[:-1].to(s["c"].dtype)


def _wgrad(s):
    case = s["case"]
    at, inside = _places(s, case["rows"])
    p = torch.where(inside[..., None], s["p"].float()[at], 0.0).transpose(1, 2).contiguous()
    return torch.bmm(p, s["q"].float()[at]).to(s["d"].dtype)


# ---------------------------------------------------------------- the library's calls

def _plan(case):
    """What a user's program builds once for an operator's sizes: its kernels, loaded on the current device."""
    from paper_2205_13603_amd import binding as B
    rows, cols = case["rows"], case["cols"]
    if case["op"] == "norm":
        op = B.rms_norm_op(rows, cols, case["type"], case["out"], residual=case["residual"], eps=EPS)
    elif case["op"] == "scaled":
        op = B.scaled_gemm_op(rows, cols, case["depth"], case["out"])
    elif case["op"] == "grouped":
        op = B.grouped_gemm_op(case["experts"], rows, cols, case["depth"], case["rows_of_k"], case["type"], case["out"])
    else:
        op = B.grouped_wgrad_op(case["experts"], rows, cols, case["depth"], case["type"], case["out"])
    space = op.space()
    variant = B.Variant(op, space, B.default_trace(space))
    variant.prepare()
    return variant


def _call(s):
    from paper_2205_13603_amd import devmem
    op, stream = s["case"]["op"], devmem.current_stream()
    names = {"norm": ("x", "w", "r"), "scaled": ("a", "b", "sa", "sb"), "grouped": ("a", "b", "offsets", "sa", "sb"), "wgrad": ("p", "q", "offsets")}[op]
    outs = {"norm": ("y", "s", "h"), "scaled": ("c",), "grouped": ("c",), "wgrad": ("d",)}[op]
    if op == "norm":  # a tensor that the operator does not have is None
        s["plan"].launch([s[n].data_ptr() if n in s else None for n in names], [s[n].data_ptr() if n in s else None for n in outs], stream=stream)
    else:
        s["plan"].launch([s[n].data_ptr() for n in names if n in s], s[outs[0]].data_ptr(), stream=stream)
    got = [s[n] for n in outs if n in s]
    return got if op == "norm" else got[0]


def run(state):
    if own:
        return _call(state)
    return {"norm": _norm, "scaled": _scaled, "grouped": _grouped, "wgrad": _wgrad}[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    rows, cols = case["rows"], case["cols"]
    size, out = BYTES[case.get("type", "f8")], BYTES[case["out"]]
    if case["op"] == "norm":
        values = rows * cols
        moved = values * (size + out) + cols * size + (2 * values * size if case["residual"] else 0)
        moved += 4 * rows * -(-cols // BLOCK) if case["out"] == "f8" else 0
        return {"bytes": moved, "flops": (8 if case["out"] == "f8" else 5) * values}
    depth = case["depth"]
    blocks = -(-depth // BLOCK)
    if case["op"] == "scaled":
        moved = rows * depth + cols * depth + 4 * blocks * (rows + -(-cols // BLOCK)) + rows * cols * out
        return {"bytes": moved, "flops": 2.0 * rows * cols * depth}
    used, active = rows - case["tail"], case["experts"] - case["empty"]
    moved = 4 * (case["experts"] + 1)
    if case["op"] == "wgrad":
        moved += used * (cols + depth) * size + case["experts"] * cols * depth * out
    else:
        moved += used * depth * size + active * cols * depth * size + used * cols * out
        moved += 4 * blocks * (used + active * -(-cols // BLOCK)) if case["type"] == "f8" else 0
    return {"bytes": moved, "flops": 2.0 * used * cols * depth}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "norm":
        x = s["x"].double()
        h = None
        if case["residual"]:
            h = (x + s["r"].double()).to(s["x"].dtype)
            x = h.double()
        rows, cols = x.shape
        y = x / (x.square().sum(1) / cols + EPS).sqrt()[:, None] * s["w"].double()
        if case["out"] != "f8":
            return [y] + ([h] if h is not None else [])
        scale = torch.empty(rows, -(-cols // BLOCK), dtype=torch.float64, device=x.device)
        for b in range(scale.shape[1]):
            part = y[:, b * BLOCK:(b + 1) * BLOCK]
            scale[:, b] = part.abs().max(1).values / LARGEST
            part /= scale[:, b:b + 1].clamp_min(2.0 ** -126)
        return [y, scale.clamp_min(2.0 ** -126)] + ([h] if h is not None else [])

    def wide(q, scale, rows_per_scale):
        """Values of 8-bit floats [rows, cols] in 64 bits."""
        v = q.float().double()
        i = torch.arange(v.shape[0], device=v.device) // rows_per_scale
        j = torch.arange(v.shape[1], device=v.device) // BLOCK
        return v * scale.double()[i][:, j]

    if op == "scaled":
        return wide(s["a"], s["sa"], 1) @ wide(s["b"], s["sb"], BLOCK).t()
    at = s["offsets"].tolist()
    if op == "wgrad":
        d = torch.zeros(case["experts"], case["cols"], case["depth"], dtype=torch.float64, device=s["p"].device)
        for e in range(case["experts"]):
            d[e] = s["p"][at[e]:at[e + 1]].double().t() @ s["q"][at[e]:at[e + 1]].double()
        return d
    c = torch.zeros(case["rows"], case["cols"], dtype=torch.float64, device=s["a"].device)
    for e in range(case["experts"]):
        if at[e + 1] > at[e]:
            a, b = s["a"][at[e]:at[e + 1]], s["b"][e]
            if case["type"] == "f8":
                a, b = wide(a, s["sa"][at[e]:at[e + 1]], 1), wide(b, s["sb"][e], BLOCK)
            a, b = a.double(), b.double()
            c[at[e]:at[e + 1]] = a @ (b.t() if case["rows_of_k"] else b)
    return c
