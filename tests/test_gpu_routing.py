"""Routing to experts on the GPU: the choice of experts and its gradient, the order of the choices, rows to their choices and back, against
their definitions in 64 bits.

Tolerances.  Ids, places, offsets, copies and quantised integers are equal.  Weights are formed in 64 bits and rounded to fp32 once, 2^-24, but for a
softmax over all logits that choose by themselves, whose sum is one of fp32 exponentials: an exponential is off by one step (2^-23) and half a step of its
argument's size, which times e^-x is less than half a step more; 32 of a lane and 6 steps over lanes add up to 38 * 2^-24; 44 * 2^-24 in all."""
import numpy as np
import pytest
import torch

from paper_2205_13603_amd import binding as B, devmem
from test_gpu_layers import HALF_STEP, TYPES, dev, guarded, normal, offsets_of, rng, variant

pytestmark = pytest.mark.gpu

TYPES = dict(TYPES, i8=torch.int8, i32=torch.int32)
INF, NAN = float("inf"), float("nan")
PART = torch.tensor(1.0) / 127  # in fp32


def call(v, inputs, out_shapes, instances=1, stream=None):
    """Outputs of two launches, equal bit for bit, nothing written around them."""
    got = []
    for _ in range(2):
        whole = [guarded(*s) if s else (None, None) for s in out_shapes]
        ws = torch.full((max(1, v.workspace_bytes() * instances),), 0x55, dtype=torch.uint8, device="cuda")
        v.launch([x.data_ptr() if x is not None else None for x in inputs], [w[1].data_ptr() if w[1] is not None else None for w in whole], instances=instances,
                 stream=stream or devmem.current_stream(), workspace=ws.data_ptr())
        torch.cuda.synchronize()
        for w in whole:
            if w[0] is not None:
                assert bool((torch.cat([w[0][:64], w[0][-64:]]).float() == 7.0).all()), "written around the output"
        got.append([w[1].cpu() if w[1] is not None else None for w in whole])
    for a, b in zip(*got):
        if a is not None:
            assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)), "two launches differ"
    return got[0]


# ---------------------------------------------------------------- the choice

def route_definition(x, bias, K, scores="softmax", groups=1, kept=1, best=1, renormalise=False, scale=1.0):
    """Token by token, with Python's numbers."""
    T, E = x.shape
    ids, w = torch.full((T, K), -1, dtype=torch.int32), torch.zeros(T, K, dtype=torch.float64)
    x = x.double()
    for t in range(T):
        row = x[t]
        nan = bool(torch.isnan(row).any()) or (scores == "softmax" and bool((row == INF).any()))
        clean = torch.where(torch.isnan(row), torch.tensor(-INF, dtype=torch.float64), row)
        if scores == "sigmoid":
            s = torch.sigmoid(row)
        else:
            m = float(clean.max())
            e = (clean - (m if m > -INF else 0)).exp()
            s = e / e.sum() if not nan and m > -INF else torch.full_like(e, NAN if nan else 0)
        by_logit = bias is None and (groups == 1 or best == 1)
        c = clean if by_logit else s + (bias.double() if bias is not None else 0)
        c = [float(c[e]) if float(clean[e]) > -INF and float(c[e]) > -INF else None for e in range(E)]
        take = list(range(E))
        if groups > 1:
            size, sums = E // groups, []
            for g in range(groups):
                own = sorted((c[e] for e in range(g * size, g * size + size) if c[e] is not None), reverse=True)[:best]
                sums.append(sum(own) if own else None)
            keep = sorted((g for g in range(groups) if sums[g] is not None), key=lambda g: (-sums[g], g))[:kept]
            take = [e for e in take if e // size in keep]
        order = sorted((e for e in take if c[e] is not None), key=lambda e: (-c[e], e))[:K]
        for j, e in enumerate(order):
            ids[t, j] = e
        if nan:
            w[t] = NAN
        elif order:
            p = s[order]
            if renormalise and scores == "softmax":  # relative to the largest of them
                p = (clean[order] - clean[order].max()).exp()
            w[t, :len(order)] = (p / p.sum() if renormalise else p) * scale
    return ids, w


def check_route(v, x, bias, K, **kw):
    T, E = x.shape
    ids, w = call(v, [dev(x), dev(bias)], [((T, K), torch.int32), ((T, K), torch.float32)])
    want, weights = route_definition(x, bias, K, **kw)
    assert torch.equal(ids, want), "the first at %s" % (ids != want).nonzero()[0].tolist()
    all_logits = kw.get("scores", "softmax") == "softmax" and not kw.get("renormalise")
    assert torch.equal(torch.isnan(w), torch.isnan(weights))
    fine = ~torch.isnan(weights)
    assert bool(((w.double() - weights).abs()[fine] <= weights.abs()[fine] * (44 if all_logits else 1.01) * 2.0 ** -24 + 1e-37).all())


ROUTES = [(1, 1, 1, {}), (1, 256, 8, dict(scores="sigmoid", bias=True, groups=8, kept=4, best=2, renormalise=True, scale=2.5)), (3, 2, 2, {}), (67, 60, 6, {}),
          (70, 64, 4, dict(renormalise=True)), (130, 7, 3, dict(scores="sigmoid")), (33, 160, 6, dict(groups=8, kept=3)), (40, 128, 32, dict(bias=True)), (9, 1024, 32, dict(renormalise=True, bias=True)),
          (21, 1000, 17, dict(scores="sigmoid", bias=True, renormalise=True)), (50, 72, 5, dict(groups=6, kept=2, best=2, scale=0.3)), (50, 72, 8, dict(groups=36, kept=3, best=2, bias=True)),
          (50, 128, 2, dict(groups=64, kept=64, best=1, scores="sigmoid")), (25, 512, 10, dict(groups=2, kept=1, best=2, scores="sigmoid", bias=True)), (12, 8, 8, dict(renormalise=True, scale=16.0)),
          (45, 48, 12, dict(groups=4, kept=1, best=2, bias=True, renormalise=True))]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("which", range(len(ROUTES)))
def test_route(which, kind):
    T, E, K, kw = ROUTES[which]
    op = B.route_op(T, E, K, kind, **kw)
    g = rng(which)
    x = (normal(g, T, E, scale=1.5) + normal(g, E, scale=0.5)).to(TYPES[kind])
    bias = normal(g, E, scale=0.2) if kw.get("bias") else None
    for t in range(0, T, 5):
        x[t, torch.rand(E, generator=g) < 0.5] = -INF  # some experts
    if T > 8:
        x[3] = -INF   # all of them
        x[4, 1:] = -INF
        x[6] = 0.5    # all alike
    rest = {k: v for k, v in kw.items() if k != "bias"}
    space = op.space()
    for c in range(space.slots[0].n_candidates):
        if space.slots[0].weight[c]:
            v = variant(op, space.slots[0].candidates[c])
            if v is not None:
                check_route(v, x, bias, K, **rest)


def test_route_of_many_tokens():
    T, E, K = 40000, 16, 2
    v = variant(B.route_op(T, E, K, "bf16", renormalise=True))
    if v is None:
        return
    x = normal(rng(5), T, E).bfloat16()
    ids, w = call(v, [dev(x), None], [((T, K), torch.int32), ((T, K), torch.float32)])
    top, order = x.double().sort(dim=1, descending=True, stable=True)
    assert torch.equal(ids, order[:, :K].int())
    want = torch.softmax(top[:, :K], 1)
    assert bool(((w.double() - want).abs() <= want * 1.01 * 2.0 ** -24).all())


def test_ties_go_to_the_lower_index():
    """Equal logits, zeros of both signs, equal scores and biases, equal sums of groups."""
    T, E, K = 6, 96, 7
    plain, biased = variant(B.route_op(T, E, K)), variant(B.route_op(T, E, K, scores="sigmoid", bias=True))
    grouped = variant(B.route_op(T, E, K, groups=12, kept=5, best=2, scores="sigmoid"))
    if plain is None:
        return
    x = torch.zeros(T, E)
    x[1, ::2] = -0.0
    x[2, 5::7] = 1
    x[3] = torch.arange(E) % 4
    x[4] = -3
    x[5, 40:] = 2.5
    check_route(plain, x, None, K)
    check_route(biased, x, torch.zeros(E), K, scores="sigmoid")
    check_route(biased, x, (torch.arange(E) % 3 == 1).float(), K, scores="sigmoid")
    check_route(grouped, x, None, K, scores="sigmoid", groups=12, kept=5, best=2)
    ids, _ = call(plain, [dev(x), None], [((T, K), torch.int32), ((T, K), torch.float32)])
    assert ids[0].tolist() == ids[1].tolist() == ids[4].tolist() == list(range(K)) and ids[2].tolist() == list(range(5, 5 + 7 * K, 7))


def test_near_choices_are_told_apart():
    """Logits one step of fp32 apart, whose fp32 scores are equal, decide; so do steps of the bias below those of fp32 scores."""
    E, K = 64, 4
    v, b, plain = variant(B.route_op(E, E, K, scores="sigmoid", bias=True)), variant(B.route_op(1, E, K, bias=True)), variant(B.route_op(E, E, K, scores="sigmoid"))
    if v is None:
        return
    x = torch.full((E, E), 3.0)
    for t in range(E):
        for n in range(K):
            x[t, (t * 7 + n * 11) % E] = float(np.float32(3.0) + np.float32(2.0 ** -22 * (n + 1)))
    assert int((torch.sigmoid(x[0]) == torch.sigmoid(torch.tensor(3.0))).sum()) > E - K  # fp32 would not see all of them
    check_route(v, x, torch.zeros(E), K, scores="sigmoid")
    check_route(plain, x + 40, None, K, scores="sigmoid")  # scores of 1 in 64 bits: the logits choose
    bias = torch.full((E,), 2.0 ** -30) * torch.arange(E)
    check_route(b, torch.full((1, E), 0.25), bias, K)
    ids, _ = call(b, [torch.full((1, E), 0.25).cuda(), dev(bias)], [((1, K), torch.int32), ((1, K), torch.float32)])
    assert ids[0].tolist() == [63, 62, 61, 60]


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_masks_infinities_and_nan(scores, renormalise):
    T, E, K = 12, 40, 5
    kw = dict(scores=scores, renormalise=renormalise)
    plain, biased, grouped = variant(B.route_op(T, E, K, **kw)), variant(B.route_op(T, E, K, bias=True, **kw)), variant(B.route_op(T, E, K, bias=True, groups=10, kept=2, best=2, **kw))
    if plain is None:
        return
    g = rng(6)
    x = normal(g, T, E)
    x[0] = -INF
    x[1, 4:] = -INF           # four to choose from
    x[2, :] = -INF
    x[2, 39] = 1
    x[3, 7] = NAN
    x[4, 8] = INF
    x[5] = torch.finfo(torch.float32).min  # a mask that is no infinity
    x[6, ::2] = torch.finfo(torch.float32).min
    x[7] = NAN
    x[8] = 80
    x[9, 3] = 300
    x[10, 4:8] = -INF         # a whole group
    x[11, :36] = -INF         # one group left
    bias = normal(g, E, scale=0.1)
    bias[5], bias[6], bias[9] = -INF, INF, NAN
    if not (scores == "sigmoid" and renormalise):  # row 5: 0 / 0
        check_route(plain, x, None, K, **kw)
    x[5] = -1
    check_route(plain, x, None, K, **kw)
    check_route(biased, x, bias, K, **kw)
    check_route(grouped, x, bias, K, groups=10, kept=2, best=2, **kw)


def test_route_strides_and_instances():
    R, T, E, K = 3, 37, 60, 6
    op = B.route_op(T, E, K, "bf16", scores="sigmoid", bias=True, a_strides=[0, 77, 1])
    v, grad = variant(op), variant(B.route_grad_op(T, E, K, "bf16", a_strides=[0, 77, 1]))
    if v is None:
        return
    g = rng(8)
    x, bias = normal(g, R, T, E).bfloat16(), normal(g, R, E, scale=0.3)
    span = op.tensor_bytes(0) // 2
    flat = torch.full((3 + R * span,), NAN, dtype=torch.bfloat16)
    for r in range(R):
        torch.as_strided(flat, (T, E), (77, 1), 3 + r * span).copy_(x[r])
    flat = dev(flat)
    ids, w = call(v, [flat[3:], dev(bias)], [((R, T, K), torch.int32), ((R, T, K), torch.float32)], instances=R)
    dw = normal(g, R, T, K)
    (dx,) = call(grad, [flat[3:], dev(ids), dev(dw)], [((R, T, E), torch.bfloat16)], instances=R)
    for r in range(R):
        want, weights = route_definition(x[r], bias[r], K, scores="sigmoid")
        assert torch.equal(ids[r], want) and bool(((w[r].double() - weights).abs() <= weights * 1.01 * 2.0 ** -24).all())
        want, mag = grad_definition(x[r], ids[r], dw[r])
        assert bool(((dx[r].double() - want).abs() <= want.abs() * 2.0 ** -8 + mag * 2.0 ** -18).all())


# ---------------------------------------------------------------- its gradient

def grad_definition(x, ids, dw, scores="softmax", renormalise=False, scale=1.0):
    """By automatic differentiation of the definition in 64 bits; and the magnitudes that its sums are made of."""
    x = x.double().requires_grad_(True)
    real = (ids >= 0) & (ids < x.shape[1])
    at = torch.where(real, ids, 0).long()
    if scores == "sigmoid":
        s = torch.sigmoid(x)
    elif renormalise:  # the sum of all exponentials cancels: left out, the other logits' gradient is zero instead of what the cancelling leaves
        s = (x - x.detach().amax(1, keepdim=True).clamp_min(-1e300)).exp()
    else:
        s = torch.softmax(torch.where(torch.isinf(x).all(1, keepdim=True), torch.zeros_like(x), x), 1)
    p = s.gather(1, at) * real
    total = p.sum(1, keepdim=True)
    w = p / torch.where(total > 0, total, torch.ones_like(total)) if renormalise else p
    (w * dw.double() * scale).sum().backward()
    g = (dw.double() * scale).abs() * real
    q = w.detach()
    mag = torch.zeros_like(s).scatter_add_(1, at, g * q + (g * q).sum(1, keepdim=True) * q)
    if scores == "softmax" and not renormalise:
        mag = mag + s.detach() * (g * q).sum(1, keepdim=True)
    return x.grad, mag


GRADS = [(1, 1, 1), (1, 256, 8), (67, 60, 6), (130, 7, 3), (40, 128, 32), (9, 1024, 32), (21, 1000, 17), (300, 16, 2)]


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("which", range(len(GRADS)))
def test_route_gradient(which, kind, renormalise, scores):
    """A sum of E fp32 terms and a handful of products: less than 64 steps of what is added up, and the one rounding."""
    T, E, K = GRADS[which]
    op = B.route_grad_op(T, E, K, kind, scores=scores, renormalise=renormalise, scale=2.5)
    g = rng(which + 100)
    x = normal(g, T, E, scale=1.5).to(TYPES[kind])
    ids = torch.stack([torch.randperm(E, generator=g)[:K] for _ in range(T)]).int()
    dw = normal(g, T, K)
    for t in range(2, T, 4):
        ids[t, torch.rand(K, generator=g) < 0.4] = -1
    if T > 8:
        ids[3] = -1
        ids[5, 0] = E      # no expert
        ids[6, K - 1] = ids[6, 0]  # twice
        x[7] = -INF        # a padded row
        ids[7] = -1
    want, mag = grad_definition(x, ids, dw, scores, renormalise, 2.5)
    want[torch.isinf(x).all(1)] = 0
    space = op.space()
    for c in range(space.slots[0].n_candidates):
        if not space.slots[0].weight[c]:
            continue
        v = variant(op, space.slots[0].candidates[c])
        if v is None:
            continue
        (dx,) = call(v, [dev(x), dev(ids), dev(dw)], [((T, E), TYPES[kind])])
        tol = want.abs() * HALF_STEP[kind] * 1.01 + mag * 64 * 2.0 ** -24 + (2.0 ** -25 if kind == "f16" else 1e-37)
        assert bool(((dx.double() - want).abs() <= tol).all())
        if not (scores == "softmax" and not renormalise):
            other = torch.ones(T, E, dtype=torch.bool)
            for t in range(T):
                other[t, [int(e) for e in ids[t] if 0 <= e < E]] = False
            assert bool((dx[other] == 0).all())


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_gradient_is_that_of_the_weights(scores, renormalise):
    """Against central differences of the choice's own weights with a step h along a direction of signs: off by h^2 / 6 times the third derivative (of a
    weight: less than 32 times it, its logarithm's derivatives being at most 2, 1.25 and 2) and by the weights' rounding over the step."""
    T, E, K, h = 60, 24, 5, 2.0 ** -8
    kw = dict(scores=scores, renormalise=renormalise)
    f, v = variant(B.route_op(T, E, K, **kw)), variant(B.route_grad_op(T, E, K, **kw))
    if f is None:
        return
    g = rng(9)
    # logits 1/8 apart, so that the choice stays what it is
    x = torch.stack([torch.randperm(E, generator=g) for _ in range(T)]).float() / 8
    u = torch.randint(0, 2, (T, E), generator=g).float() * 2 - 1
    dw = normal(g, T, K)
    shapes = [((T, K), torch.int32), ((T, K), torch.float32)]
    ids, _ = call(f, [dev(x), None], shapes)
    (dx,) = call(v, [dev(x), dev(ids), dev(dw)], [((T, E), torch.float32)])
    sides = []
    for step in (h, -h):
        i, w = call(f, [dev(x + step * u), None], shapes)
        assert torch.equal(i, ids)
        sides.append((w.double() * dw.double()).sum(1))
    slope = (sides[0] - sides[1]) / (2 * h)
    assert bool(((dx.double() * u.double()).sum(1) - slope).abs().le(dw.double().abs().sum(1) * (h * h / 6 * 32 + 45 * 2.0 ** -24 / h)).all())


LEVELS = (300.0, 90.0, 0.0, -60.0, -87.0, -90.0, -95.0, -100.0, -103.0, -110.0, -300.0, -600.0)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("E,K", [(8, 3), (100, 20)])
def test_gradient_of_small_scores_over_their_sum(E, K, kind):
    """Sigmoids that fp32 holds as few bits or none: their parts of the sum are ordinary numbers.  In 64 bits by logarithms, weights = softmax(log sigmoid).
    Tolerances as above: a difference of two logits is off by 2^-24 of itself, d, and so its exponential by less than d e^-d, half a step of the largest."""
    T = 4 * len(LEVELS)
    op = B.route_grad_op(T, E, K, kind, scores="sigmoid", renormalise=True, scale=2.5)
    g = rng(K)
    level = torch.tensor(LEVELS).repeat_interleave(4)[:, None]
    x = normal(g, T, E) + level
    ids = torch.stack([torch.randperm(E, generator=g)[:K] for _ in range(T)]).int()
    for t in range(1, T, 4):  # one ordinary logit among them
        x[t, int(ids[t, 1])] = 0.5
    for t in range(2, T, 4):  # a choice that is none
        ids[t, 0] = -1
    for t in range(3, T, 4):  # the same for all
        x[t] = level[t]
    x = x.to(TYPES[kind])
    dw = normal(g, T, K)
    real = ids >= 0
    of = x.double().requires_grad_(True)
    logs = torch.nn.functional.logsigmoid(of).gather(1, torch.where(real, ids, 0).long())
    w = torch.softmax(torch.where(real, logs, torch.full_like(logs, -INF)), 1)
    (w * dw.double() * 2.5).sum().backward()
    parts, q = (dw.double() * 2.5).abs() * real, w.detach()
    mag = torch.zeros(T, E, dtype=torch.float64).scatter_add_(1, torch.where(real, ids, 0).long(), parts * q + (parts * q).sum(1, keepdim=True) * q)
    assert bool((of.grad.abs().amax(1)[level[:, 0] < 0] > 1e-4).sum() > T // 3)  # no level's gradients vanish
    space = op.space()
    for c in range(space.slots[0].n_candidates):
        if not space.slots[0].weight[c]:
            continue
        v = variant(op, space.slots[0].candidates[c])
        if v is None:
            continue
        (dx,) = call(v, [dev(x), dev(ids), dev(dw)], [((T, E), TYPES[kind])])
        tol = of.grad.abs() * HALF_STEP[kind] * 1.01 + mag * 64 * 2.0 ** -24 + (2.0 ** -25 if kind == "f16" else 1e-37)
        off = ((dx.double() - of.grad).abs() <= tol).all(1)
        assert bool(off.all()), "at logits about %s" % sorted(set(level[~off, 0].tolist()))


@pytest.mark.parametrize("level", [-95.0, -110.0, -600.0])
def test_gradient_of_small_scores_is_that_of_their_weights(level):
    """As test_gradient_is_that_of_the_weights, where fp32 holds no sigmoid: steps of 2^-8 and logits 1/8 apart are exact down to -1024 (2^-13)."""
    T, E, K, h = 60, 24, 5, 2.0 ** -8
    kw = dict(scores="sigmoid", renormalise=True)
    f, v = variant(B.route_op(T, E, K, **kw)), variant(B.route_grad_op(T, E, K, **kw))
    if f is None:
        return
    g = rng(12)
    x = torch.stack([torch.randperm(E, generator=g) for _ in range(T)]).float() / 8 + level
    u = torch.randint(0, 2, (T, E), generator=g).float() * 2 - 1
    dw = normal(g, T, K)
    shapes = [((T, K), torch.int32), ((T, K), torch.float32)]
    ids, _ = call(f, [dev(x), None], shapes)
    (dx,) = call(v, [dev(x), dev(ids), dev(dw)], [((T, E), torch.float32)])
    sides = []
    for step in (h, -h):
        i, w = call(f, [dev(x + step * u), None], shapes)
        assert torch.equal(i, ids)
        sides.append((w.double() * dw.double()).sum(1))
    slope = (sides[0] - sides[1]) / (2 * h)
    assert bool(((dx.double() * u.double()).sum(1) - slope).abs().le(dw.double().abs().sum(1) * (h * h / 6 * 32 + 45 * 2.0 ** -24 / h)).all())


def test_gradient_over_its_logits():
    T, E, K = 90, 40, 4
    v = variant(B.route_grad_op(T, E, K, "bf16"))
    if v is None:
        return
    g = rng(10)
    x, dw = normal(g, T, E).bfloat16(), normal(g, T, K)
    ids = torch.stack([torch.randperm(E, generator=g)[:K] for _ in range(T)]).int()
    (want,) = call(v, [dev(x), dev(ids), dev(dw)], [((T, E), torch.bfloat16)])
    d, i, w = dev(x), dev(ids), dev(dw)
    v.launch([d.data_ptr(), i.data_ptr(), w.data_ptr()], d.data_ptr(), stream=devmem.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(d.cpu(), want)


# ---------------------------------------------------------------- the order of the choices

def order_definition(ids, E):
    flat = ids.reshape(-1).numpy()
    real = (flat >= 0) & (flat < E)
    place = np.full(flat.shape, -1, np.int32)
    place[np.flatnonzero(real)[np.argsort(flat[real], kind="stable")]] = np.arange(int(real.sum()))
    counts = np.bincount(flat[real], minlength=E)
    return offsets_of(counts), torch.from_numpy(place).view(ids.shape)


@pytest.mark.parametrize("E,T,K,code", [(1, 1, 1, 0), (32, 2, 8, 0), (5, 13, 3, 0), (64, 64, 1, 0), (60, 43, 6, 0), (256, 300, 8, 0), (1024, 1000, 1, 0), (65, 1024, 1, 0), (256, 129, 8, 1), (3, 4097, 7, 0),
                                        (256, 16384, 8, 0), (1000, 20011, 3, 0), (17, 300007, 1, 0), (64, 5000, 8, 2), (64, 5000, 8, 4), (300, 5000, 8, 8), (64, 5001, 8, 16), (1024, 40000, 8, 16)])
def test_expert_order(E, T, K, code):
    v = variant(B.expert_order_op(E, T, K), code)
    if v is None:
        return
    g = rng(E + T)
    share = torch.rand(E, generator=g) ** 3 + 1e-3
    for k, ids in enumerate([torch.multinomial(share, T * K, True, generator=g).int().view(T, K), torch.randint(-3, E + 3, (T, K), generator=g).int(), torch.full((T, K), E - 1).int(),
                             torch.full((T, K), -1).int(), torch.arange(T * K).flip(0).remainder(E).int().view(T, K), torch.randint(-2 ** 31, 2 ** 31, (T, K), generator=g).int()]):
        offsets, place = call(v, [dev(ids)], [((E + 1,), torch.int32), ((T, K), torch.int32)])
        want, places = order_definition(ids, E)
        assert torch.equal(offsets, want) and torch.equal(place, places), k


@pytest.mark.parametrize("E", [1, 64, 256, 1024])
@pytest.mark.parametrize("T,K", [(65, 1), (20, 8), (32, 8), (257, 1)])
def test_order_of_a_few_wavefronts(T, K, E):
    """A decoding batch: workgroups of one, four and sixteen wavefronts, and the counts at which they change."""
    v = variant(B.expert_order_op(E, T, K))
    if v is None:
        return
    g = rng(T + E)
    for ids in (torch.randint(0, E, (T, K), generator=g).int(), torch.randint(-2, E + 2, (T, K), generator=g).int(), torch.full((T, K), E - 1).int()):
        offsets, place = call(v, [dev(ids)], [((E + 1,), torch.int32), ((T, K), torch.int32)])
        want, places = order_definition(ids, E)
        assert torch.equal(offsets, want) and torch.equal(place, places)


@pytest.mark.parametrize("E,T,K", [(1024, 1050001, 8), (256, 1 << 22, 3), (7, 1 << 21, 32)])
def test_order_of_millions_of_choices(E, T, K):
    """Up to the most that there may be, MS_MAX_CHOICES; the definition by a stable sort on the GPU."""
    v = variant(B.expert_order_op(E, T, K))
    if v is None:
        return
    n = T * K
    ids = torch.randint(0, E, (n,), generator=rng(E)).int().cuda()
    ids[::1001] = -1
    offsets, place = torch.full((E + 1,), 7, dtype=torch.int32, device="cuda"), torch.full((n,), 7, dtype=torch.int32, device="cuda")
    ws = torch.full((v.workspace_bytes(),), 0x55, dtype=torch.uint8, device="cuda")
    v.launch([ids.data_ptr()], [offsets.data_ptr(), place.data_ptr()], stream=devmem.current_stream(), workspace=ws.data_ptr())
    key = torch.where(ids < 0, torch.full_like(ids, E), ids).short()
    order = key.sort(stable=True)[1]
    counts = torch.bincount(key.int(), minlength=E + 1)[:E]
    real = int(counts.sum())
    want = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    want[order[:real]] = torch.arange(real, dtype=torch.int32, device="cuda")
    assert torch.equal(place, want) and int(offsets[0]) == 0 and torch.equal(offsets[1:].long(), counts.cumsum(0))


def test_order_of_several_instances():
    for E, T, K in ((7, 9, 2), (70, 3000, 4)):
        R = 3
        v = variant(B.expert_order_op(E, T, K))
        if v is None:
            continue
        ids = torch.randint(-1, E, (R, T, K), generator=rng(T)).int()
        offsets, place = call(v, [dev(ids)], [((R, E + 1), torch.int32), ((R, T, K), torch.int32)], instances=R)
        for r in range(R):
            want, places = order_definition(ids[r], E)
            assert torch.equal(offsets[r], want) and torch.equal(place[r], places)


# ---------------------------------------------------------------- rows to their choices and back

def places_of(g, T, K, P, none=0.2):
    """Different rows for the choices there are, numbers outside of the rows for the others."""
    place = torch.randperm(max(P, T * K), generator=g)[:T * K].int().view(T, K)
    place[torch.rand(T, K, generator=g) < none] = -1
    place[place >= P] = P + 5
    if T > 3:
        place[1] = -7
    return place


ROWS = [(1, 1, 1, 1, 0), (1, 8, 4096, 8, 0), (5, 3, 129, 20, 0), (33, 8, 64, 264, 1), (7, 64, 200, 448, 2), (12, 6, 2050, 72, 0), (9, 2, 2056, 10, 4), (3, 5, 9001, 15, 2), (300, 2, 24, 700, 0), (2, 4, 20000, 8, 16),
        (40, 1, 520, 50, 8), (6, 7, 1033, 42, 1)]


@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("bf16", "i8"), ("f32", "i8"), ("f16", "f8"), ("f32", "f8"), ("i8", "i8"), ("f8", "f8")])
@pytest.mark.parametrize("which", range(len(ROWS)))
def test_rows_to_their_choices(which, kind, out):
    T, K, N, P, code = ROWS[which]
    v = variant(B.spread_rows_op(T, K, N, P, kind, out), code)
    if v is None:
        return
    g = rng(which)
    place = places_of(g, T, K, P)
    blocks = {"i8": 1, "f8": -(-N // 128)}.get(out, 0)
    x = normal(g, T, N, scale=3.0)
    x[0, :64] = 0
    sx = torch.rand(T, blocks, generator=g) if kind in ("i8", "f8") else None
    if kind == "i8":
        x = torch.randint(-128, 128, (T, N), generator=g)
    x = x.to(TYPES[kind])
    a, s = call(v, [dev(x), dev(place), dev(sx)], [((P, N), TYPES[out]), ((P, blocks), torch.float32) if blocks else None])
    check_spread(a, s, x, place, sx, out, blocks)


def check_spread(a, s, x, place, sx, out, blocks):
    """Copies and fp32 quotients: the same."""
    T, N = x.shape
    if sx is not None or blocks == 0:
        q, scale = x, sx
    else:
        f = x.float()
        if out == "i8":
            scale = (f.abs().amax(1, keepdim=True) * PART).clamp_min(2.0 ** -126)
            q = (f / scale).round().to(torch.int8)
        else:
            pad = torch.nn.functional.pad(f, (0, blocks * 128 - N)).view(T, blocks, 128)
            scale = (pad.abs().amax(-1) / 448).clamp_min(2.0 ** -126)
            q = (pad / scale[..., None]).to(TYPES["f8"]).view(T, -1)[:, :N]
    left = torch.ones(a.shape[0], dtype=torch.bool)
    bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    for t in range(T):
        for p in place[t].tolist():
            if 0 <= p < a.shape[0]:
                left[p] = False
                assert torch.equal(a[p].view(bits), q[t].contiguous().view(bits)), (t, p)
                if blocks:
                    assert torch.equal(s[p], scale[t]), (t, p)
    assert bool((a[left].float() == 7).all()) and (not blocks or bool((s[left] == 7).all())), "rows that no place names were written"


def test_rows_quantised_where_they_are():
    """One choice of each token and no places: the row is the token's.  Ties of the rounding, zeros, NaN, infinities, small and large rows."""
    T, N = 12, 300
    for kind in ("f32", "bf16"):
        v, f8 = variant(B.spread_rows_op(T, 1, N, T + 2, kind, "i8")), variant(B.spread_rows_op(T, 1, N, T, kind, "f8"))
        copy = variant(B.spread_rows_op(T, 1, N, T, kind))
        if v is None:
            continue
        g = rng(3)
        x = normal(g, T, N)
        x[0] = 0
        x[1] = torch.randint(-254, 255, (N,), generator=g).float() / 2  # halves
        x[1, 0] = 127
        x[2] *= 1e-38
        x[3] *= 1e-45
        x[4] *= 1e37
        x[5, 1:] = 0
        x[8, 7] = INF
        x[9, 8] = NAN
        x = x.to(TYPES[kind])
        a, s = call(v, [dev(x), None, None], [((T + 2, N), torch.int8), ((T + 2, 1), torch.float32)])
        fine = [t for t in range(T) if t not in (8, 9)]
        f = x.float()
        scale = (f.abs().amax(1, keepdim=True) * PART).clamp_min(2.0 ** -126)
        assert torch.equal(s[:T][fine], scale[fine]) and torch.equal(a[:T][fine], (f / scale).round().to(torch.int8)[fine])
        assert bool((a[0] == 0).all()) and float(s[0]) == 2.0 ** -126 and bool((a[T:] == 7).all())
        assert float(s[8]) == INF and bool((a[8] == 0).all()) and bool(torch.isnan(s[9]).all())
        a, s = call(f8, [dev(x), None, None], [((T, N), TYPES["f8"]), ((T, 3), torch.float32)])
        pad = torch.nn.functional.pad(f, (0, 84)).view(T, 3, 128)
        scale = (pad.abs().amax(-1) / 448).clamp_min(2.0 ** -126)
        want = (pad / scale[..., None]).to(TYPES["f8"]).view(T, -1)[:, :N]
        assert torch.equal(s[fine], scale[fine]) and torch.equal(a[fine].view(torch.uint8), want[fine].view(torch.uint8))
        assert bool(torch.isnan(s[9, 0])) and bool(torch.isnan(a[9, :128].float()).all()) and torch.equal(a[9, 128:].view(torch.uint8), want[9, 128:].contiguous().view(torch.uint8))
        (a, _) = call(copy, [dev(x), None, None], [((T, N), TYPES[kind]), None])
        assert torch.equal(a.view(torch.uint8), x.view(torch.uint8))


def join_definition(c, place, w, r):
    """And the magnitudes that are added up."""
    T, K = place.shape
    y = r.double().clone() if r is not None else torch.zeros(T, c.shape[1], dtype=torch.float64)
    mag = y.abs()
    for t in range(T):
        for j in range(K):
            p = int(place[t, j])
            if 0 <= p < c.shape[0]:
                part = c[p].double() * (float(w[t, j]) if w is not None else 1)
                y[t] += part
                mag[t] += part.abs()
    return y, mag


@pytest.mark.parametrize("kind,out,weights,residual", [("bf16", "bf16", True, False), ("bf16", "f32", True, True), ("f16", "f16", True, True), ("f32", "f32", True, False), ("f16", "f32", False, False),
                                                       ("bf16", "bf16", False, True)])
@pytest.mark.parametrize("which", range(len(ROWS)))
def test_rows_back(which, kind, out, weights, residual):
    """K fused products in fp32: half a step of the magnitudes each; and the one rounding."""
    T, K, N, P, code = ROWS[which]
    v = variant(B.join_rows_op(T, K, N, P, kind, out, weights=weights, residual=residual), code)
    if v is None:
        return
    g = rng(which + 50)
    place = places_of(g, T, K, P)
    c, w, r = normal(g, P, N).to(TYPES[kind]), normal(g, T, K) if weights else None, normal(g, T, N).to(TYPES[out]) if residual else None
    unused = torch.ones(P, dtype=torch.bool)
    unused[[int(p) for p in place.reshape(-1) if 0 <= p < P]] = False
    c[unused] = NAN  # rows of no choice add nothing
    if weights:
        w[(place < 0) | (place >= P)] = NAN
    (y,) = call(v, [dev(c), dev(place), dev(w), dev(r)], [((T, N), TYPES[out])])
    want, mag = join_definition(c, place, w, r)
    tol = mag * (K + 1) * 2.0 ** -24 + want.abs() * (HALF_STEP[out] if out != "f32" else 0) * 1.01 + (2.0 ** -25 if out == "f16" else 1e-37)
    assert bool(((y.double() - want).abs() <= tol).all())
    if residual:  # R may be Y
        d, dp, dw, dr = dev(c), dev(place), dev(w), dev(r)
        v.launch([d.data_ptr(), dp.data_ptr(), dw.data_ptr() if weights else None, dr.data_ptr()], dr.data_ptr(), stream=devmem.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(dr.cpu(), y)


def test_infinities_and_nan_of_rows_come_through():
    T, K, N = 4, 3, 40
    v = variant(B.join_rows_op(T, K, N, T * K, "f32"))
    if v is None:
        return
    c, w = torch.ones(T * K, N), torch.ones(T, K)
    c[0, 5], c[1, 5], c[3, 6], c[4, 6], c[6, 7], w[3, 1] = INF, 1, INF, -INF, NAN, 0
    place = torch.arange(T * K).int().view(T, K)
    place[0, 2] = -1
    (y,) = call(v, [dev(c), dev(place), dev(w), None], [((T, N), torch.float32)])
    want, _ = join_definition(c, place, w, None)
    fine = ~torch.isnan(want)
    assert torch.equal(torch.isnan(y), ~fine) and torch.equal(y.double()[fine], want[fine])
    assert float(y[0, 5]) == INF and bool(torch.isnan(y[1, 6])) and bool(torch.isnan(y[2, 7])) and float(y[3, 0]) == 2 and float(y[0, 0]) == 2


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("which", range(len(ROWS)))
def test_gradients_of_rows_back(which, kind):
    """The rows' gradient is one fp32 product, rounded; the weights' a sum of N products in fp32, off by less than half a step of the magnitudes each:
    8 of a chunk after each other, the chunks of a lane, and 6 steps over the lanes."""
    T, K, N, P, code = ROWS[which]
    v = variant(B.join_grad_op(T, K, N, P, kind), code)
    if v is None:
        return
    g = rng(which + 70)
    place = places_of(g, T, K, P)
    dy, w, c = normal(g, T, N).to(TYPES[kind]), normal(g, T, K), normal(g, P, N).to(TYPES[kind])
    real = (place >= 0) & (place < P)
    unused = torch.ones(P, dtype=torch.bool)
    unused[place[real].long()] = False
    c[unused] = NAN
    w[~real] = NAN
    dc, dw = call(v, [dev(dy), dev(place), dev(w), dev(c)], [((P, N), TYPES[kind]), ((T, K), torch.float32)])
    assert bool((dc[unused].float() == 7).all()) and bool((dw[~real] == 0).all())
    for t in range(T):
        for j in range(K):
            if real[t, j]:
                p = int(place[t, j])
                want = dy[t].double() * float(w[t, j])
                assert bool(((dc[p].double() - want).abs() <= want.abs() * (HALF_STEP[kind] + 2.0 ** -24) * 1.01 + (2.0 ** -25 if kind == "f16" else 1e-37)).all())
                products = dy[t].double() * c[p].double()
                assert abs(float(dw[t, j]) - float(products.sum())) <= float(products.abs().sum()) * (N / 64 + 32) * 2.0 ** -24


def test_gradients_of_rows_back_are_those_of_its_sums():
    """loss = sum(Y G) is linear in C and in W: the central difference is the derivative; multiples of 1/8, whose sums are exact in fp32."""
    T, K, N, P = 11, 4, 72, 50
    f, v = variant(B.join_rows_op(T, K, N, P, "f32")), variant(B.join_grad_op(T, K, N, P, "f32"))
    if f is None:
        return
    g = rng(12)

    def grid(*shape):
        return torch.randint(-8, 9, shape, generator=g).float() / 8

    place = places_of(g, T, K, P)
    c, w, G, uc, uw = grid(P, N), grid(T, K), grid(T, N), grid(P, N), grid(T, K)
    dc, dw = call(v, [dev(G), dev(place), dev(w), dev(c)], [((P, N), torch.float32), ((T, K), torch.float32)])
    dc[~torch.isin(torch.arange(P), place.long())] = 0  # rows that no place names were left as they were

    def loss(c, w):
        (y,) = call(f, [dev(c), dev(place), dev(w), None], [((T, N), torch.float32)])
        return float((y.double() * G.double()).sum())

    h = 0.125
    assert abs((loss(c + h * uc, w) - loss(c - h * uc, w)) / (2 * h) - float((dc.double() * uc.double()).sum())) < 1e-6
    assert abs((loss(c, w + h * uw) - loss(c, w - h * uw)) / (2 * h) - float((dw.double() * uw.double()).sum())) < 1e-6


def test_rows_strides_and_instances():
    R, T, K, N, P = 2, 9, 3, 100, 30
    ops = [B.spread_rows_op(T, K, N, P, "bf16", "i8", a_strides=[0, 117, 1]), B.join_rows_op(T, K, N, P, "bf16", a_strides=[0, 131, 1]),
           B.join_grad_op(T, K, N, P, "bf16", a_strides=[0, 117, 1], b_strides=[0, 131, 1])]
    out, back, grad = [variant(o) for o in ops]
    if out is None:
        return
    g = rng(15)
    place = torch.stack([places_of(g, T, K, P) for _ in range(R)])
    x, c, w = normal(g, R, T, N).bfloat16(), normal(g, R, P, N).bfloat16(), normal(g, R, T, K)
    c[:] = torch.where(torch.isnan(c), torch.zeros_like(c), c)

    def spread_out(values, op, idx, stride):  # copies whose rows lie `stride` apart and start off 16-byte boundaries
        span = op.tensor_bytes(idx) // 2
        flat = torch.full((1 + R * span,), NAN, dtype=torch.bfloat16)
        for r in range(R):
            torch.as_strided(flat, values.shape[1:], (stride, 1), 1 + r * span).copy_(values[r])
        return dev(flat)[1:]

    px, pc = spread_out(x, ops[0], 0, 117), spread_out(c, ops[1], 0, 131)
    a, s = call(out, [px, dev(place), None], [((R, P, N), torch.int8), ((R, P, 1), torch.float32)], instances=R)
    (y,) = call(back, [pc, dev(place), dev(w), None], [((R, T, N), torch.bfloat16)], instances=R)
    dc, dw = call(grad, [px, dev(place), dev(w), pc], [((R, P, N), torch.bfloat16), ((R, T, K), torch.float32)], instances=R)
    for r in range(R):
        check_spread(a[r], s[r], x[r], place[r], None, "i8", 1)
        want, mag = join_definition(c[r], place[r], w[r], None)
        assert bool(((y[r].double() - want).abs() <= mag * (K + 1) * 2.0 ** -24 + want.abs() * 2.0 ** -8 * 1.01).all())
        for t in range(T):
            for j in range(K):
                p = int(place[r, t, j])
                if 0 <= p < P:
                    products = x[r, t].double() * c[r, p].double()
                    assert abs(float(dw[r, t, j]) - float(products.sum())) <= float(products.abs().sum()) * 40 * 2.0 ** -24
                    want = x[r, t].double() * float(w[r, t, j])
                    assert bool(((dc[r, p].double() - want).abs() <= want.abs() * 2.0 ** -8 * 1.01).all())


@pytest.mark.parametrize("N", [1, 3, 7, 8, 9, 511, 513])
def test_rows_of_few_columns_and_ends(N):
    """Rows shorter than a lane's eight columns, and just beside; rows in place of the residual, whose ends two lanes share."""
    T, K, P = 13, 3, 39
    for kind in ("bf16", "f32"):
        ops = [variant(o) for o in (B.spread_rows_op(T, K, N, P, kind), B.spread_rows_op(T, K, N, P, kind, "i8"), B.spread_rows_op(T, K, N, P, kind, "f8"), B.join_rows_op(T, K, N, P, kind, residual=True),
                                    B.join_rows_op(T, K, N, P, kind), B.join_grad_op(T, K, N, P, kind))]
        if ops[0] is None:
            continue
        g = rng(N)
        place = places_of(g, T, K, P)
        x, c, w, r = normal(g, T, N).to(TYPES[kind]), normal(g, P, N).to(TYPES[kind]), normal(g, T, K), normal(g, T, N).to(TYPES[kind])
        blocks = -(-N // 128)
        (a, _) = call(ops[0], [dev(x), dev(place), None], [((P, N), TYPES[kind]), None])
        check_spread(a, None, x, place, None, kind, 0)
        a, s = call(ops[1], [dev(x), dev(place), None], [((P, N), torch.int8), ((P, 1), torch.float32)])
        check_spread(a, s, x, place, None, "i8", 1)
        a, s = call(ops[2], [dev(x), dev(place), None], [((P, N), TYPES["f8"]), ((P, blocks), torch.float32)])
        check_spread(a, s, x, place, None, "f8", blocks)
        for v, res in ((ops[3], r), (ops[4], None)):
            (y,) = call(v, [dev(c), dev(place), dev(w), dev(res)], [((T, N), TYPES[kind])])
            want, mag = join_definition(c, place, w, res)
            assert bool(((y.double() - want).abs() <= mag * (K + 1) * 2.0 ** -24 + want.abs() * (HALF_STEP[kind] if kind != "f32" else 0) * 1.01 + 1e-37).all())
            if res is not None:
                d, dp, dw, dr = dev(c), dev(place), dev(w), dev(res)
                v.launch([d.data_ptr(), dp.data_ptr(), dw.data_ptr(), dr.data_ptr()], dr.data_ptr(), stream=devmem.current_stream())
                torch.cuda.synchronize()
                assert torch.equal(dr.cpu(), y)
        dc, dw = call(ops[5], [dev(x), dev(place), dev(w), dev(c)], [((P, N), TYPES[kind]), ((T, K), torch.float32)])
        for t in range(T):
            for j in range(K):
                p = int(place[t, j])
                if 0 <= p < P:
                    products = x[t].double() * c[p].double()
                    assert abs(float(dw[t, j]) - float(products.sum())) <= float(products.abs().sum()) * (N / 64 + 32) * 2.0 ** -24
                    want = x[t].double() * float(w[t, j])
                    assert bool(((dc[p].double() - want).abs() <= want.abs() * HALF_STEP[kind] * 1.01).all())
                else:
                    assert float(dw[t, j]) == 0


def test_infinities_at_the_shared_end_of_a_row():
    """What two lanes hold of a row's end counts once: an infinity stays one."""
    T, N = 2, 1003
    v = variant(B.join_grad_op(T, 1, N, T, "f32"))
    if v is None:
        return
    dy, c, w = torch.ones(T, N), torch.ones(T, N), torch.ones(T, 1)
    c[0, N - 6], c[1, N - 1] = INF, -INF
    place = torch.arange(T).int().view(T, 1)
    dc, dw = call(v, [dev(dy), dev(place), dev(w), dev(c)], [((T, N), torch.float32), ((T, 1), torch.float32)])
    assert dw.reshape(-1).tolist() == [INF, -INF] and bool((dc == 1).all())


def test_rows_beyond_4_gib():
    """Places behind the first 4 GiB of rows, of tokens behind theirs."""
    T, K, N = 330000, 1, 8192
    ops = [variant(B.spread_rows_op(T, K, N, T, "bf16")), variant(B.join_rows_op(T, K, N, T, "bf16")), variant(B.join_grad_op(T, K, N, T, "bf16"))]
    if ops[0] is None:
        return
    place = torch.full((T, K), -1, dtype=torch.int32)
    place[-3:, 0] = torch.tensor([T - 1, 5, T - 2])
    place[4, 0] = T - 3
    x = torch.zeros(T, N, dtype=torch.bfloat16, device="cuda")
    some = normal(rng(2), 4, N).bfloat16()
    tokens = [T - 3, T - 2, T - 1, 4]
    for t, row in zip(tokens, some):
        x[t] = dev(row)
    a = torch.zeros(T, N, dtype=torch.bfloat16, device="cuda")
    p, w = dev(place), torch.full((T, K), 2.0, device="cuda")
    at = devmem.current_stream()
    ops[0].launch([x.data_ptr(), p.data_ptr(), None], [a.data_ptr(), None], stream=at)
    torch.cuda.synchronize()
    for t, row in zip(tokens, some):
        assert torch.equal(a[int(place[t, 0])].cpu(), row)
    assert int((a[6:-3] != 0).sum()) == 0
    y = torch.empty_like(x)
    ops[1].launch([a.data_ptr(), p.data_ptr(), w.data_ptr(), None], y.data_ptr(), stream=at)
    torch.cuda.synchronize()
    for t, row in zip(tokens, some):
        assert torch.equal(y[t].cpu(), row * 2)
    y.zero_()
    dw = torch.empty(T, K, device="cuda")
    ops[2].launch([x.data_ptr(), p.data_ptr(), w.data_ptr(), a.data_ptr()], [y.data_ptr(), dw.data_ptr()], stream=at)
    torch.cuda.synchronize()
    for t, row in zip(tokens, some):
        assert torch.equal(y[int(place[t, 0])].cpu(), row * 2)
        want = float(row.double().square().sum())
        assert abs(float(dw[t, 0]) - want) <= want * (N / 64 + 32) * 2.0 ** -24
    assert int((dw != 0).sum()) == 4


# ---------------------------------------------------------------- together, and the ways of calling

class Layer:
    """A layer of experts with one matrix each: route, order, rows out, product by expert, rows back; and the way back."""

    def __init__(self, T, E, K, F, N, kind):
        P = T * K
        self.sizes = (T, E, K, F, N)
        self.kind = kind
        make = {"route": B.route_op(T, E, K, "f32", scores="sigmoid", bias=True, groups=4, kept=2, best=2, renormalise=True, scale=2.5), "order": B.expert_order_op(E, T, K),
                "out": B.spread_rows_op(T, K, F, P, "bf16", kind), "product": B.grouped_gemm_op(E, P, N, F, True, kind, "bf16"), "back": B.join_rows_op(T, K, N, P, residual=True),
                "back_grad": B.join_grad_op(T, K, N, P), "input_grad": B.grouped_gemm_op(E, P, F, N, False, "bf16"), "weight_grad": B.grouped_wgrad_op(E, P, N, F, "bf16", "f32"),
                "out_grad": B.join_rows_op(T, K, F, P, "bf16", "f32", weights=False), "route_grad": B.route_grad_op(T, E, K, "f32", scores="sigmoid", renormalise=True, scale=2.5)}
        if kind != "bf16":
            make = {k: make[k] for k in ("route", "order", "out", "product", "back")}
        self.ops = {k: variant(o) for k, o in make.items()}

    def buffers(self):
        T, E, K, F, N = self.sizes
        P, e = T * K, lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
        f32, i32 = torch.float32, torch.int32
        return dict(ids=e(T, K, t=i32), w=e(T, K, t=f32), offsets=e(E + 1, t=i32), place=e(T, K, t=i32), a=e(P, F, t=TYPES[self.kind]), sa=e(P, t=f32), c=e(P, N), y=e(T, N), dc=e(P, N), dw=e(T, K, t=f32),
                    da=e(P, F), dm=e(E, N, F, t=f32), dx=e(T, F, t=f32), dl=e(T, E, t=f32), ws=e(max(1, self.ops["order"].workspace_bytes()), t=torch.uint8))

    def forward(self, i, o, static=False):
        def go(name, ins, outs):
            ins, outs = ([t.data_ptr() if t is not None else None for t in ts] for ts in (ins, outs))
            if static:
                self.ops[name].launch_static(ins, outs, stream=devmem.current_stream())
            else:
                self.ops[name].launch(ins, outs, stream=devmem.current_stream(), workspace=o["ws"].data_ptr())
        self.go = go
        go("route", [i["logits"], i["bias"]], [o["ids"], o["w"]])
        go("order", [o["ids"]], [o["offsets"], o["place"]])
        scaled = self.kind != "bf16"
        go("out", [i["x"], o["place"], None], [o["a"], o["sa"] if scaled else None])
        go("product", [o["a"], i["m"], o["offsets"]] + ([o["sa"], i["sm"]] if scaled else []), [o["c"]])
        go("back", [o["c"], o["place"], o["w"], i["r"]], [o["y"]])

    def backward(self, i, o):
        go = self.go
        go("back_grad", [i["dy"], o["place"], o["w"], o["c"]], [o["dc"], o["dw"]])
        go("input_grad", [o["dc"], i["m"], o["offsets"]], [o["da"]])
        go("weight_grad", [o["dc"], o["a"], o["offsets"]], [o["dm"]])
        go("out_grad", [o["da"], o["place"], None, None], [o["dx"]])
        go("route_grad", [i["logits"], o["ids"], o["dw"]], [o["dl"]])

    def inputs(self, g, masked=0):
        T, E, K, F, N = self.sizes
        i = dict(logits=normal(g, T, E, scale=1.5), bias=normal(g, E, scale=0.1), x=normal(g, T, F).bfloat16(), m=normal(g, E, N, F, scale=0.3), r=normal(g, T, N).bfloat16(), dy=normal(g, T, N).bfloat16())
        if masked:
            i["logits"][-masked:] = -INF
        if self.kind == "i8":
            i["sm"] = i["m"].abs().amax(-1) / 127
            i["m"] = (i["m"] / i["sm"][..., None]).round().to(torch.int8)
        else:
            i["m"] = i["m"].bfloat16()
        return i


def test_a_layer_of_experts_forward_and_backward():
    """All operators of a training step, each held to what its own inputs say, on another stream than the current one."""
    T, E, K, F, N = 150, 16, 3, 96, 136
    layer = Layer(T, E, K, F, N, "bf16")
    if layer.ops["route"] is None:
        return
    i = layer.inputs(rng(1), masked=7)
    d, o = {k: dev(t) for k, t in i.items()}, layer.buffers()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer.forward(d, o)
        layer.backward(d, o)
    stream.synchronize()
    o = {k: t.cpu() for k, t in o.items()}
    ids, w = route_definition(i["logits"], i["bias"], K, scores="sigmoid", groups=4, kept=2, best=2, renormalise=True, scale=2.5)
    assert torch.equal(o["ids"], ids) and bool(((o["w"].double() - w).abs() <= w * 1.01 * 2.0 ** -24).all())
    # the layer as one function in 64 bits of what it was given, rows rounded where the operators round them
    x, m, w = i["x"].double().requires_grad_(True), i["m"].double().requires_grad_(True), o["w"].double().requires_grad_(True)
    y = i["r"].double()
    mag = y.abs()
    for j in range(K):
        real = ids[:, j] >= 0
        rows = torch.zeros(T, N, dtype=torch.float64)
        rows[real] = torch.bmm(m[ids[real, j].long()], x[real][..., None])[..., 0]
        y = y + w[:, j:j + 1] * rows
        mag = mag + (w[:, j:j + 1] * rows).abs().detach()
    # rows are rounded to bf16 ahead of their sum, the sum once more
    assert bool(((o["y"].double() - y.detach()).abs() <= mag * 2.0 ** -8 * 1.05 + y.detach().abs() * 2.0 ** -8 * 1.05).all())
    (y * i["dy"].double()).sum().backward()
    for got, want in ((o["dx"], x.grad), (o["dm"], m.grad), (o["dw"], w.grad)):
        # sums of rows rounded to bf16 once or twice on the way: 2^-8 each of their largest
        assert float((got.double() - want).norm() / want.norm()) < 2.0 ** -7
    want, mag = grad_definition(i["logits"], ids, o["dw"], "sigmoid", True, 2.5)
    want[-7:] = 0
    assert bool(((o["dl"].double() - want).abs() <= mag * 64 * 2.0 ** -24 + 1e-37).all()) and bool((o["dx"][-7:] == 0).all()) and torch.equal(o["y"][-7:], i["r"][-7:])


def test_a_layer_of_experts_in_8_bit_integers():
    T, E, K, F, N = 70, 12, 4, 160, 72
    layer = Layer(T, E, K, F, N, "i8")
    if layer.ops["route"] is None:
        return
    i = layer.inputs(rng(2), masked=3)
    d, o = {k: dev(t) for k, t in i.items()}, layer.buffers()
    layer.forward(d, o)
    torch.cuda.synchronize()
    o = {k: t.cpu() for k, t in o.items()}
    s = i["x"].float().abs().amax(1, keepdim=True) * PART
    q = (i["x"].float() / s).round().double() * s.double()
    y, mag = i["r"].double(), i["r"].double().abs()
    for j in range(K):
        real = o["ids"][:, j] >= 0
        e = o["ids"][real, j].long()
        rows = torch.bmm(i["m"][e].double() * i["sm"][e].double()[..., None], q[real][..., None])[..., 0]
        y[real] += o["w"][real, j:j + 1].double() * rows
        mag[real] += (o["w"][real, j:j + 1].double() * rows).abs()
    assert bool(((o["y"].double() - y).abs() <= (mag + y.abs()) * 2.0 ** -8 * 1.05).all())


def test_captured_layer_follows_its_inputs():
    """Forward and backward in one graph, replayed with other logits and rows and the program's own eager run in between; the order needs its workspace."""
    T, E, K, F, N = 2200, 16, 2, 64, 72
    layer = Layer(T, E, K, F, N, "bf16")
    if layer.ops["route"] is None:
        return
    assert layer.ops["order"].workspace_bytes() > 0
    for v in layer.ops.values():
        v.prepare()
    g = rng(3)
    d, o = {k: dev(t) for k, t in layer.inputs(g).items()}, layer.buffers()

    def step():
        layer.forward(d, o, static=True)
        layer.backward(d, o)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    names = [n for n in o if n != "ws"]
    for masked in (0, 2199, 2200, 50):
        for k, t in layer.inputs(g, masked).items():
            d[k].copy_(t)
        got = []
        for run in (graph.replay, step):
            for n in names:
                o[n].fill_(3)
            run()
            torch.cuda.synchronize()
            got.append([o[n].cpu().clone() for n in names])
        assert all(torch.equal(p.contiguous().view(torch.uint8), q.contiguous().view(torch.uint8)) for p, q in zip(*got)), masked
        rows = (T - masked) * K
        assert int(got[0][names.index("offsets")][-1]) == rows and bool((got[0][names.index("a")][rows:].float() == 3).all())


def test_two_streams_at_once():
    """Each with a workspace of its own."""
    E, T, K, N = 64, 3000, 4, 264
    order, out = variant(B.expert_order_op(E, T, K)), variant(B.spread_rows_op(T, K, N, T * K, "bf16", "i8"))
    if order is None:
        return
    g = rng(7)
    sets = [(torch.randint(-1, E, (T, K), generator=g).int().cuda(), normal(g, T, N).bfloat16().cuda()) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in sets]
    bufs = [[torch.zeros(E + 1, dtype=torch.int32, device="cuda"), torch.zeros(T, K, dtype=torch.int32, device="cuda"), torch.zeros(T * K, N, dtype=torch.int8, device="cuda"),
             torch.zeros(T * K, device="cuda"), torch.zeros(order.workspace_bytes(), dtype=torch.uint8, device="cuda")] for _ in sets]
    torch.cuda.synchronize()
    for _ in range(10):
        for (ids, x), st, b in zip(sets, streams, bufs):
            order.launch([ids.data_ptr()], [b[0].data_ptr(), b[1].data_ptr()], stream=st.cuda_stream, workspace=b[4].data_ptr())
            out.launch([x.data_ptr(), b[1].data_ptr(), None], [b[2].data_ptr(), b[3].data_ptr()], stream=st.cuda_stream)
    torch.cuda.synchronize()
    for (ids, x), b in zip(sets, bufs):
        offsets, place = order_definition(ids.cpu(), E)
        assert torch.equal(b[0].cpu(), offsets) and torch.equal(b[1].cpu(), place)
        f = x.float().cpu()
        q = (f / (f.abs().amax(1, keepdim=True) * PART)).round().to(torch.int8)
        t, j = torch.nonzero(place >= 0, as_tuple=True)
        assert torch.equal(b[2].cpu()[place[t, j].long()], q[t])


def test_measure_and_search():
    """Both outputs lie in one block; an order that needs a workspace gets it from the buffer set."""
    up = lambda x: -(-x // 256) * 256  # noqa: E731
    g = rng(11)
    ids = torch.randint(0, 40, (3000, 2), generator=g).int()
    for op, ins in ((B.route_op(100, 40, 4, bias=True), [normal(g, 100, 40), normal(g, 40)]), (B.expert_order_op(40, 3000, 2), [ids]),
                    (B.spread_rows_op(10, 2, 300, 20, "bf16", "f8"), [normal(g, 10, 300).bfloat16(), torch.arange(20).int()]),
                    (B.join_grad_op(10, 2, 300, 20), [normal(g, 10, 300).bfloat16(), torch.arange(20).int(), normal(g, 10, 2), normal(g, 20, 300).bfloat16()])):
        v = variant(op)
        if v is None:
            continue
        ins = [dev(t) for t in ins]
        sizes = [op.tensor_bytes(-1), op.tensor_bytes(-2)]
        block, ws = torch.zeros(up(sizes[0]) + sizes[1], dtype=torch.uint8, device="cuda"), torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
        want = [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in sizes]
        pointers = [t.data_ptr() for t in ins]
        v.launch(pointers + [None] * (4 - len(pointers)), [t.data_ptr() for t in want], stream=devmem.current_stream(), workspace=ws.data_ptr())
        m = v.measure([(pointers, block.data_ptr(), ws.data_ptr())], stream=devmem.current_stream())
        assert 0 < m.min_us < 1e5
        cfg = B.search_cfg_default()
        cfg.trials, cfg.init_population = 3, 3
        res = B.search(op, op.space(), cfg, [(pointers, block.data_ptr(), ws.data_ptr())], stream=devmem.current_stream())
        torch.cuda.synchronize()
        assert res.n_measured >= 2 and res.n_failed == 0
        assert torch.equal(block[:sizes[0]], want[0])
        if op.desc().kind != B.OP_JOIN_GRAD:  # sums in another order under another number of wavefronts
            assert torch.equal(block[up(sizes[0]):], want[1])
