"""Routing to experts on the host: what is accepted and refused, coverage, tensors, workspaces, launches' checks.  No GPU."""
import os
import subprocess

import numpy as np
import pytest

from paper_2205_13603_amd import binding as B, devmem, tuned

OPS = {
    "route": lambda: B.route_op(37, 60, 6, "bf16"),
    "route by groups": lambda: B.route_op(300, 256, 8, scores="sigmoid", bias=True, groups=8, kept=4, best=2, renormalise=True, scale=2.5),
    "route of many": lambda: B.route_op(9, 1000, 32, "f16", bias=True),
    "route gradient": lambda: B.route_grad_op(70, 130, 5, "bf16"),
    "order": lambda: B.expert_order_op(60, 7, 5),
    "order in runs": lambda: B.expert_order_op(300, 5000, 8),
    "out": lambda: B.spread_rows_op(13, 3, 1030, 39, "bf16", "i8"),
    "out f8": lambda: B.spread_rows_op(13, 3, 130, 39, "f32", "f8"),
    "copy": lambda: B.spread_rows_op(13, 3, 130, 39, "f8"),
    "back": lambda: B.join_rows_op(13, 3, 1030, 39, "bf16", "f32", residual=True),
    "back gradient": lambda: B.join_grad_op(13, 3, 1030, 39, "f16"),
}


def refused(code, f, *args, **kw):
    with pytest.raises(B.MsError) as e:
        f(*args, **kw)
    assert e.value.code == code, str(e.value)


def variant(op, code=0):
    space = op.space()
    return B.Variant(op, space, B.make_trace(space, [[code]]))


@pytest.mark.parametrize("name", sorted(OPS))
def test_every_block_covers_outputs_and_reduction_once(name):
    op = OPS[name]()
    space = op.space()
    assert space.family == B.FAM_ROUTING and space.n_slots == 1 and space.slots[0].slot_id == B.SLOT_BLOCK and space.slots[0].candidates[0] == 0
    d = op.desc()
    size = {B.F32: 4, B.F16: 2, B.BF16: 2, B.F8E4M3: 1, B.I8: 1, B.I32: 4}[d.out_dtype]
    seen = set()
    for c in range(space.slots[0].n_candidates):
        t = B.make_trace(space, [[space.slots[0].candidates[c]]])
        if not space.slots[0].weight[c]:
            refused(B.MS_ERR_INVALID_TRACE, B.trace_validate, op, space, t)
            continue
        p = B.trace_validate(op, space, t)
        assert (B.variant_coverage(op, p, op.tensor_bytes(-1) // size) == 1).all()
        assert (B.variant_reduction_coverage(op, p) == 1).all()
        assert np.isfinite(B.variant_features(op, p)).all()
        assert p.threads == 64 * p.waves <= 1024 and p.lds_bytes <= 160 << 10 and p.rfactor == 1
        text = B.trace_to_text(op, space, t)
        assert "body=" in text and B.trace_from_text(space, text).decisions() == t.decisions()
        seen.add(p.body_tile)
    assert B.trace_validate(op, space, B.default_trace(space)).body_tile in seen
    assert len(seen) >= 2


def test_coverage_is_that_of_the_workgroups_there_are():
    for name in ("route", "route gradient", "out", "back", "back gradient"):
        op = OPS[name]()
        space = op.space()
        p = B.trace_validate(op, space, B.default_trace(space))
        size = {B.F32: 4, B.F16: 2, B.BF16: 2, B.I8: 1}[op.desc().out_dtype]
        p.grid[0] -= 1
        counts = B.variant_coverage(op, p, op.tensor_bytes(-1) // size)
        assert counts.max() <= 1 and (counts == 0).any()


def test_coverage_refuses_the_parameters_of_another_operator():
    route, norm = OPS["route"](), B.rms_norm_op(37, 6)
    p, q = (B.trace_validate(op, op.space(), B.default_trace(op.space())) for op in (route, norm))
    refused(B.MS_ERR_BAD_ARG, B.variant_coverage, route, q, 37 * 6)
    refused(B.MS_ERR_BAD_ARG, B.variant_coverage, norm, p, 37 * 6)
    refused(B.MS_ERR_BAD_ARG, B.variant_reduction_coverage, route, q)
    p.body_tile = 0
    refused(B.MS_ERR_BAD_ARG, B.variant_coverage, route, p, 37 * 6)
    refused(B.MS_ERR_BAD_ARG, B.trace_validate, route, norm.space(), B.default_trace(norm.space()))


def test_sizes_select_code_by_their_power_of_two_only():
    def text(op, code):
        space = op.space()
        p = B.trace_validate(op, space, B.make_trace(space, [[code]]))
        return p.key, B.variant_kernel_text(op, p)

    a = text(B.route_op(37, 60, 6, "bf16"), 16)
    assert a == text(B.route_op(1000, 33, 5, "bf16", a_strides=[0, 99, 1], scale=3.0), 16)
    for other in (B.route_op(37, 70, 6, "bf16"), B.route_op(37, 60, 3, "bf16"), B.route_op(37, 60, 6, "f16"), B.route_op(37, 60, 6, "bf16", bias=True), B.route_op(37, 60, 6, "bf16", scores="sigmoid"),
                  B.route_op(37, 60, 6, "bf16", renormalise=True), B.route_op(37, 60, 6, "bf16", groups=2, kept=1)):
        assert text(other, 16)[0] != a[0]
    a = text(B.join_rows_op(37, 4, 600, 148), 4)
    assert a == text(B.join_rows_op(5, 9, 2222, 45), 4) and a[0] != text(B.join_rows_op(37, 4, 600, 148, residual=True), 4)[0]
    assert text(B.expert_order_op(60, 3000, 8), 1) == text(B.expert_order_op(50, 9000, 2), 1) != text(B.expert_order_op(70, 3000, 8), 1)


def test_tensors_work_loops_and_workspaces():
    op = B.route_op(10, 64, 4, "bf16", bias=True, a_strides=[0, 80, 1])
    assert [op.tensor_bytes(i) for i in (-2, -1, 0, 1)] == [160, 160, (9 * 80 + 64) * 2, 256] and op.work() == (5 * 640, 1280 + 320 + 256)
    assert op.loops() == [("i", 10, False), ("j", 4, False), ("k", 64, True)]
    refused(B.MS_ERR_BAD_ARG, B.route_op(10, 64, 4).tensor_bytes, 1)
    op = B.route_grad_op(10, 64, 4, "bf16")
    assert [op.tensor_bytes(i) for i in (-1, 0, 1, 2)] == [1280, 1280, 160, 160] and op.work()[1] == 2560 + 320
    op = B.expert_order_op(64, 10, 4)
    assert [op.tensor_bytes(i) for i in (-2, -1, 0)] == [160, 260, 160] and variant(op).workspace_bytes() == 0
    op = B.expert_order_op(300, 5000, 8)
    p = variant(op).params()
    assert variant(op).workspace_bytes() == p.grid[0] * 300 * 4 and p.grid[0] * p.block_m >= 40000
    op = B.spread_rows_op(10, 4, 300, 50, "bf16", "f8")
    assert [op.tensor_bytes(i) for i in (-2, -1, 0, 1)] == [50 * 3 * 4, 15000, 6000, 160]
    refused(B.MS_ERR_BAD_ARG, op.tensor_bytes, 2)
    assert B.spread_rows_op(10, 4, 300, 50, "i8").tensor_bytes(2) == 40 and B.spread_rows_op(10, 4, 300, 50, "f8").tensor_bytes(2) == 120 and B.spread_rows_op(10, 4, 300, 50).tensor_bytes(-2) == 0
    op = B.join_rows_op(10, 4, 300, 50, "bf16", "f32", residual=True, a_strides=[0, 304, 1])
    assert [op.tensor_bytes(i) for i in (-1, 0, 1, 2, 3)] == [12000, (49 * 304 + 300) * 2, 160, 160, 12000] and op.loops() == [("i", 10, False), ("j", 4, True), ("k", 300, False)]
    refused(B.MS_ERR_BAD_ARG, B.join_rows_op(10, 4, 300, 50, weights=False).tensor_bytes, 2)
    op = B.join_grad_op(10, 4, 300, 50, a_strides=[0, 310, 1], b_strides=[0, 304, 1])
    assert [op.tensor_bytes(i) for i in (-2, -1, 0, 1, 2, 3)] == [160, 30000, (9 * 310 + 300) * 2, 160, 160, (49 * 304 + 300) * 2]


def test_refused_operators():
    bad, no = B.MS_ERR_BAD_ARG, B.MS_ERR_UNSUPPORTED
    refused(bad, B.route_op, 0, 8, 2)
    refused(bad, B.route_op, 4, 8, 9)                       # more than there are
    refused(bad, B.route_op, 4, 8, 0)
    refused(no, B.route_op, 4, 64, B.MAX_CHOSEN + 1)
    refused(no, B.route_op, 4, B.MAX_EXPERTS + 1, 2)
    refused(no, B.route_op, 4, 128, 2, groups=128)
    refused(bad, B.route_op, 4, 60, 2, groups=7)            # no divisor
    refused(bad, B.route_op, 4, 60, 2, groups=6, kept=7)
    refused(bad, B.route_op, 4, 60, 2, groups=6, kept=0)
    refused(bad, B.route_op, 4, 60, 2, groups=6, kept=1, best=3)
    refused(no, B.route_op, 4, 8, 2, "i8")
    refused(no, B.Op, B.OP_ROUTE, "f16", "f16", [4, 8, 2, 1, 1, 1, 0, 0])
    refused(bad, B.Op, B.OP_ROUTE, "f16", "f32", [4, 8, 2, 1, 1, 1, 4, 0])
    refused(bad, B.Op, B.OP_ROUTE, "f16", "f32", [4, 8, 2, 1, 1, 1, 0, 0x7f800000])   # an infinite scale
    refused(bad, B.Op, B.OP_ROUTE, "f16", "f32", [4, 8, 2, 1, 1, 1, 0, 0x80000001])   # a negative one
    refused(bad, B.Op, B.OP_ROUTE, "f16", "f32", [4, 8, 2, 1, 1, 1, 0, 1])            # a subnormal one
    refused(bad, B.Op, B.OP_ROUTE, "f16", "f32", [4, 8, 2, 1, 1, 1, 0, -5])
    refused(bad, B.Op, B.OP_ROUTE, "f16", "f32", [4, 8, 2])
    for scale in (0, -1, float("nan"), float("inf")):
        with pytest.raises(ValueError):
            B.route_op(4, 8, 2, scale=scale)
    with pytest.raises(ValueError):
        B.route_op(4, 8, 2, scores="tanh")
    refused(bad, B.route_op, 4, 8, 2, relu=True)
    refused(bad, B.route_op, 4, 8, 2, a_strides=[0, 7, 1])
    refused(bad, B.route_op, 4, 8, 2, a_strides=[0, 16, 2])
    refused(bad, B.route_op, 4, 8, 2, a_strides=[0, -8, 1])
    refused(bad, B.route_op, 4, 8, 2, b_strides=[0, 8, 1])
    refused(bad, B.route_op, 1 << 30, 1024, 2, a_strides=[0, 1 << 20, 1])
    refused(bad, B.route_grad_op, 4, 8, 9)
    refused(bad, B.route_grad_op, 4, 8, 2, has_bias=True)
    refused(no, B.Op, B.OP_ROUTE_GRAD, "f16", "f32", [4, 8, 2, 0, 0])
    refused(no, B.expert_order_op, B.MAX_EXPERTS + 1, 4, 2)
    refused(no, B.expert_order_op, 8, B.MAX_CHOICES // 2 + 1, 2)
    refused(no, B.Op, B.OP_EXPERT_ORDER, "f32", "i32", [8, 4, 2])
    refused(bad, B.Op, B.OP_EXPERT_ORDER, "i32", "i32", [8, 4, 2], a_strides=[0, 3, 1])
    refused(no, B.spread_rows_op, 4, B.MAX_ROW_CHOICES + 1, 8, 500)
    refused(no, B.spread_rows_op, 4, 2, 8, 8, "f16", "f32")
    refused(no, B.spread_rows_op, 4, 2, 8, 8, "i8", "f16")
    refused(no, B.spread_rows_op, 4, 2, 8, 8, "i32")
    refused(bad, B.spread_rows_op, 4, 2, 8, 0)
    refused(bad, B.spread_rows_op, 4, 2, 8, 8, has_bias=True)
    refused(bad, B.spread_rows_op, 4, 2, 8, 1 << 31)
    refused(bad, B.spread_rows_op, 4, 2, 1 << 20, 1 << 30)  # 2^50 elements
    refused(no, B.join_rows_op, 4, 2, 8, 8, "i8")
    refused(no, B.join_rows_op, 4, 2, 8, 8, "f32", "f16")
    refused(bad, B.Op, B.OP_JOIN_ROWS, "f16", "f16", [4, 2, 8, 8, 2])
    refused(no, B.Op, B.OP_JOIN_GRAD, "f16", "f32", [4, 2, 8, 8])
    refused(bad, B.join_grad_op, 4, 2, 8, 8, b_strides=[0, 7, 1])
    refused(bad, B.join_grad_op, 4, 2, 8, 8, a_strides=[1, 8, 1])
    for op in (B.route_op(1 << 30, 8, 2), B.route_grad_op(1 << 30, 8, 2), B.join_rows_op(1 << 27, 1, 8, 8), B.spread_rows_op(1 << 27, 1, 8, 8)):  # more threads than a grid has
        refused(B.MS_ERR_INVALID_TRACE, B.trace_validate, op, op.space(), B.default_trace(op.space()))


def test_refused_launches():
    """Everything that a launch checks ahead of its first call of the GPU's runtime; what is allowed gets as far as that, which is not there."""
    bad, at = B.MS_ERR_BAD_ARG, 1 << 20

    def one_off(v, n_in, n_out, optional=(), wide=(), workspace=None):
        """Each tensor in turn not there, and off its alignment."""
        ins, outs = [at * (1 + i) for i in range(n_in)], [at * (9 + i) for i in range(n_out)]
        if not devmem.gpu_available():
            refused(B.MS_ERR_HIP, v.launch, ins, outs, workspace=workspace)
        for i in range(n_in):
            if i not in optional:
                refused(bad, v.launch, [None if k == i else p for k, p in enumerate(ins)], outs, workspace=workspace)
            if i in wide:
                refused(bad, v.launch, [p + 1 if k == i else p for k, p in enumerate(ins)], outs, workspace=workspace)
        for i in range(n_out):
            refused(bad, v.launch, ins, [None if k == i else p for k, p in enumerate(outs)], workspace=workspace)
            refused(bad, v.launch, ins, [p + 1 if k == i else p for k, p in enumerate(outs)], workspace=workspace)
        refused(bad, v.launch, ins, outs, instances=0, workspace=workspace)
        refused(bad, v.launch, ins, outs, instances=65536, workspace=workspace)

    one_off(variant(B.route_op(4, 8, 2, "bf16", bias=True)), 2, 2, wide=(0, 1))
    one_off(variant(B.route_op(4, 8, 2, "bf16")), 1, 2, wide=(0,))
    one_off(variant(B.route_grad_op(4, 8, 2, "f16")), 3, 1, wide=(0, 1, 2))
    one_off(variant(B.expert_order_op(8, 4, 2)), 1, 2, wide=(0,))
    one_off(variant(B.spread_rows_op(4, 2, 8, 8, "f32")), 2, 1, wide=(0, 1))
    one_off(variant(B.spread_rows_op(4, 1, 8, 8, "f32")), 2, 1, optional=(1,), wide=(0, 1))
    one_off(variant(B.join_rows_op(4, 2, 8, 8, "f16", residual=True)), 4, 1, wide=(0, 1, 2, 3))
    one_off(variant(B.join_rows_op(4, 2, 8, 8, "f16", weights=False)), 2, 1, wide=(0, 1))
    one_off(variant(B.join_grad_op(4, 2, 8, 8, "f16")), 4, 2, wide=(0, 1, 2, 3))
    many = variant(B.expert_order_op(8, 9000, 2))
    one_off(many, 1, 2, wide=(0,), workspace=at * 20)
    refused(bad, many.launch, [at], [2 * at, 3 * at])
    refused(bad, many.launch, [at], [2 * at, 3 * at], workspace=at * 20 + 8)
    # 8-bit integers have scales, and rows in 8 bits bring theirs
    v = variant(B.spread_rows_op(4, 2, 8, 8, "bf16", "i8"))
    refused(bad, v.launch, [at, 2 * at], [3 * at, None])
    refused(bad, v.launch, [at, 2 * at], [3 * at, 4 * at + 2])
    v = variant(B.spread_rows_op(4, 2, 8, 8, "f8"))
    refused(bad, v.launch, [at, 2 * at, None], [3 * at, 4 * at])
    # without places: a row for each token
    refused(bad, variant(B.spread_rows_op(4, 1, 8, 3, "bf16")).launch, [at, None], [3 * at])
    # outputs over what other tokens have yet to read
    refused(bad, variant(B.spread_rows_op(4, 1, 8, 4, "bf16")).launch, [at, None], [at])
    refused(bad, variant(B.join_rows_op(4, 2, 8, 8)).launch, [at, 2 * at, 3 * at], [at])
    v = variant(B.join_grad_op(4, 2, 8, 8))
    refused(bad, v.launch, [at, 2 * at, 3 * at, 4 * at], [at, 5 * at])
    refused(bad, v.launch, [at, 2 * at, 3 * at, 4 * at], [4 * at, 5 * at])
    refused(bad, variant(B.route_grad_op(4, 8, 2, a_strides=[0, 9, 1])).launch, [at, 2 * at, 3 * at], [at])
    if not devmem.gpu_available():
        refused(B.MS_ERR_HIP, variant(B.route_grad_op(4, 8, 2)).launch, [at, 2 * at, 3 * at], [at])
        refused(B.MS_ERR_HIP, variant(B.join_rows_op(4, 2, 8, 8, residual=True)).launch, [at, 2 * at, 3 * at, 4 * at], [4 * at])


def test_rules():
    """More lanes to a token, or wavefronts, the fewer tokens there are; never more than there is for them to do."""
    def block(op):
        return B.trace_validate(op, op.space(), B.default_trace(op.space())).body_tile

    assert [block(B.route_op(T, 256, 8)) for T in (1, 1024, 2048, 4096, 16384, 100000)] == [64, 64, 32, 16, 16, 8]
    assert block(B.route_op(100000, 1024, 8)) == 32 and block(B.route_op(100000, 300, 8)) == 16 and block(B.route_op(16384, 60, 6)) == 8
    assert [block(B.join_rows_op(9, 8, N, 72)) for N in (8, 512, 513, 2050, 8192, 8193, 20000)] == [1, 1, 2, 5, 16, 10, 14]
    assert [block(B.expert_order_op(8, T, 8)) for T in (1, 500, 16384, 1 << 20)] == [1, 4, 1, 16] and [block(B.expert_order_op(E, 16384, 8)) for E in (64, 256, 1024)] == [1, 1, 2]


def test_no_size_needs_a_kernel_that_is_not_built_ahead():
    """Of the operators and types that are built ahead: the kernels of drawn sizes are among those of layer_ops(), for every block of theirs."""
    import random
    built = set()
    for op in tuned.layer_ops():
        space = op.space()
        for c in range(space.slots[0].n_candidates):
            if space.slots[0].weight[c]:
                built.add(B.trace_validate(op, space, B.make_trace(space, [[space.slots[0].candidates[c]]])).key)
    r = random.Random(7)
    some = lambda least, most: round(least * (most / least) ** r.random())
    ops = [B.expert_order_op(E, T, K) for E in (64, 256, 1024) for T, K in ((1, 64), (13, 5), (20, 8), (12, 6), (40, 2), (32, 8), (257, 1), (4097, 1), (1 << 23, 8))]
    ops += [B.expert_order_op(some(1, 1024), some(1, 1 << 20), some(1, 16)) for _ in range(60)]
    for _ in range(40):
        T, K, N = some(1, 20000), some(1, 16), some(1, 20000)
        ops += [B.spread_rows_op(T, K, N, T * K, "bf16", r.choice(("bf16", "i8", "f8"))), B.join_grad_op(T, K, N, T * K),
                B.join_rows_op(T, K, N, T * K, "bf16", r.choice(("bf16", "f32")), residual=r.random() < 0.5)]
        ops += [B.scaled_gemm_op(T, N, some(1, 20000), r.choice(("bf16", "f16", "f32")), in_dtype=r.choice(("f8", "i8"))),
                B.grouped_gemm_op(some(1, 64), T, N, some(1, 20000), True, r.choice(("f8", "i8")), r.choice(("bf16", "f16", "f32")))]
    ops.append(B.join_grad_op(50, 1, 1, 50))  # its strides could be those of either order
    for op in ops:
        p = B.trace_validate(op, op.space(), B.default_trace(op.space()))
        assert p.key in built, (op.work(), p.body, p.body_tile, p.threads)


def test_the_exponential_is_as_near_as_it_says():
    """route.hip's steps in exact arithmetic, each rounded to 64 bits once, against e^x in 60 digits: within 2^-45.3 up to 100, 2^-44.4 up to 710."""
    import random
    import re
    from decimal import Decimal, getcontext
    from fractions import Fraction
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "paper_2205_13603_amd", "csrc", "kernels", "route.hip")).read()
    c, per_ln2, ln2, start = re.search(r"series_t s = \{\{([^}]*)\},\s*([^,]+), ([^,]+), ([^}]+)\}", text).groups()
    c, (per_ln2, ln2, start) = [float.fromhex(x.strip()) for x in c.split(",")], [float.fromhex(x.strip()) for x in (per_ln2, ln2, start)]
    fma = lambda a, b, d: float(Fraction(a) * Fraction(b) + Fraction(d))
    getcontext().prec = 60
    r = random.Random(3)
    for most, bound in ((100, 2.0 ** -45.3), (710, 2.0 ** -44.4)):
        for k in range(1500):
            x = r.uniform(-most, most) if k % 3 else (r.randrange(int(most / ln2)) + 0.5) * ln2 * (1 - 2.0 ** -40) * r.choice((1, -1))  # the ends of the polynomial's range
            t = fma(x, per_ln2, start)
            n = t - start
            rest, p = fma(n, -ln2, x), c[0]
            for k in c[1:]:
                p = fma(p, rest, k)
            want = Decimal(x).exp()
            assert abs(Decimal(p) * Decimal(2) ** int(n) - want) <= want * Decimal(bound), x


def test_sampled_composed_and_searched():
    for name, make in OPS.items():
        op = make()
        space = op.space()
        blocks = {tuple(B.trace_sample_valid(op, space, 1, i).d[0].v)[0] for i in range(64)}
        assert len(blocks) == sum(1 for c in range(space.slots[0].n_candidates) if space.slots[0].weight[c]), name
        composed, mask = B.space_compose(op, ["multi-level-tiling", "unroll"])
        assert mask == 0 and composed.n_slots == 1
    op = OPS["back"]()
    cfg = B.search_cfg_default()
    cfg.trials, cfg.init_population, cfg.population, cfg.children = 16, 4, 4, 4
    res = B.search(op, op.space(), cfg, fake_latency=lambda p: 1.0 + abs(p.body_tile - 4))
    assert B.trace_validate(op, op.space(), res.best_trace).body_tile == 4


def test_launches_run_the_kernels_that_they_say(tmp_path):
    """On a stand-in for HIP that keeps book of launches, under the address sanitizer: grids, instances, the first kernel of an order in runs, workspaces."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "ms_routing")
    srcs = [os.path.join(root, "paper_2205_13603_amd", "csrc", f) for f in ("ms_core.cpp", "ms_interp.cpp", "ms_model.cpp", "ms_search.cpp", "ms_runtime.cpp")]
    r = subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-D__align__(n)=", "-DHIP_SYMBOL(x)=(&x)",
                        "-I", "/opt/rocm/include", "-o", exe] + srcs + [os.path.join(root, "tests", "sanitize", "routing_driver.cpp"), "-lm", "-lpthread"],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-4000:]
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=600)
    assert r.returncode == 0 and "routing checks ok" in r.stdout, r.stdout[-6000:]
