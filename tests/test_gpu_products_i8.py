"""Products in 8-bit integers with a scale for each row and each column, of one matrix and grouped by expert, against their definition in 64 bits.

Tolerances.  The sum of products is exact in 32 bits; its rounding to fp32 and the two products with scales are off by half a step each,
3 * 2^-24 of the result, and the rounding to the output type by half a step of that: 2^-24 (fp32: none, it is fp32 already), 2^-11 in fp16 (2^-25
where it is subnormal), 2^-8 in bf16."""
import numpy as np
import pytest
import torch

from paper_2205_13603_amd import binding as B, devmem
from test_gpu_layers import TYPES, dev, launch_twice, offsets_of, rng, variant

pytestmark = pytest.mark.gpu

STEP = {"f32": 0.0, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
CODES = [0, 16016, 16032, 32032, 64032, 64128, 128128, 256256]


def ints(g, *shape, low=-128, high=128):
    return torch.randint(low, high, shape, generator=g, dtype=torch.int8)


def scales(g, *shape):
    return torch.rand(*shape, generator=g) * 0.02 + 0.001


def close(got, want, kind):
    got = got.double()
    tol = want.abs() * (3 * 2.0 ** -24 + STEP[kind]) * 1.01 + (2.0 ** -25 if kind == "f16" else 1e-37)
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), "%d values off, the first at %s: %r, %r" % (int(bad.sum()), bad.nonzero()[0].tolist(), float(got[bad][0]), float(want[bad][0]))


@pytest.mark.parametrize("M,N,K,out,code", [
    (1, 1, 1, "f32", 0), (1, 16, 16, "bf16", 0), (1, 128, 128, "f16", 0), (3, 201, 272, "bf16", 0), (16, 256, 1024, "f32", 0), (17, 384, 640, "f16", 0), (33, 130, 2064, "bf16", 0),
    (70, 77, 144, "f16", 0), (129, 257, 400, "bf16", 0), (300, 520, 1360, "f32", 0), (513, 263, 1152, "f16", 0)]
    + [(41, 151, 656, "bf16", c) for c in CODES[1:]] + [(270, 301, 2192, "f32", c) for c in CODES[1:]] + [(129, 260, 16, "f16", c) for c in CODES[1:]]
    + [(20, 48, 100, "bf16", 0), (65, 131, 517, "f16", 0), (130, 129, 1, "f32", 0), (5, 7, 129, "f32", 0)])
def test_product(M, N, K, out, code):
    v = variant(B.scaled_gemm_op(M, N, K, out, in_dtype="i8"), code)
    if v is None:
        return
    g = rng(M * 7 + N * 5 + K)
    a, b, sa, sb = ints(g, M, K), ints(g, N, K), scales(g, M), scales(g, N)
    (c,) = launch_twice(v, [dev(x) for x in (a, b, sa, sb)], [((M, N), TYPES[out])])
    close(c, a.double() @ b.double().t() * sa.double()[:, None] * sb.double(), out)


@pytest.mark.parametrize("code", CODES[1:])
def test_longest_sums_are_exact(code):
    """-128 times -128 all along the longest reduction is 2^31 - 2^14, the largest sum of 32 bits that there is; one sign only overflows nowhere else."""
    M, N, K = 3, 5, B.MAX_I8_DEPTH // 16 * 16
    v = variant(B.scaled_gemm_op(M, N, K, "f32", in_dtype="i8"), code)
    if v is None:
        return
    a, b = torch.full((M, K), -128, dtype=torch.int8), torch.full((N, K), -128, dtype=torch.int8)
    a[1] = 127
    b[2] = 127
    b[3, 1::2] = 127
    (c,) = launch_twice(v, [dev(a), dev(b), torch.ones(M).cuda(), torch.ones(N).cuda()], [((M, N), torch.float32)])
    assert torch.equal(c, (a.double() @ b.double().t()).float())


def test_scales_are_those_of_their_row_and_column():
    """Small, large, zero, negative, infinite and NaN scales stay with their row or column; no product of two small scales is formed."""
    M, N, K = 150, 140, 64
    v = variant(B.scaled_gemm_op(M, N, K, "f32", in_dtype="i8"))
    if v is None:
        return
    g = rng(3)
    a, b, sa, sb = ints(g, M, K, low=1), ints(g, N, K, low=1), scales(g, M), scales(g, N)
    sa[3], sa[5], sa[7], sa[149] = 1e-30, -0.5, 0, float("nan")
    sb[2], sb[4], sb[139] = 1e-20, 1e30, float("inf")
    (c,) = launch_twice(v, [dev(x) for x in (a, b, sa, sb)], [((M, N), torch.float32)])
    want = a.double() @ b.double().t() * sa.double()[:, None] * sb.double()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(c), nan) and int(nan.sum()) == N + 1  # 0 times infinity
    same = ~nan & torch.isinf(want)
    assert torch.equal(c[same].double(), want[same])
    fine = ~nan & ~same
    assert bool(((c[fine].double() - want[fine]).abs() <= want[fine].abs() * 3 * 2.0 ** -24 * 1.01 + 2.0 ** -148).all())


def test_strides_and_instances():
    M, N, K, R = 37, 96, 160, 3
    op = B.scaled_gemm_op(M, N, K, "bf16", in_dtype="i8", a_strides=[0, 192, 1], b_strides=[0, 1, 176])
    v = variant(op)
    if v is None:
        return
    g = rng(5)
    a, b, sa, sb = ints(g, R, M, K), ints(g, R, N, K), scales(g, R, M), scales(g, R, N)
    spans = [op.tensor_bytes(i) for i in range(2)]
    pa, pb = (torch.full((R * s,), 77, dtype=torch.int8) for s in spans)
    for r in range(R):
        torch.as_strided(pa, (M, K), (192, 1), r * spans[0]).copy_(a[r])
        torch.as_strided(pb, (N, K), (176, 1), r * spans[1]).copy_(b[r])
    (c,) = launch_twice(v, [dev(x) for x in (pa, pb, sa, sb)], [((R, M, N), TYPES["bf16"])], instances=R)
    close(c, a.double() @ b.double().transpose(1, 2) * sa.double()[..., None] * sb.double()[:, None], "bf16")


# experts' rows, rows of no expert ahead and behind, N, K
GROUPED = [([1], 0, 0, 33, 64), ([0, 1, 0], 0, 0, 48, 128), ([5, 0, 16, 1], 0, 3, 161, 192), ([0, 0, 37], 2, 1, 128, 80), ([64, 65, 0, 63, 1, 130], 1, 7, 264, 336),
           ([300, 0, 270], 0, 5, 272, 528), ([3] * 70, 0, 0, 64, 96), ([257, 1, 256, 255], 3, 0, 521, 272), ([0, 0, 0], 2, 3, 40, 64), ([3, 0, 65, 130], 1, 1, 50, 77)]


def check_grouped(v, counts, ahead, behind, N, K, out, seed=1):
    E, T = len(counts), ahead + sum(counts) + behind
    g = rng(seed + T + N + K)
    a, b, sa, sb = ints(g, T, K), ints(g, E, N, K), scales(g, T), scales(g, E, N)
    off = offsets_of(counts, ahead)
    sa[:ahead] = sa[T - behind:] = float("nan")  # of rows of no expert
    (c,) = launch_twice(v, [dev(x) for x in (a, b, off, sa, sb)], [((T, N), TYPES[out])])
    assert bool((c[:ahead].float() == 7).all()) and bool((c[T - behind:].float() == 7).all()), "rows of no expert were written"
    for e in range(E):
        rows = slice(int(off[e]), int(off[e + 1]))
        close(c[rows], a[rows].double() @ b[e].double().t() * sa[rows].double()[:, None] * sb[e].double(), out)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("which", range(len(GROUPED)))
@pytest.mark.parametrize("code", [0, -1, 128128, 256256])
def test_grouped_product(which, out, code):
    counts, ahead, behind, N, K = GROUPED[which]
    if K % 16:
        code = 0
    if code == -1:  # another small tile each time
        code = [16016, 16032, 32032, 64032, 64128][which % 5]
    v = variant(B.grouped_gemm_op(len(counts), ahead + sum(counts) + behind, N, K, True, "i8", out), code)
    if v is not None:
        check_grouped(v, counts, ahead, behind, N, K, out)


@pytest.mark.parametrize("code", [16032, 64128, 128128, 256256])
def test_tiles_of_which_several_lie_on_a_compute_unit(code):
    """More tiles than compute units, rests of experts' rows, more than one round of whole tiles."""
    counts = [130 + e for e in range(21)] + [0, 256 + 97]
    for K in (64, 208, 1168):
        v = variant(B.grouped_gemm_op(len(counts), sum(counts) + 3, 4600, K, True, "i8", "bf16"), code)
        if v is not None:
            check_grouped(v, counts, 1, 2, 4600, K, "bf16")


@pytest.mark.parametrize("K", [16, 128, 144, 400])
@pytest.mark.parametrize("code", [128128, 256256])
def test_turns_of_few_steps(code, K):
    """Several tiles for each workgroup, of one step of 128 bytes to four: scales come in ahead of tiles whose products are still to be made."""
    M, N = 6001, 8200
    v = variant(B.scaled_gemm_op(M, N, K, "bf16", in_dtype="i8"), code)
    if v is None:
        return
    g = rng(K)
    a, b, sa, sb = ints(g, M, K), ints(g, N, K), scales(g, M), scales(g, N)
    (c,) = launch_twice(v, [dev(x) for x in (a, b, sa, sb)], [((M, N), torch.bfloat16)])
    close(c, a.double() @ b.double().t() * sa.double()[:, None] * sb.double(), "bf16")


def test_many_experts():
    E = B.MAX_EXPERTS
    counts = [(e * 7) % 3 for e in range(E)]
    v = variant(B.grouped_gemm_op(E, sum(counts) + 4, 17, 32, True, "i8", "f16"))
    if v is not None:
        check_grouped(v, counts, 2, 2, 17, 32, "f16")


@pytest.mark.parametrize("code", [0, 16016, 64128, 128128, 256256])
def test_experts_of_several_instances(code):
    R, E, T, N, K = 3, 4, 320, 264, 144
    counts = [[100, 0, 200, 3], [0, 0, 0, 320], [1, 130, 64, 125]]
    v = variant(B.grouped_gemm_op(E, T, N, K, True, "i8", "bf16"), code)
    if v is None:
        return
    g = rng(91)
    off = torch.stack([offsets_of(c) for c in counts])
    a, b, sa, sb = ints(g, R, T, K), ints(g, R, E, N, K), scales(g, R, T), scales(g, R, E, N)
    (c,) = launch_twice(v, [dev(x) for x in (a, b, off, sa, sb)], [((R, T, N), torch.bfloat16)], instances=R)
    for r in range(R):
        for e in range(E):
            rows = slice(int(off[r, e]), int(off[r, e + 1]))
            close(c[r, rows], a[r, rows].double() @ b[r, e].double().t() * sa[r, rows].double()[:, None] * sb[r, e].double(), "bf16")
        assert bool((c[r, int(off[r, -1]):] == 7).all())


def test_captured_products_follow_their_inputs():
    """One operator of each in a graph, replayed with other rows, scales and offsets and the program's own work in between."""
    E, T, N, K = 4, 130, 136, 128
    ops = [variant(B.scaled_gemm_op(T, N, K, in_dtype="i8")), variant(B.grouped_gemm_op(E, T, N, K, True, "i8"))]
    if ops[0] is None:
        return
    for v in ops:
        v.prepare()
    g = rng(31)
    a, b, sa, sb, off = (dev(x) for x in (ints(g, T, K), ints(g, E, N, K), scales(g, T), scales(g, E, N), offsets_of([30, 40, 0, 60])))
    c, ce = (torch.zeros(T, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def step():
        at = devmem.current_stream()
        ops[0].launch_static([a.data_ptr(), b.data_ptr(), sa.data_ptr(), sb.data_ptr()], c.data_ptr(), stream=at)
        ops[1].launch_static([a.data_ptr(), b.data_ptr(), off.data_ptr(), sa.data_ptr(), sb.data_ptr()], ce.data_ptr(), stream=at)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k, counts in enumerate([[30, 40, 0, 60], [0, 0, 130, 0], [1, 2, 3, 4], [65, 0, 0, 65]]):
        off.copy_(offsets_of(counts))
        a.copy_(ints(g, T, K))
        sa.copy_(scales(g, T))
        got = []
        for run in (graph.replay, step):
            c.fill_(3)
            ce.fill_(3)
            run()
            torch.cuda.synchronize()
            got.append([c.cpu().clone(), ce.cpu().clone()])
        assert all(torch.equal(p, q) for p, q in zip(*got)), "replay %d" % k
        assert bool((got[0][1][sum(counts):] == 3).all())


def test_measure_and_search():
    E, T, N, K = 2, 60, 128, 256
    op = B.grouped_gemm_op(E, T, N, K, True, "i8", "bf16")
    v = variant(op)
    if v is None:
        return
    g = rng(51)
    a, b, sa, sb = ints(g, T, K), ints(g, E, N, K), scales(g, T), scales(g, E, N)
    block = torch.zeros(-(-op.tensor_bytes(3) // 256) * 256 + op.tensor_bytes(4), dtype=torch.uint8)  # both scales in one block
    block[:op.tensor_bytes(3)] = sa.reshape(-1).view(torch.uint8)
    block[-op.tensor_bytes(4):] = sb.reshape(-1).view(torch.uint8)
    ins = [dev(x) for x in (a, b, offsets_of([20, 40]), block)]
    c, want = (torch.zeros(T, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m = v.measure([([t.data_ptr() for t in ins], c.data_ptr())], stream=devmem.current_stream())
    assert 0 < m.min_us < 1e5 and m.flop == 2 * T * N * K
    sa, sb = dev(sa), dev(sb)
    v.launch([t.data_ptr() for t in ins[:3]] + [sa.data_ptr(), sb.data_ptr()], want.data_ptr(), stream=devmem.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(c, want)
    cfg = B.search_cfg_default()
    cfg.trials, cfg.init_population = 4, 4
    res = B.search(op, op.space(), cfg, [([t.data_ptr() for t in ins], c.data_ptr())], stream=devmem.current_stream())
    assert res.n_measured >= 2 and res.n_failed == 0 and torch.equal(c, want)


def test_against_numpy_integers():
    """The definition once more, from another library's integer products."""
    M, N, K = 19, 23, 304
    v = variant(B.scaled_gemm_op(M, N, K, "f32", in_dtype="i8"))
    if v is None:
        return
    g = np.random.default_rng(4)
    a, b = g.integers(-128, 128, (M, K)).astype(np.int8), g.integers(-128, 128, (N, K)).astype(np.int8)
    (c,) = launch_twice(v, [torch.from_numpy(a).cuda(), torch.from_numpy(b).cuda(), torch.ones(M).cuda(), torch.ones(N).cuda()], [((M, N), torch.float32)])
    assert np.array_equal(c.numpy().astype(np.int64), a.astype(np.int64) @ b.astype(np.int64).T)
