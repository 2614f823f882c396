"""Layers of language models on the GPU: the RMS norm with 8-bit outputs, block-scaled products, products grouped by expert and the
gradient of the experts' matrices, against their definitions in 64 bits.

Tolerances.  A sum of n fp32 terms in any order is off by at most n 2^-24 of the sum of their magnitudes (to first order), here doubled for
the matrix cores' own order.  Those add the 128 products of one 8-bit instruction with less than fp32 precision, 1e-4 of the root mean
square at random operands, which is 2^-16 of the sum of magnitudes; 2^-13 allows for operands of one sign.  The one rounding of the result adds half a
step: 2^-11 in fp16, 2^-8 in bf16 (2^-25 and below where fp16 is subnormal)."""
import numpy as np
import pytest
import torch

import gpu_util
from paper_2205_13603_amd import binding as B, devmem

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "f8": torch.float8_e4m3fn}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f8": 2.0 ** -4}
GUARD = 64  # elements around an output that have to stay as they are


def variant(op, code=0):
    space = op.space()
    v = B.Variant(op, space, B.make_trace(space, [[code]]) if code else B.default_trace(space))
    if not devmem.gpu_available():
        gpu_util.PRECOMPILED_ONLY = True
        return None
    return v


def rng(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, dtype=torch.float32) * scale


def f8_and_scales(x, rows_per_scale):
    """[..., rows, cols] in 8-bit floats, scales for blocks of rows_per_scale x 128, and the values these stand for in 64 bits."""
    rows, cols = x.shape[-2:]
    rb, cb = -(-rows // rows_per_scale), -(-cols // 128)
    s = torch.ones(*x.shape[:-2], rb, cb)
    for i in range(rb):
        for j in range(cb):
            part = x[..., i * rows_per_scale:(i + 1) * rows_per_scale, j * 128:(j + 1) * 128]
            s[..., i, j] = part.abs().amax((-2, -1)) / 448 + 1e-9
    wide = s.repeat_interleave(rows_per_scale, -2)[..., :rows, :].repeat_interleave(128, -1)[..., :cols]
    q = (x / wide).to(TYPES["f8"])
    return q, s, q.double() * wide.double()


def guarded(shape, dtype, fill=7.0):
    n = int(np.prod(shape))
    t = torch.full((n + 2 * GUARD,), fill, dtype=torch.float32).to(dtype).cuda()
    return t, t[GUARD:GUARD + n].view(shape)


def dev(x):
    return x.cuda() if x is not None else None


def launch_twice(v, inputs, out_shapes, instances=1, stream=None):
    """Outputs of two launches, equal bit for bit, nothing written around them."""
    got = []
    for _ in range(2):
        whole = [guarded(*s) if s else (None, None) for s in out_shapes]
        v.launch([x.data_ptr() if x is not None else None for x in inputs], [w[1].data_ptr() if w[1] is not None else None for w in whole], instances=instances,
                 stream=stream or devmem.current_stream())
        torch.cuda.synchronize()
        for w in whole:
            if w[0] is not None:
                edge = torch.cat([w[0][:GUARD], w[0][-GUARD:]]).float()
                assert bool((edge == 7.0).all()), "written around the output"
        got.append([w[1].cpu() if w[1] is not None else None for w in whole])
    for a, b in zip(*got):
        if a is not None:
            a, b = a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)
            assert torch.equal(a, b), "two launches differ"
    return got[0]


def close(got, want, magnitudes, terms, kind, f8=False):
    got = got.double()
    tol = magnitudes * (2 * terms * 2.0 ** -24 + (2.0 ** -13 if f8 else 0)) + want.abs() * HALF_STEP[kind] * 1.01 + (2.0 ** -24 if kind == "f16" else 1e-37)
    off = (got - want).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), "%d values off, worst %.3g of its tolerance at %s" % (int(bad.sum()), float((off / tol).max()), bad.nonzero()[0].tolist())


# ---------------------------------------------------------------- block-scaled products

CODES = [0, 16016, 16032, 32032, 64032, 64128, 128128, 256256]


@pytest.mark.parametrize("M,N,K,out,code", [
    (1, 16, 16, "bf16", 0), (1, 128, 128, "f16", 0), (3, 200, 272, "bf16", 0), (16, 256, 1024, "f32", 0), (17, 384, 640, "f16", 0), (33, 130, 2064, "bf16", 0),
    (70, 77, 144, "f16", 0), (129, 257, 400, "bf16", 0), (300, 520, 1360, "f32", 0), (513, 264, 1152, "f16", 0)]
    + [(41, 152, 656, "bf16", c) for c in CODES[1:]] + [(270, 301, 2192, "f16", c) for c in CODES[1:]]
    + [(20, 48, 100, "bf16", 0), (65, 131, 517, "f16", 0), (130, 129, 1, "f32", 0)])
def test_scaled_product(M, N, K, out, code):
    v = variant(B.scaled_gemm_op(M, N, K, out), code)
    if v is None:
        return
    g = rng(M * 7 + N * 5 + K)
    a, sa, av = f8_and_scales(normal(g, M, K), 1)
    b, sb, bv = f8_and_scales(normal(g, N, K, scale=0.3), 128)
    (c,) = launch_twice(v, [dev(x) for x in (a, b, sa, sb)], [((M, N), TYPES[out])])
    close(c, av @ bv.t(), av.abs() @ bv.abs().t(), K // 64 + 4, out, f8=True)


def test_scaled_product_strides_and_instances():
    M, N, K, R = 37, 96, 160, 3
    op = B.scaled_gemm_op(M, N, K, "bf16", a_strides=[0, 192, 1], b_strides=[0, 1, 176])
    v = variant(op)
    if v is None:
        return
    g = rng(5)
    a, sa, av = f8_and_scales(normal(g, R, M, K), 1)
    b, sb, bv = f8_and_scales(normal(g, R, N, K), 128)
    # consecutive copies of the spans that the strides touch, NaN between the rows
    spans = [op.tensor_bytes(i) for i in range(2)]
    pa, pb = (torch.full((R * s,), 0x7f, dtype=torch.uint8) for s in spans)
    for r in range(R):
        torch.as_strided(pa, (M, K), (192, 1), r * spans[0]).copy_(a[r].view(torch.uint8))
        torch.as_strided(pb, (N, K), (176, 1), r * spans[1]).copy_(b[r].view(torch.uint8))
    if spans[0] % 16 or spans[1] % 16:
        pytest.fail("sizes of this test make whole 16 bytes")
    (c,) = launch_twice(v, [dev(x) for x in (pa, pb, sa, sb)], [((R, M, N), TYPES["bf16"])], instances=R)
    close(c, av @ bv.transpose(1, 2), av.abs() @ bv.abs().transpose(1, 2), 8, "bf16", f8=True)


# ---------------------------------------------------------------- products grouped by expert

def offsets_of(counts, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(counts)]), dtype=torch.int32)


GROUPED = [
    # experts' rows, rows of no expert ahead and behind, N, K
    ([1], 0, 0, 32, 64), ([0, 1, 0], 0, 0, 48, 128), ([5, 0, 16, 1], 0, 3, 160, 192), ([0, 0, 37], 2, 1, 128, 72), ([64, 65, 0, 63, 1, 130], 1, 7, 264, 328),
    ([300, 0, 270], 0, 5, 272, 520), ([3] * 70, 0, 0, 64, 96), ([257, 1, 256, 255], 3, 0, 520, 264)]


@pytest.mark.parametrize("kind,out,rows_of_k", [("bf16", "bf16", True), ("f16", "f32", True), ("f16", "f16", False), ("bf16", "f32", False), ("f8", "bf16", True), ("f8", "f16", True)])
@pytest.mark.parametrize("which", range(len(GROUPED)))
@pytest.mark.parametrize("code", [0, -1, 128128, 256256])
def test_grouped_product(which, kind, out, rows_of_k, code):
    counts, ahead, behind, N, K = GROUPED[which]
    if kind == "f8":
        K = max(-(-K // 16) * 16, 144 if code == 256256 else 16)  # tiles of 256 x 256 need two blocks of scales
    E, T = len(counts), ahead + sum(counts) + behind
    if code == -1:  # another small tile each time
        code = [16016, 16032, 32032, 64032, 64128][which % 5] if rows_of_k else 64128
    v = variant(B.grouped_gemm_op(E, T, N, K, rows_of_k, kind, out), code)
    if v is None:
        return
    check_grouped(v, counts, ahead, behind, N, K, kind, out, rows_of_k)


def check_grouped(v, counts, ahead, behind, N, K, kind, out, rows_of_k, seed=1):
    E, T = len(counts), ahead + sum(counts) + behind
    g = rng(seed + T + N + K)
    a, b = normal(g, T, K), normal(g, E, N, K, scale=0.3)
    off = offsets_of(counts, ahead)
    ins = []
    if kind == "f8":
        a, sa, av = f8_and_scales(a, 1)
        b, sb, bv = f8_and_scales(b, 128)
        ins = [dev(sa), dev(sb)]
    else:
        a, b = a.to(TYPES[kind]), b.to(TYPES[kind])
        av, bv = a.double(), b.double()
        if not rows_of_k:
            b = b.transpose(1, 2).contiguous()
    a = a.clone()
    a.view(torch.uint8 if kind == "f8" else torch.int16)[:ahead] = 0x7f if kind == "f8" else 0x7fff  # NaN in rows of no expert
    a.view(torch.uint8 if kind == "f8" else torch.int16)[T - behind:] = 0x7f if kind == "f8" else 0x7fff
    (c,) = launch_twice(v, [dev(a), dev(b), dev(off)] + ins, [((T, N), TYPES[out])])
    assert bool((c[:ahead].float() == 7).all()) and bool((c[T - behind:].float() == 7).all()), "rows of no expert were written"
    want, mag = torch.zeros(T, N, dtype=torch.float64), torch.zeros(T, N, dtype=torch.float64)
    for e in range(E):
        rows = slice(int(off[e]), int(off[e + 1]))
        want[rows], mag[rows] = av[rows] @ bv[e].t(), av[rows].abs() @ bv[e].abs().t()
    inside = slice(ahead, T - behind)
    close(c[inside], want[inside], mag[inside], K, out, f8=kind == "f8")


@pytest.mark.parametrize("kind,rows_of_k,N,K", [("f16", True, 50, 77), ("bf16", False, 51, 80), ("bf16", False, 131, 67), ("f8", True, 33, 130), ("f16", True, 64, 100)])
def test_grouped_product_of_odd_sizes(kind, rows_of_k, N, K):
    """Rows that start off 16-byte boundaries, extents that are no whole 16 bytes."""
    counts = [3, 0, 65, 130]
    v = variant(B.grouped_gemm_op(4, 200, N, K, rows_of_k, kind, "bf16" if kind == "f8" else kind))
    if v is not None:
        check_grouped(v, counts, 1, 1, N, K, kind, "bf16" if kind == "f8" else kind, rows_of_k)


@pytest.mark.parametrize("code", [16016, 16032, 32032, 64032])
@pytest.mark.parametrize("kind", ["f8", "bf16"])
def test_few_rows_in_more_workgroups_than_compute_units(kind, code):
    counts = [70, 0, 1, 33, 3]
    v = variant(B.grouped_gemm_op(5, sum(counts) + 3, 4200, 656, True, kind, "bf16"), code)
    if v is not None:
        check_grouped(v, counts, 1, 2, 4200, 656, kind, "bf16", True)


def test_grouped_product_takes_offsets_outside_for_the_nearer_end():
    v = variant(B.grouped_gemm_op(3, 40, 32, 64))
    if v is None:
        return
    g = rng(3)
    a, b = normal(g, 40, 64).bfloat16(), normal(g, 3, 32, 64).bfloat16()
    off = torch.tensor([-5, 10, 10, 1000], dtype=torch.int32)
    (c,) = launch_twice(v, [dev(a), dev(b), dev(off)], [((40, 32), torch.bfloat16)])
    want = torch.cat([a[:10].double() @ b[0].double().t(), a[10:].double() @ b[2].double().t()])
    mag = torch.cat([a[:10].double().abs() @ b[0].double().abs().t(), a[10:].double().abs() @ b[2].double().abs().t()])
    close(c, want, mag, 64, "bf16")


def test_grouped_product_with_many_experts():
    E = B.MAX_EXPERTS
    counts = [(e * 7) % 3 for e in range(E)]
    v = variant(B.grouped_gemm_op(E, sum(counts) + 4, 16, 32, True, "f16"))
    if v is not None:
        check_grouped(v, counts, 2, 2, 16, 32, "f16", "f16", True)


@pytest.mark.parametrize("kind,rows_of_k,K", [("bf16", True, 40), ("bf16", True, 72), ("f16", True, 192), ("f16", False, 328), ("f8", True, 144), ("f8", True, 1040), ("f8", True, 2064)])
def test_workgroups_that_go_on_to_further_tiles(kind, rows_of_k, K):
    """More tiles of 256 x 256 than compute units, of experts with and without rows."""
    counts = [(e * 5) % 4 for e in range(800)]
    counts[400] = 300
    v = variant(B.grouped_gemm_op(800, sum(counts) + 3, 72, K, rows_of_k, kind, "bf16" if kind == "f8" else kind), 256256)
    if v is not None:
        check_grouped(v, counts, 1, 2, 72, K, kind, "bf16" if kind == "f8" else kind, rows_of_k)


@pytest.mark.parametrize("kind,rows_of_k,K", [("bf16", True, 40), ("bf16", True, 136), ("f16", False, 200), ("f8", True, 144), ("f8", True, 1168)])
def test_whole_tiles_in_more_than_one_round(kind, rows_of_k, K):
    """22 experts of more than half a tile's rows by 18 tiles of columns: 396 whole tiles, a last round too full to be made in quarters; and rests
    of experts' rows, which are."""
    counts = [130 + e for e in range(21)] + [256 + 97]
    v = variant(B.grouped_gemm_op(22, sum(counts) + 3, 4600, K, rows_of_k, kind, "bf16" if kind == "f8" else kind), 256256)
    if v is not None:
        check_grouped(v, counts, 1, 2, 4600, K, kind, "bf16" if kind == "f8" else kind, rows_of_k)


def test_scaled_whole_tiles_and_quarters():
    for M, N, K, out in ((2816, 9176, 272, "bf16"), (2900, 6000, 400, "f16")):  # 396 whole tiles; 264 and 24 halves
        v = variant(B.scaled_gemm_op(M, N, K, out), 256256)
        if v is None:
            continue
        g = rng(M)
        a, sa, av = f8_and_scales(normal(g, M, K), 1)
        b, sb, bv = f8_and_scales(normal(g, N, K, scale=0.3), 128)
        (c,) = launch_twice(v, [dev(x) for x in (a, b, sa, sb)], [((M, N), TYPES[out])])
        close(c, av @ bv.t(), av.abs() @ bv.abs().t(), K // 64 + 4, out, f8=True)


def test_weight_gradients_of_more_tiles_than_compute_units():
    check_wgrad([(e * 5) % 4 * 17 for e in range(700)], 1, 2, 24, 40, "bf16", "f32", 256256)
    check_wgrad([(e % 64 == 5) * 100 for e in range(700)], 1, 2, 24, 40, "f16", "f16", 256256)


@pytest.mark.parametrize("code", [64128, 128128])
def test_tiles_of_which_several_lie_on_a_compute_unit(code):
    """More tiles than compute units: the kernels of one group of wavefronts; and at most as many, of two groups, at depths of one step and of an odd and an
    even number of steps."""
    counts = [130 + e for e in range(10)] + [0, 97]
    for kind, rows_of_k, K, N in (("bf16", True, 136, 4600), ("f16", False, 200, 4600), ("f8", True, 1168, 4600), ("bf16", True, 64, 264), ("bf16", True, 192, 264), ("f16", False, 256, 264),
                                  ("f8", True, 128, 264), ("f8", True, 1168, 264), ("f8", True, 2192, 264)):
        v = variant(B.grouped_gemm_op(len(counts), sum(counts) + 3, N, K, rows_of_k, kind, "bf16" if kind == "f8" else kind), code)
        if v is not None:
            check_grouped(v, counts, 1, 2, N, K, kind, "bf16" if kind == "f8" else kind, rows_of_k)
    check_wgrad([65, 0, 130, 1] * 6, 1, 2, 264, 520, "bf16", "f32", code)
    check_wgrad([65, 0, 130, 1] * 6, 1, 2, 264, 520, "f16", "f16", code)


def test_grouped_product_strides():
    E, T, N, K = 3, 50, 40, 64
    v = variant(B.grouped_gemm_op(E, T, N, K, True, "bf16", a_strides=[0, 72, 1], b_strides=[44 * 80, 1, 80]))
    w = variant(B.grouped_gemm_op(E, T, N, K, False, "bf16", b_strides=[70 * 48, 48, 1]))
    if v is None:
        return
    g = rng(9)
    a, b = normal(g, T, 72).bfloat16(), normal(g, E, 44, 80).bfloat16()
    off = offsets_of([20, 0, 30])
    (c,) = launch_twice(v, [dev(a), dev(b), dev(off)], [((T, N), torch.bfloat16)])
    av, bv = a[:, :K].double(), b[:, :N, :K].double()
    close(c, torch.cat([av[:20] @ bv[0].t(), av[20:] @ bv[2].t()]), torch.cat([av[:20].abs() @ bv[0].abs().t(), av[20:].abs() @ bv[2].abs().t()]), K, "bf16")
    a, b = normal(g, T, K).bfloat16(), normal(g, E, 70, 48).bfloat16()
    (c,) = launch_twice(w, [dev(a), dev(b), dev(off)], [((T, N), torch.bfloat16)])
    av, bv = a.double(), b[:, :K, :N].double()
    close(c, torch.cat([av[:20] @ bv[0], av[20:] @ bv[2]]), torch.cat([av[:20].abs() @ bv[0].abs(), av[20:].abs() @ bv[2].abs()]), K, "bf16")


@pytest.mark.parametrize("code", [16016, 64128, 128128, 256256])
def test_products_beyond_4_gib(code):
    """The last experts of matrices of 5 GiB, and the last rows of inputs of 5 GiB."""
    E, N, K = 80, 4096, 8192
    many, long = variant(B.grouped_gemm_op(E, 40, N, K, True, "bf16", "f32"), code), variant(B.grouped_gemm_op(2, 330000, 128, K, True, "bf16", "f32"), code)
    if many is None:
        return
    g = rng(61)
    a, last = normal(g, 40, K).bfloat16(), normal(g, N, K).bfloat16()
    b = torch.zeros(E, N, K, dtype=torch.bfloat16, device="cuda")
    b[-1] = dev(last)
    c = torch.full((40, N), 7.0, device="cuda")
    da, off = dev(a), dev(offsets_of([0] * 30 + [3] + [0] * (E - 33) + [7, 30]))
    many.launch([da.data_ptr(), b.data_ptr(), off.data_ptr()], c.data_ptr(), stream=devmem.current_stream())
    torch.cuda.synchronize()
    assert bool((c[:10] == 0).all())
    some = slice(0, N, 97)
    close(c[10:].cpu()[:, some], a[10:].double() @ last[some].double().t(), a[10:].double().abs() @ last[some].double().abs().t(), K, "f32")
    del b
    x = torch.zeros(330000, K, dtype=torch.bfloat16, device="cuda")
    x[-40:] = da
    w = normal(g, 2, 128, K).bfloat16()
    c, dw, off = torch.full((330000, 128), 7.0, device="cuda"), dev(w), dev(torch.tensor([330000 - 40, 330000 - 25, 330000], dtype=torch.int32))
    long.launch([x.data_ptr(), dw.data_ptr(), off.data_ptr()], c.data_ptr(), stream=devmem.current_stream())
    torch.cuda.synchronize()
    assert bool((c[:-40] == 7).all())
    av, wv = a.double(), w.double()
    close(c[-40:].cpu(), torch.cat([av[:15] @ wv[0].t(), av[15:] @ wv[1].t()]), torch.cat([av[:15].abs() @ wv[0].abs().t(), av[15:].abs() @ wv[1].abs().t()]), K, "f32")


@pytest.mark.parametrize("code", [64128, 128128, 256256])
def test_weight_gradients_and_norms_beyond_4_gib(code):
    E, I, J = 20, 8192, 8192
    v, n = variant(B.grouped_wgrad_op(E, 70, I, J, "bf16", "f32"), code), variant(B.rms_norm_op(330000, 8192, "bf16", "f8", residual=False))
    if v is None:
        return
    g = rng(62)
    p, q = normal(g, 70, I).bfloat16(), normal(g, 70, J).bfloat16()
    d, dp, dq = torch.full((E, I, J), 7.0, device="cuda"), dev(p), dev(q)
    off = dev(offsets_of([0] * (E - 2) + [5, 65]))
    v.launch([dp.data_ptr(), dq.data_ptr(), off.data_ptr()], d.data_ptr(), stream=devmem.current_stream())
    torch.cuda.synchronize()
    assert bool((d[:-2] == 0).all())
    some = slice(0, J, 101)
    close(d[-1, :, some].cpu(), p[5:].double().t() @ q[5:, some].double(), p[5:].double().abs().t() @ q[5:, some].double().abs(), 65, "f32")
    del d
    if code == 64128:
        x = torch.zeros(330000, 8192, dtype=torch.bfloat16, device="cuda")
        x[-1] = dp[0]
        w, y, s = torch.ones(8192, dtype=torch.bfloat16, device="cuda"), torch.full((330000, 8192), 0x55, dtype=torch.uint8, device="cuda"), torch.empty(330000, 64, device="cuda")
        n.launch([x.data_ptr(), w.data_ptr()], [y.data_ptr(), s.data_ptr(), None], stream=devmem.current_stream())
        torch.cuda.synchronize()
        assert bool((y[:-1] == 0).all())
        yv = p[0].double() / (p[0].double().square().mean() + 1e-6).sqrt()
        wide = s[-1].cpu().double().repeat_interleave(128)
        got = y[-1].cpu().view(TYPES["f8"]).double() * wide
        assert bool(((got - yv).abs() <= yv.abs() * (HALF_STEP["f8"] + 1e-5) * 1.01 + wide * 2.0 ** -10 * 1.01).all())


def test_infinities_and_nan_stay_in_their_rows():
    v = variant(B.grouped_gemm_op(2, 40, 64, 128, True, "bf16"))
    if v is None:
        return
    g = rng(4)
    a, b = normal(g, 40, 128).bfloat16(), normal(g, 2, 64, 128).bfloat16()
    clean = launch_twice(v, [dev(a), dev(b), dev(offsets_of([18, 22]))], [((40, 64), torch.bfloat16)])[0]
    a[5, 7], a[17, 3], a[18, 0] = float("nan"), float("inf"), float("-inf")
    dirty = launch_twice(v, [dev(a), dev(b), dev(offsets_of([18, 22]))], [((40, 64), torch.bfloat16)])[0]
    rows = [r for r in range(40) if r not in (5, 17, 18)]
    assert torch.equal(clean[rows], dirty[rows])
    assert not bool(torch.isfinite(dirty[[5, 17, 18]].float()).any())


# ---------------------------------------------------------------- gradient of the experts' matrices

@pytest.mark.parametrize("kind,out", [("bf16", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("counts,ahead,behind,I,J", [([1], 0, 0, 8, 8), ([0, 3, 0], 1, 2, 64, 40), ([64, 65, 63, 1, 0, 128], 0, 5, 136, 264), ([200, 7], 3, 0, 264, 520), ([2] * 20, 0, 0, 24, 136)])
@pytest.mark.parametrize("code", [0, 64128, 128128, 256256])
def test_weight_gradient(counts, ahead, behind, I, J, kind, out, code):
    check_wgrad(counts, ahead, behind, I, J, kind, out, code)


@pytest.mark.parametrize("I,J", [(7, 9), (33, 64), (64, 35)])
def test_weight_gradient_of_odd_sizes(I, J):
    check_wgrad([5, 0, 70], 1, 1, I, J, "bf16", "f32", 0)


def check_wgrad(counts, ahead, behind, I, J, kind, out, code):
    E, T = len(counts), ahead + sum(counts) + behind
    v = variant(B.grouped_wgrad_op(E, T, I, J, kind, out), code)
    if v is None:
        return
    g = rng(I + J + T)
    p, q = normal(g, T, I).to(TYPES[kind]), normal(g, T, J).to(TYPES[kind])
    off = offsets_of(counts, ahead)
    pv, qv = p.double(), q.double()
    for x in (p, q):
        x[:ahead] = float("nan")
        x[T - behind:] = float("nan")
    (d,) = launch_twice(v, [dev(p), dev(q), dev(off)], [((E, I, J), TYPES[out])])
    for e in range(E):
        rows = slice(int(off[e]), int(off[e + 1]))
        close(d[e], pv[rows].t() @ qv[rows], pv[rows].t().abs() @ qv[rows].abs(), max(1, counts[e]), out)


def test_gradients_are_those_of_the_product():
    """loss = sum(C * G): the gradient of A is the product with B read the other way, that of B the weights' gradient.  Against the formula
    (above) and, here, against differences of the product itself along a direction."""
    E, T, N, K = 3, 90, 64, 96
    f = variant(B.grouped_gemm_op(E, T, N, K, True, "f16", "f32"))
    da = variant(B.grouped_gemm_op(E, T, K, N, False, "f16", "f32"))
    db = variant(B.grouped_wgrad_op(E, T, N, K, "f16", "f32"))
    if f is None:
        return
    g = rng(12)
    off = dev(offsets_of([40, 0, 50]))

    # multiples of 1/8 up to 1: a step of 1/8 along a direction of signs is exact in fp16, and so are the sums in fp32
    def grid(*shape):
        return (torch.randint(-8, 9, shape, generator=g).float() / 8).half()

    a, b, G = grid(T, K), grid(E, N, K), grid(T, N)
    ua, ub = (torch.randint(0, 2, s, generator=g).half() * 2 - 1 for s in ((T, K), (E, N, K)))

    def loss(a, b):
        (c,) = launch_twice(f, [dev(a), dev(b), off], [((T, N), torch.float32)])
        return float((c.double() * G.double()).sum())

    (ga,) = launch_twice(da, [dev(G), dev(b), off], [((T, K), torch.float32)])
    (gb,) = launch_twice(db, [dev(G), dev(a), off], [((E, N, K), torch.float32)])
    h = 0.125
    # the loss is linear in each of A and B: the central difference is the derivative
    assert abs((loss(a + h * ua, b) - loss(a - h * ua, b)) / (2 * h) - float((ga.double() * ua.double()).sum())) < 1e-6
    assert abs((loss(a, b + h * ub) - loss(a, b - h * ub)) / (2 * h) - float((gb.double() * ub.double()).sum())) < 1e-6


# ---------------------------------------------------------------- RMS norm

def rms_definition(x, w, r, eps, kind):
    h = x.double() if r is None else (x.float() + r.float()).to(TYPES[kind]).double()
    return h, h / (h.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("f8", [True, False])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("M,N,code", [(1, 1, 0), (1, 4096, 0), (3, 127, 1), (2, 129, 2), (5, 640, 4), (7, 2050, 1), (9, 1000, 16), (600, 264, 0), (2, 9001, 2), (1, 40000, 0), (1500, 24, 1)])
def test_rms_norm(M, N, code, kind, f8, residual):
    v = variant(B.rms_norm_op(M, N, kind, "f8" if f8 else kind, residual=residual, eps=1e-5), code)
    if v is None:
        return
    g = rng(M + N)
    x, w, r = normal(g, M, N).to(TYPES[kind]), (1 + normal(g, N, scale=0.2)).to(TYPES[kind]), normal(g, M, N, scale=3.0).to(TYPES[kind]) if residual else None
    blocks = -(-N // 128)
    y, s, h = launch_twice(v, [dev(x), dev(w), dev(r)], [((M, N), TYPES["f8" if f8 else kind]), ((M, blocks), torch.float32) if f8 else None,
                                                        ((M, N), TYPES[kind]) if residual else None])
    hv, yv = rms_definition(x, w, r, 1e-5, kind)
    if residual:
        assert torch.equal(h.double(), hv)  # one rounding, the same
    # the mean of N squares in fp32 is off by at most N 2^-24 of itself (half of that after the root); quotient, root, two products and
    # their roundings add less than 8 steps
    rel = (N / 2 + 8) * 2.0 ** -24
    if not f8:
        assert bool(((y.double() - yv).abs() <= yv.abs() * (rel + HALF_STEP[kind]) * 1.01 + 2.0 ** -25).all())
        return
    pad = torch.nn.functional.pad(yv, (0, blocks * 128 - N)).view(M, blocks, 128)
    sv = pad.abs().amax(-1) / 448
    assert bool(((s.double() - sv).abs() <= sv * (rel + 2.0 ** -23) + 2.0 ** -126).all())
    wide = s.double().repeat_interleave(128, 1)[:, :N]
    # the nearest 8-bit float: half a step of the value, or of the smallest subnormal (2^-9) times the scale
    tol = yv.abs() * (HALF_STEP["f8"] + 4 * rel) * 1.01 + wide * 2.0 ** -10 * 1.01
    assert bool(((y.double() * wide - yv).abs() <= tol).all())


def test_rms_norm_in_place_strided_and_several_instances():
    M, N, R = 5, 200, 3
    v = variant(B.rms_norm_op(M, N, "bf16", "bf16"))
    s = variant(B.rms_norm_op(M, N, "f16", "f16", residual=False, a_strides=[0, 301, 1]))
    if v is None:
        return
    g = rng(8)
    x, w, r = normal(g, R, M, N).bfloat16(), normal(g, R, N).bfloat16(), normal(g, R, M, N).bfloat16()
    y, _, h = launch_twice(v, [dev(x), dev(w), dev(r)], [((R, M, N), torch.bfloat16), None, ((R, M, N), torch.bfloat16)], instances=R)
    hv, yv = rms_definition(x, w[:, None], r, 1e-6, "bf16")
    assert torch.equal(h.double(), hv) and bool(((y.double() - yv).abs() <= yv.abs() * 2.0 ** -8 * 1.02).all())
    for mine in (0, 2):  # H over X, H over R
        ts = [dev(x), dev(w), dev(r)]
        o = torch.empty_like(ts[0])
        v.launch([t.data_ptr() for t in ts], [o.data_ptr(), None, ts[mine].data_ptr()], instances=R, stream=devmem.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(ts[mine].cpu(), h) and torch.equal(o.cpu(), y)
    # rows 301 elements apart that start at any element
    flat = torch.full((7 + R * (4 * 301 + N),), float("nan"), dtype=torch.float16)
    x = normal(g, R, M, N).half()
    for i in range(R):
        torch.as_strided(flat, (M, N), (301, 1), 7 + i * (4 * 301 + N)).copy_(x[i])
    w = normal(g, R, N).half()
    d, dw = dev(flat), dev(w)
    o = torch.empty(R, M, N, dtype=torch.float16, device="cuda")
    s.launch([d.data_ptr() + 14, dw.data_ptr()], o.data_ptr(), instances=R, stream=devmem.current_stream())
    torch.cuda.synchronize()
    _, yv = rms_definition(x, w[:, None], None, 1e-6, "f16")
    assert bool(((o.cpu().double() - yv).abs() <= yv.abs() * 2.0 ** -11 * 1.02 + 2.0 ** -25).all())


@pytest.mark.parametrize("M,N,code", [((4 << 20) + 9, 16, 1), ((1 << 20) + 300, 72, 4)])
def test_rms_norm_of_more_rows_than_workgroups(M, N, code):
    v = variant(B.rms_norm_op(M, N, "bf16"), code)
    if v is None:
        return
    g = torch.Generator(device="cuda").manual_seed(71)
    x, r, w = (torch.randn(*s, generator=g, device="cuda").bfloat16() for s in ((M, N), (M, N), (N,)))
    y, h = torch.empty_like(x), torch.empty_like(x)
    v.launch([x.data_ptr(), w.data_ptr(), r.data_ptr()], [y.data_ptr(), None, h.data_ptr()], stream=devmem.current_stream())
    hv = (x.float() + r.float()).bfloat16()
    assert torch.equal(h, hv)
    yv = hv.double() * (hv.double().square().mean(1, keepdim=True) + 1e-6).rsqrt() * w.double()
    assert bool(((y.double() - yv).abs() <= yv.abs() * 2.0 ** -8 * 1.01 + 1e-37).all())


def test_rms_norm_of_zeros_nan_and_large_values():
    M, N = 6, 256
    v = variant(B.rms_norm_op(M, N, "f32", "f8", residual=False, eps=0))
    e = variant(B.rms_norm_op(M, N, "f32", "f8", residual=False, eps=1e-6))
    if v is None:
        return
    x = normal(rng(2), M, N)
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 200] = float("inf")
    x[4] *= 1e15
    x[5, :128] = 0
    y, s, _ = launch_twice(e, [dev(x), dev(torch.ones(N)), None], [((M, N), TYPES["f8"]), ((M, 2), torch.float32), None])
    y, s = y.float(), s.float()
    assert bool((y[1] == 0).all()) and bool((s[1] == 2.0 ** -126).all()) and bool((y[5, :128] == 0).all()) and float(s[5, 0]) == 2.0 ** -126
    assert bool(torch.isnan(y[2]).all()) and bool(torch.isnan(s[2]).all())
    # an infinite mean: finite values become 0, the infinity NaN, and with it its block
    assert bool((y[3, :128] == 0).all()) and bool(torch.isnan(y[3, 128:]).all())
    for r in (0, 4):
        assert bool(torch.isfinite(y[r]).all()) and float(y[r].abs().max()) == 448
    y, s, _ = launch_twice(v, [dev(x), dev(torch.ones(N)), None], [((M, N), TYPES["f8"]), ((M, 2), torch.float32), None])
    assert bool(torch.isnan(y[1].float()).all())  # 0 / 0, as the definition without eps says


# ---------------------------------------------------------------- together, and the ways of calling

def test_norm_feeds_products():
    """A quantised layer as a model runs it: residual and norm into 8-bit floats with scales, the shared product and the experts' products on
    them, on another stream."""
    M, N, K = 96, 144, 256
    norm, dense = variant(B.rms_norm_op(M, K, "bf16", "f8")), variant(B.scaled_gemm_op(M, N, K, "bf16"))
    experts = variant(B.grouped_gemm_op(4, M, N, K, True, "f8", "bf16"))
    if norm is None:
        return
    g = rng(21)
    x, w, r = dev(normal(g, M, K).bfloat16()), dev((1 + normal(g, K, scale=0.1)).bfloat16()), dev(normal(g, M, K).bfloat16())
    b, sb, bv = f8_and_scales(normal(g, 4, N, K, scale=0.2), 128)
    b, sb, off = dev(b), dev(sb), dev(offsets_of([30, 0, 50, 16]))
    y = torch.empty(M, K, dtype=TYPES["f8"], device="cuda")
    s, h = torch.empty(M, 2, device="cuda"), torch.empty_like(x)
    c, ce = (torch.zeros(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        at = devmem.current_stream()
        norm.launch([x.data_ptr(), w.data_ptr(), r.data_ptr()], [y.data_ptr(), s.data_ptr(), h.data_ptr()], stream=at)
        dense.launch([y.data_ptr(), b.data_ptr(), s.data_ptr(), sb.data_ptr()], c.data_ptr(), stream=at)
        experts.launch([y.data_ptr(), b.data_ptr(), off.data_ptr(), s.data_ptr(), sb.data_ptr()], ce.data_ptr(), stream=at)
    stream.synchronize()
    yv = y.cpu().double() * s.cpu().double().repeat_interleave(128, 1)
    close(c.cpu(), yv @ bv[0].t(), yv.abs() @ bv[0].abs().t(), 8, "bf16", f8=True)
    e = torch.tensor([0] * 30 + [2] * 50 + [3] * 16)
    want = torch.stack([yv[t] @ bv[e[t]].t() for t in range(M)])
    close(ce.cpu(), want, torch.stack([yv[t].abs() @ bv[e[t]].abs().t() for t in range(M)]), 8, "bf16", f8=True)


def test_captured_launches_follow_their_offsets():
    """A graph of the four operators, replayed with other offsets and inputs and the program's own work in between."""
    E, T, N, K = 4, 130, 128, 128
    ops = [variant(B.rms_norm_op(T, K, "bf16", "f8")), variant(B.grouped_gemm_op(E, T, N, K, True, "f8", "bf16")), variant(B.grouped_gemm_op(E, T, K, N, False, "bf16")),
           variant(B.grouped_wgrad_op(E, T, N, K, "bf16", "f32"))]
    if ops[0] is None:
        return
    for v in ops:
        v.prepare()
    g = rng(31)
    x, r, w = dev(normal(g, T, K).bfloat16()), dev(normal(g, T, K).bfloat16()), dev(torch.ones(K).bfloat16())
    b, sb, _ = f8_and_scales(normal(g, E, N, K), 128)
    b, sb, wb = dev(b), dev(sb), dev(normal(g, E, N, K).bfloat16())
    off = dev(offsets_of([30, 40, 0, 60]))
    y, s, h = torch.empty(T, K, dtype=TYPES["f8"], device="cuda"), torch.empty(T, 1, device="cuda"), torch.empty_like(x)
    c, dx, dw = torch.zeros(T, N, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, K, dtype=torch.bfloat16, device="cuda"), torch.zeros(E, N, K, device="cuda")

    def step():
        at = devmem.current_stream()
        ops[0].launch_static([x.data_ptr(), w.data_ptr(), r.data_ptr()], [y.data_ptr(), s.data_ptr(), h.data_ptr()], stream=at)
        ops[1].launch_static([y.data_ptr(), b.data_ptr(), off.data_ptr(), s.data_ptr(), sb.data_ptr()], c.data_ptr(), stream=at)
        ops[2].launch_static([c.data_ptr(), wb.data_ptr(), off.data_ptr()], dx.data_ptr(), stream=at)
        ops[3].launch_static([c.data_ptr(), h.data_ptr(), off.data_ptr()], dw.data_ptr(), stream=at)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k, counts in enumerate([[30, 40, 0, 60], [0, 0, 130, 0], [1, 2, 3, 4], [65, 0, 0, 65]]):
        off.copy_(offsets_of(counts))
        x.copy_(normal(g, T, K).bfloat16())
        got = []
        for run in (graph.replay, step):
            for t in (c, dx, dw):
                t.fill_(3)
            run()
            torch.cuda.synchronize()
            got.append([t.cpu().clone() for t in (y.view(torch.uint8), s, h, c, dx, dw)])
        assert all(torch.equal(p, q) for p, q in zip(*got)), "replay %d" % k
        assert bool((got[0][3][sum(counts):] == 3).all())


def test_two_streams_at_once():
    v = variant(B.grouped_gemm_op(2, 300, 256, 512))
    if v is None:
        return
    g = rng(41)
    off = dev(offsets_of([100, 200]))
    sets = [(dev(normal(g, 300, 512).bfloat16()), dev(normal(g, 2, 256, 512).bfloat16())) for _ in range(2)]
    alone = []
    for a, b in sets:
        c = torch.empty(300, 256, dtype=torch.bfloat16, device="cuda")
        v.launch([a.data_ptr(), b.data_ptr(), off.data_ptr()], c.data_ptr(), stream=devmem.current_stream())
        torch.cuda.synchronize()
        alone.append(c)
    streams, out = [torch.cuda.Stream() for _ in sets], [torch.empty_like(alone[0]) for _ in sets]
    torch.cuda.synchronize()
    for _ in range(10):
        for (a, b), st, o in zip(sets, streams, out):
            v.launch([a.data_ptr(), b.data_ptr(), off.data_ptr()], o.data_ptr(), stream=st.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(alone, out))


def test_measure_and_search():
    """ms_measure and ms_search take an operator's further inputs and outputs from one block."""
    E, T, N, K = 2, 60, 128, 256
    op = B.grouped_gemm_op(E, T, N, K, True, "f8", "bf16")
    norm = B.rms_norm_op(T, K, "bf16", "f8")
    v, n = variant(op), variant(norm)
    if v is None:
        return
    g = rng(51)
    a, sa, _ = f8_and_scales(normal(g, T, K), 1)
    b, sb, _ = f8_and_scales(normal(g, E, N, K), 128)
    block = torch.zeros(-(-op.tensor_bytes(3) // 256) * 256 + op.tensor_bytes(4), dtype=torch.uint8)
    block[:op.tensor_bytes(3)] = sa.reshape(-1).view(torch.uint8)
    block[-op.tensor_bytes(4):] = sb.reshape(-1).view(torch.uint8)
    ins = [dev(a), dev(b), dev(offsets_of([20, 40])), dev(block)]
    c = torch.zeros(T, N, dtype=torch.bfloat16, device="cuda")
    m = v.measure([([t.data_ptr() for t in ins], c.data_ptr())], stream=devmem.current_stream())
    assert 0 < m.min_us < 1e5 and m.flop == 2 * T * N * K
    want = torch.empty_like(c)
    sa, sb = dev(sa), dev(sb)
    v.launch([t.data_ptr() for t in ins[:3]] + [sa.data_ptr(), sb.data_ptr()], want.data_ptr(), stream=devmem.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(c, want)
    cfg = B.search_cfg_default()
    cfg.trials, cfg.init_population = 4, 4
    res = B.search(op, op.space(), cfg, [([t.data_ptr() for t in ins], c.data_ptr())], stream=devmem.current_stream())
    assert res.n_measured >= 2 and res.n_failed == 0 and torch.equal(c, want)
    # the norm: Y, S and H in one block
    x, w, r = dev(normal(g, T, K).bfloat16()), dev(torch.ones(K).bfloat16()), dev(normal(g, T, K).bfloat16())
    up = lambda x: -(-x // 256) * 256  # noqa: E731
    places = [0, up(norm.tensor_bytes(-1)), up(norm.tensor_bytes(-1)) + up(norm.tensor_bytes(-2))]
    out = torch.zeros(places[2] + norm.tensor_bytes(-3), dtype=torch.uint8, device="cuda")
    n.measure([([x.data_ptr(), w.data_ptr(), r.data_ptr()], out.data_ptr())], stream=devmem.current_stream())
    y, s, h = (torch.empty(norm.tensor_bytes(i), dtype=torch.uint8, device="cuda") for i in (-1, -2, -3))
    n.launch([x.data_ptr(), w.data_ptr(), r.data_ptr()], [y.data_ptr(), s.data_ptr(), h.data_ptr()], stream=devmem.current_stream())
    torch.cuda.synchronize()
    for at, t in zip(places, (y, s, h)):
        assert torch.equal(out[at:at + t.numel()], t)


def test_rms_norm_divides_by_its_scales():
    """Rows of ones have a norm of one, so that Y is W in 8-bit floats: values at and next to the ties of each block's scale, of all magnitudes,
    come out as the fp32 quotient W / S rounds."""
    blocks = 4096
    N = blocks * 128
    v = variant(B.rms_norm_op(1, N, "f32", "f8", residual=False, eps=0))
    if v is None:
        return
    g = rng(77)
    most = 448 * torch.ldexp(1 + torch.rand(blocks, generator=g), torch.randint(-132, 116, (blocks,), generator=g))
    most[:256] = 448 * torch.ldexp(torch.tensor(1.0), torch.randint(-126, 116, (256,), generator=g))  # powers of two
    s = (most / 448).clamp_min(2.0 ** -126)
    normal_ties = torch.ldexp((torch.randint(8, 16, (blocks, 64), generator=g) * 2 + 1).float(), torch.randint(-10, 5, (blocks, 64), generator=g))
    subnormal_ties = (torch.randint(0, 8, (blocks, 63), generator=g) * 2 + 1) * 2.0 ** -10
    w = torch.cat([normal_ties, subnormal_ties], 1).clamp(max=440) * s[:, None]
    w = (w.view(torch.int32) + torch.randint(-3, 4, w.shape, generator=g, dtype=torch.int32)).clamp_min(0).view(torch.float32)
    w = torch.cat([torch.minimum(w, most[:, None]), most[:, None]], 1)
    w[-1, 5] = float("inf")  # its scale too: finite values become 0, the infinity NaN
    s = (w.amax(1) / 448).clamp_min(2.0 ** -126)
    w = w * (torch.randint(0, 2, w.shape, generator=g) * 2 - 1)
    want = (w / s[:, None]).to(TYPES["f8"])
    assert int(((w * (1 / s)[:, None]).to(TYPES["f8"]).view(torch.uint8) != want.view(torch.uint8)).sum()) > 10000  # a reciprocal does not do
    y, got, _ = launch_twice(v, [dev(torch.ones(1, N)), dev(w.reshape(-1)), None], [((1, N), TYPES["f8"]), ((1, blocks), torch.float32), None])
    assert torch.equal(got[0], s)
    y = y.view(blocks, 128)
    nan = torch.isnan(want.float())
    assert torch.equal(torch.isnan(y.float()), nan) and int(nan.sum()) == 1
    off = (y.view(torch.uint8) != want.view(torch.uint8)) & ~nan
    assert not bool(off.any()), "%d values off, the first %r / %r" % (int(off.sum()), float(w[off][0]), float(s[off.nonzero()[0, 0]]))


@pytest.mark.parametrize("code", [16032, 64128, 256256])
def test_scaled_products_of_unlike_magnitudes(code):
    """The bound that ms.h gives for the 8-bit instruction: of each eight products in a row what lies below 2^-13 of the largest is cut off, 7 times at most;
    16 sums of eights in fp32, truncated, are off by 16 * 2^-23 of their magnitudes, the blocks by less."""
    M, N, K = 70, 136, 384
    v = variant(B.scaled_gemm_op(M, N, K, "f32"), code)
    if v is None:
        return
    g = rng(88)
    a, b = ((normal(g, n, K) * 2.0 ** torch.randint(-8, 7, (n, K), generator=g)).clamp(-448, 448).to(TYPES["f8"]) for n in (M, N))
    sa, sb = torch.rand(M, 3, generator=g) + 0.5, torch.rand(2, 3, generator=g) + 0.5
    av = a.double() * sa.double().repeat_interleave(128, 1)
    bv = b.double() * sb.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)
    (c,) = launch_twice(v, [dev(x) for x in (a, b, sa, sb)], [((M, N), torch.float32)])
    products = (av[:, None] * bv[None]).abs()
    tol = products.view(M, N, K // 8, 8).amax(-1).sum(-1) * 7 * 2.0 ** -13 + products.sum(-1) * 2.0 ** -18
    off = (c.double() - av @ bv.t()).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


@pytest.mark.parametrize("code", [0, 16016, 64128, 128128, 256256])
def test_experts_of_several_instances(code):
    """Consecutive copies of all tensors, offsets among them, of products both ways round and of the gradient."""
    R, E, T, N, K = 3, 4, 320, 264, 136
    counts = [[100, 0, 200, 3], [0, 0, 0, 320], [1, 130, 64, 125]]
    ops = [variant(B.grouped_gemm_op(E, T, N, K, by_k, "bf16"), code if by_k or code != 16016 else 64128) for by_k in (True, False)]
    w = variant(B.grouped_wgrad_op(E, T, N, K, "f16", "f32"), code if code != 16016 else 64128)
    if w is None:
        return
    g = rng(91)
    off = torch.stack([offsets_of(c) for c in counts])
    a, b = normal(g, R, T, K).bfloat16(), normal(g, R, E, N, K).bfloat16()
    p, q = normal(g, R, T, N).half(), normal(g, R, T, K).half()
    for v, by_k in zip(ops, (True, False)):
        (c,) = launch_twice(v, [dev(a), dev(b if by_k else b.transpose(2, 3).contiguous()), dev(off)], [((R, T, N), torch.bfloat16)], instances=R)
        for r in range(R):
            for e in range(E):
                rows = slice(int(off[r, e]), int(off[r, e + 1]))
                close(c[r, rows], a[r, rows].double() @ b[r, e].double().t(), a[r, rows].double().abs() @ b[r, e].double().abs().t(), K, "bf16")
            assert bool((c[r, int(off[r, -1]):] == 7).all())
    (d,) = launch_twice(w, [dev(p), dev(q), dev(off)], [((R, E, N, K), torch.float32)], instances=R)
    for r in range(R):
        for e in range(E):
            rows = slice(int(off[r, e]), int(off[r, e + 1]))
            close(d[r, e], p[r, rows].double().t() @ q[r, rows].double(), p[r, rows].double().abs().t() @ q[r, rows].double().abs(), max(1, counts[r][e]), "f32")


def test_rms_norm_in_place_beyond_the_registers():
    """H over X and over R where most of a row is read again from H."""
    M, N = 3, 40000
    for kind in ("bf16", "f32"):
        v = variant(B.rms_norm_op(M, N, kind, "f8"))
        if v is None:
            continue
        g = rng(95)
        x, w, r = normal(g, M, N).to(TYPES[kind]), (1 + normal(g, N, scale=0.1)).to(TYPES[kind]), normal(g, M, N).to(TYPES[kind])
        want = launch_twice(v, [dev(x), dev(w), dev(r)], [((M, N), TYPES["f8"]), ((M, 313), torch.float32), ((M, N), TYPES[kind])])
        for mine in (0, 2):
            ts = [dev(x), dev(w), dev(r)]
            y, s = torch.empty(M, N, dtype=TYPES["f8"], device="cuda"), torch.empty(M, 313, device="cuda")
            v.launch([t.data_ptr() for t in ts], [y.data_ptr(), s.data_ptr(), ts[mine].data_ptr()], stream=devmem.current_stream())
            torch.cuda.synchronize()
            assert torch.equal(y.cpu().view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(s.cpu(), want[1]) and torch.equal(ts[mine].cpu(), want[2])


def test_rms_norm_of_more_instances_than_a_grid_has_rows():
    M, N, R = 1, 24, 70000
    v = variant(B.rms_norm_op(M, N, "f32", "f32", residual=False))
    if v is None:
        return
    g = rng(96)
    x, w = normal(g, R, M, N), normal(g, R, N)
    (y, _, _) = launch_twice(v, [dev(x), dev(w), None], [((R, M, N), torch.float32), None, None], instances=R)
    _, yv = rms_definition(x, w[:, None], None, 1e-6, "f32")
    assert bool(((y.double() - yv).abs() <= yv.abs() * (N / 2 + 9) * 2.0 ** -24 * 1.01 + 1e-37).all())
