"""Products in 8-bit integers on the host: what is accepted and refused, coverage, tensors.  No GPU."""
import pytest

from paper_2205_13603_amd import binding as B

OPS = {
    "dense": lambda: B.scaled_gemm_op(77, 201, 272, in_dtype="i8"),
    "deep": lambda: B.scaled_gemm_op(300, 500, 64, "f32", in_dtype="i8"),
    "few": lambda: B.scaled_gemm_op(4, 200, 256, "f32", in_dtype="i8"),
    "experts": lambda: B.grouped_gemm_op(5, 301, 137, 64, in_dtype="i8"),
    "odd": lambda: B.grouped_gemm_op(5, 301, 131, 67, in_dtype="i8"),
}


def refused(code, f, *args, **kw):
    with pytest.raises(B.MsError) as e:
        f(*args, **kw)
    assert e.value.code == code, str(e.value)


@pytest.mark.parametrize("name", sorted(OPS))
def test_every_block_covers_outputs_and_reduction_once(name):
    op = OPS[name]()
    space = op.space()
    seen = set()
    for c in range(space.slots[0].n_candidates):
        if not space.slots[0].weight[c]:
            continue
        p = B.trace_validate(op, space, B.make_trace(space, [[space.slots[0].candidates[c]]]))
        n = op.tensor_bytes(-1) // {B.F32: 4, B.F16: 2, B.BF16: 2}[op.desc().out_dtype]
        assert (B.variant_coverage(op, p, n) == 1).all() and (B.variant_reduction_coverage(op, p) == 1).all()
        assert p.block_k == 128 and p.lds_bytes <= 160 << 10
        seen.add(p.body_tile)
    assert seen == {64128} if name == "odd" else 256256 in seen and 16016 in seen


def test_tensors_and_work():
    op = B.scaled_gemm_op(100, 256, 384, in_dtype="i8")
    assert [op.tensor_bytes(i) for i in range(-1, 4)] == [100 * 256 * 2, 100 * 384, 256 * 384, 100 * 4, 256 * 4]
    assert op.work() == (2 * 100 * 256 * 384, 100 * 384 + 256 * 384 + 100 * 256 * 2 + 4 * (100 + 256))
    op = B.grouped_gemm_op(4, 100, 256, 384, in_dtype="i8")
    assert op.desc().out_dtype == B.BF16
    assert [op.tensor_bytes(i) for i in range(-1, 5)] == [100 * 256 * 2, 100 * 384, 4 * 256 * 384, 20, 100 * 4, 4 * 256 * 4]
    assert op.work() == (2 * 100 * 256 * 384, 100 * 384 + 4 * 256 * 384 + 100 * 256 * 2 + 4 * (100 + 4 * 256) + 20)


def test_refusals():
    no, bad = B.MS_ERR_UNSUPPORTED, B.MS_ERR_BAD_ARG
    for out in ("i8", "i32", "f8"):
        refused(no, B.scaled_gemm_op, 4, 8, 16, out, in_dtype="i8")
        refused(no, B.grouped_gemm_op, 2, 4, 8, 16, True, "i8", out)
    refused(no, B.grouped_gemm_op, 2, 8, 16, 16, False, "i8")               # columns of B contiguous
    refused(no, B.grouped_wgrad_op, 2, 8, 16, 16, "i8", "f32")
    refused(no, B.scaled_gemm_op, 4, 8, B.MAX_I8_DEPTH + 1, in_dtype="i8")  # sums beyond 32 bits
    B.scaled_gemm_op(4, 8, B.MAX_I8_DEPTH, in_dtype="i8")
    refused(no, B.scaled_gemm_op, 4, 8, 16, in_dtype="i8", b_strides=[0, 8, 1])
    op = B.scaled_gemm_op(4, 8, 32, in_dtype="i8")
    space = op.space()
    v = B.Variant(op, space, B.default_trace(space))
    at = 1 << 20
    for i in range(4):
        refused(bad, v.launch, [None if k == i else at for k in range(4)], at)
        refused(bad, v.launch, [at + 2 if k == i else at for k in range(4)], at)
    refused(bad, v.launch, [at] * 4, None)
    refused(bad, v.launch, [at] * 4, at + 8)
