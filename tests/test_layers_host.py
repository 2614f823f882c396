"""Layers of language models on the host: what is accepted and refused, the tiles that the rules choose, coverage, the trace that leaves
all decisions to them.  No GPU."""
import os
import subprocess

import numpy as np
import pytest

from paper_2205_13603_amd import binding as B, devmem

OPS = {
    "norm": lambda: B.rms_norm_op(37, 1000, "bf16", "f8"),
    "plain norm": lambda: B.rms_norm_op(3, 129, "f32", residual=False),
    "scaled": lambda: B.scaled_gemm_op(77, 200, 272),
    "few": lambda: B.scaled_gemm_op(4, 200, 256, "f32"),
    "grouped": lambda: B.grouped_gemm_op(5, 301, 136, 64),
    "grouped f8": lambda: B.grouped_gemm_op(5, 301, 136, 64, in_dtype="f8"),
    "input gradient": lambda: B.grouped_gemm_op(5, 301, 136, 64, False, "f16"),
    "odd": lambda: B.grouped_gemm_op(5, 301, 131, 67, False, "f16"),
    "wgrad": lambda: B.grouped_wgrad_op(3, 90, 136, 72, "f16", "f32"),
}


def refused(code, f, *args, **kw):
    with pytest.raises(B.MsError) as e:
        f(*args, **kw)
    assert e.value.code == code, str(e.value)


@pytest.mark.parametrize("name", sorted(OPS))
def test_every_block_covers_outputs_and_reduction_once(name):
    op = OPS[name]()
    space = op.space()
    assert space.n_slots == 1 and space.slots[0].slot_id == B.SLOT_BLOCK and space.slots[0].candidates[0] == 0
    d = op.desc()
    size = {B.F32: 4, B.F16: 2, B.BF16: 2, B.F8E4M3: 1}[d.out_dtype]
    seen = set()
    for c in range(space.slots[0].n_candidates):
        if not space.slots[0].weight[c]:
            with pytest.raises(B.MsError):
                B.trace_validate(op, space, B.make_trace(space, [[space.slots[0].candidates[c]]]))
            continue
        t = B.make_trace(space, [[space.slots[0].candidates[c]]])
        p = B.trace_validate(op, space, t)
        assert (B.variant_coverage(op, p, op.tensor_bytes(-1) // size) == 1).all()
        assert (B.variant_reduction_coverage(op, p) == 1).all()
        assert np.isfinite(B.variant_features(op, p)).all()
        assert p.threads == 64 * p.waves <= 1024 and p.lds_bytes <= 160 << 10 and p.rfactor == 1
        text = B.trace_to_text(op, space, t)
        assert "body=r" in text and B.trace_from_text(space, text).decisions() == t.decisions()
        seen.add(p.body_tile)
    default = B.default_trace(space)
    assert default.decisions() == [(B.SLOT_BLOCK, [0])] and B.trace_validate(op, space, default).body_tile in seen


def test_sizes_do_not_select_code():
    def key(op):
        space = op.space()
        p = B.trace_validate(op, space, B.make_trace(space, [[128128]]))
        return p.key, B.variant_kernel_text(op, p)

    a = key(B.grouped_gemm_op(5, 301, 136, 64))
    assert a == key(B.grouped_gemm_op(2, 77, 1032, 1024, a_strides=[0, 2048, 1]))
    # launches of more workgroups than compute units take the kernel of which two fit beside each other
    b = key(B.grouped_gemm_op(64, 30100, 4096, 1024))
    assert a[0] != b[0] and b == key(B.grouped_gemm_op(16, 9000, 2048, 512, a_strides=[0, 2048, 1]))
    assert a[0] != key(B.grouped_gemm_op(5, 301, 136, 64, False))[0]
    assert a[0] != key(B.grouped_gemm_op(5, 301, 136, 64, in_dtype="f16"))[0]
    assert a[0] != key(B.grouped_gemm_op(5, 301, 136, 64, out_dtype="f32"))[0]
    assert a[0] != key(B.grouped_wgrad_op(5, 301, 136, 64))[0]


def test_work_loops_and_tensors():
    op = B.grouped_gemm_op(4, 100, 256, 384, in_dtype="f8")
    assert op.work() == (2 * 100 * 256 * 384, 100 * 384 + 4 * 256 * 384 + 100 * 256 * 2 + 4 * 3 * (100 + 4 * 2) + 4 * 5)
    assert [op.tensor_bytes(i) for i in range(-1, 5)] == [100 * 256 * 2, 100 * 384, 4 * 256 * 384, 20, 100 * 3 * 4, 4 * 2 * 3 * 4]
    assert [n for n, _, _ in op.loops()] == ["i", "j", "k"]
    op = B.rms_norm_op(10, 300, "f16", "f8")
    assert [op.tensor_bytes(i) for i in (-3, -2, -1, 0, 1, 2)] == [6000, 120, 3000, 6000, 600, 6000]
    refused(B.MS_ERR_BAD_ARG, B.rms_norm_op(10, 300, "f16", residual=False).tensor_bytes, 2)
    assert [n for n, _, _ in op.loops()] == ["i", "k"]
    op = B.grouped_wgrad_op(4, 100, 64, 32, "bf16", "f32")
    assert op.work() == (2 * 100 * 64 * 32, 100 * 96 * 2 + 4 * 64 * 32 * 4 + 20)
    assert [n for n, _, _ in op.loops()] == ["e", "i", "j", "k"]
    d = B.grouped_gemm_op(4, 100, 256, 384, False).desc()
    assert list(d.a_strides) == [0, 384, 1] and list(d.b_strides) == [256 * 384, 256, 1]


def test_refused_operators():
    bad, no = B.MS_ERR_BAD_ARG, B.MS_ERR_UNSUPPORTED
    refused(no, B.scaled_gemm_op, 4, 8, 16, "i32")
    refused(no, B.Op, B.OP_SCALED_GEMM, "f16", "f16", [4, 8, 16])
    refused(no, B.Op, B.OP_SCALED_GEMM, "i8", "i32", [4, 8, 16])
    refused(bad, B.Op, B.OP_SCALED_GEMM, 9, "f16", [4, 8, 16])
    refused(bad, B.scaled_gemm_op, 0, 8, 16)
    refused(bad, B.Op, B.OP_SCALED_GEMM, "f8", "f16", [4, 8, 16, 1])
    refused(bad, B.scaled_gemm_op, 4, 8, 16, relu=True)
    refused(no, B.scaled_gemm_op, 4, 8, 16, b_strides=[0, 8, 1])           # columns of B contiguous
    refused(no, B.scaled_gemm_op, 4, 8, 16, a_strides=[0, 8, 1])           # rows overlap
    refused(no, B.scaled_gemm_op, 4, 8, 16, a_strides=[0, 32, 2])
    refused(bad, B.scaled_gemm_op, 4, 8, 16, a_strides=[0, -16, 1])
    refused(no, B.scaled_gemm_op, 4, 8, 16, a_strides=[0, (4 << 20) + 16, 1])
    refused(no, B.grouped_gemm_op, B.MAX_EXPERTS + 1, 8, 16, 16)
    refused(no, B.grouped_gemm_op, 2, 8, 16, 16, False, "f8")
    refused(no, B.grouped_gemm_op, 2, 8, 16, 16, True, "f16", "bf16")
    refused(no, B.grouped_gemm_op, 2, 8, 16, 16, True, "f32")
    refused(bad, B.grouped_gemm_op, 2, 8, 16, 16, b_strides=[100, 1, 16])  # matrices overlap
    refused(bad, B.grouped_gemm_op, 2, 1 << 31, 16, 16)
    refused(no, B.grouped_wgrad_op, 2, 8, 16, 16, "f8", "f16")
    refused(no, B.grouped_wgrad_op, 2, 8, 16, 16, a_strides=[0, 8, 1])
    refused(no, B.rms_norm_op, 4, 16, "f8")
    refused(no, B.rms_norm_op, 4, 16, "f16", "f32")
    refused(bad, B.rms_norm_op, 4, 16, a_strides=[0, 8, 1])
    refused(bad, B.rms_norm_op, 4, 16, b_strides=[0, 16, 1])
    refused(bad, B.Op, B.OP_RMS_NORM, "f16", "f16", [4, 16, -1])
    refused(bad, B.Op, B.OP_RMS_NORM, "f16", "f16", [4, 16, 0], has_bias=2)
    with pytest.raises(ValueError):
        B.rms_norm_op(4, 16, eps=-1)


def test_refused_traces_and_limits():
    op = B.grouped_gemm_op(5, 301, 136, 64, False)
    space = op.space()
    refused(B.MS_ERR_INVALID_TRACE, B.trace_validate, op, space, B.make_trace(space, [[16032]]))  # tiles of few rows need rows of k
    refused(B.MS_ERR_BAD_ARG, B.trace_validate, B.gemm_op(64, 64, 64), space, B.default_trace(space))
    refused(B.MS_ERR_BAD_ARG, B.trace_validate, B.rms_norm_op(4, 16), space, B.default_trace(space))
    refused(B.MS_ERR_UNSUPPORTED, B.default_trace, B.gemm_op(64, 64, 64).space())
    before = B.get_limits()
    try:
        for field, value in (("max_lds_bytes", 4096), ("max_threads", 128), ("max_acc_per_thread", 8)):
            lim = B.get_limits()
            setattr(lim, field, value)
            B.set_limits(lim)
            refused(B.MS_ERR_INVALID_TRACE, B.trace_validate, op, space, B.default_trace(space))
            B.set_limits(before)
    finally:
        B.set_limits(before)


def test_refused_launches():
    """Everything that a launch checks ahead of its first call of the GPU's runtime."""
    bad = B.MS_ERR_BAD_ARG

    def variant(op):
        space = op.space()
        return B.Variant(op, space, B.default_trace(space))

    at = 1 << 20
    v = variant(B.grouped_gemm_op(2, 8, 16, 16, in_dtype="f8"))
    ins = [at] * 5
    for i in range(5):
        refused(bad, v.launch, [None if k == i else at for k in range(5)], at)
        refused(bad, v.launch, [at + 2 if k == i else at for k in range(5)], at)
    refused(bad, v.launch, ins, None)
    refused(bad, v.launch, ins, at + 8)
    refused(bad, v.launch, ins, at, instances=0)
    refused(bad, v.launch, ins, at, instances=65536)
    v = variant(B.scaled_gemm_op(3, 5, 16))
    refused(bad, v.launch, [at] * 4, at, instances=2)  # copies of 30 bytes
    v = variant(B.rms_norm_op(4, 16, "bf16", "f8"))
    refused(bad, v.launch, [at, at, None], [at, at, at])
    refused(bad, v.launch, [at, at, at], [at, None, at])
    refused(bad, v.launch, [at, at, at], [at, at, None])
    refused(bad, v.launch, [at + 1, at, at], [at, at, at])
    refused(bad, v.launch, [at, at, at], [at, at + 2, at])
    with pytest.raises(ValueError):
        v.launch([at] * 9, [at])
    with pytest.raises(TypeError):
        v.launch([at] * 3, [at, "x", at])


def test_sampled_mutated_and_composed_spaces():
    for name, make in OPS.items():
        op = make()
        space = op.space()
        traces = {tuple(B.trace_sample_valid(op, space, 1, i).d[0].v)[0] for i in range(64)}
        assert len(traces) == sum(1 for c in range(space.slots[0].n_candidates) if space.slots[0].weight[c]), name
        composed, mask = B.space_compose(op, ["multi-level-tiling", "unroll"])
        assert mask == 0 and composed.n_slots == 1
        assert B.space_log10_size(space) > 0


def test_search_on_a_synthetic_latency_finds_the_block():
    op = OPS["grouped"]()
    cfg = B.search_cfg_default()
    cfg.trials, cfg.init_population, cfg.population, cfg.children = 16, 4, 4, 4
    res = B.search(op, op.space(), cfg, fake_latency=lambda p: 1.0 + abs(p.body_tile - 128128) / 1e5)
    p = B.trace_validate(op, op.space(), res.best_trace)
    assert p.body_tile == 128128


def test_launches_on_several_threads_and_devices(tmp_path):
    """Launches on a stand-in for HIP that keeps book of modules and devices, under the thread sanitizer: each call runs the kernel of its own
    device, loaded once, and what is not there or not aligned is refused before anything is launched."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "ms_layers")
    srcs = [os.path.join(root, "paper_2205_13603_amd", "csrc", f) for f in ("ms_core.cpp", "ms_interp.cpp", "ms_model.cpp", "ms_search.cpp", "ms_runtime.cpp")]
    r = subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-fsanitize=thread", "-D__HIP_PLATFORM_AMD__", "-D__align__(n)=", "-DHIP_SYMBOL(x)=(&x)", "-I", "/opt/rocm/include",
                        "-o", exe] + srcs + [os.path.join(root, "tests", "sanitize", "layer_driver.cpp"), "-lm", "-lpthread"],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-4000:]
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=600)
    assert r.returncode == 0 and "layer checks ok" in r.stdout, r.stdout[-6000:]


def test_scales_of_whole_tiles_are_read_before_their_place_is_taken(tmp_path):
    """The kernel's own arithmetic of the two places (ragged_schedule.h), walked phase by phase for 2 to 200 blocks of k."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "ms_scales")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-o", exe, os.path.join(root, "tests", "sanitize", "scales_driver.cpp")], check=True)
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60)
    assert r.returncode == 0 and "scales ok" in r.stdout, r.stdout


def test_the_sum_is_not_written_over_rows_further_apart():
    """H is dense: over an X of longer rows it would cover rows that other workgroups have yet to read.  What is allowed gets as far as the GPU's
    runtime, which is not there."""
    def norm(M, **kw):
        op = B.rms_norm_op(M, 16, "bf16", **kw)
        space = op.space()
        return B.Variant(op, space, B.default_trace(space))

    x, w, r, y = ((1 + i) << 20 for i in range(4))
    wide = dict(a_strides=[0, 24, 1])
    refused(B.MS_ERR_BAD_ARG, norm(4, **wide).launch, [x, w, r], [y, None, x])
    refused(B.MS_ERR_BAD_ARG, norm(4, **wide).launch, [x, w, r], [y, None, x], instances=2)
    if not devmem.gpu_available():
        for v, h in ((norm(4), x), (norm(4, a_strides=[0, 16, 1]), x), (norm(4, **wide), r), (norm(1, **wide), x)):
            refused(B.MS_ERR_HIP, v.launch, [x, w, r], [y, None, h])


@pytest.mark.parametrize("make,code", [
    (lambda: B.scaled_gemm_op(300, 500, 256), 16032), (lambda: B.scaled_gemm_op(300, 500, 256), 64128), (lambda: B.grouped_gemm_op(1, 700, 1500, 64), 128128),
    (lambda: B.grouped_wgrad_op(3, 90, 136, 200), 64128)])
def test_coverage_is_that_of_the_workgroups_there_are(make, code):
    """One workgroup fewer than the launch has leaves its tile without a visit."""
    op = make()
    space = op.space()
    p = B.trace_validate(op, space, B.make_trace(space, [[code]]))
    d = op.desc()
    n = op.tensor_bytes(-1) // {B.F32: 4, B.F16: 2, B.BF16: 2}[d.out_dtype]
    assert (B.variant_coverage(op, p, n) == 1).all()
    p.grid[0] -= 1
    counts = B.variant_coverage(op, p, n)
    assert counts.max() == 1 and 0 < (counts == 0).sum() <= p.block_m * p.block_n


@pytest.mark.parametrize("M,N,K", [(2900, 6000, 400), (2816, 9176, 272), (8492, 4104, 144), (100, 70, 256), (129, 70, 256), (128 * 7, 257, 256), (256 * 16 + 1, 256 * 16 - 3, 256),
                                   (256 * 33, 256 * 9, 144)])
def test_whole_tiles_halves_and_quarters_cover_each_result_once(M, N, K):
    op = B.scaled_gemm_op(M, N, K)
    space = op.space()
    p = B.trace_validate(op, space, B.make_trace(space, [[256256]]))
    assert (B.variant_coverage(op, p, M * N) == 1).all()


def test_tiles_of_gradients_cover_each_result_once():
    for E, I, J in ((24, 1032, 520), (3, 2048, 2048), (700, 24, 40), (1, 304, 4000)):
        op = B.grouped_wgrad_op(E, 100, I, J)
        space = op.space()
        for code in (64128, 128128, 256256):
            p = B.trace_validate(op, space, B.make_trace(space, [[code]]))
            assert (B.variant_coverage(op, p, E * I * J) == 1).all()


def test_an_eps_between_units_is_refused():
    for eps in (1e-13, 4e-13, 5e-13, 1.5e-12, 2.45e-11):
        with pytest.raises(ValueError):
            B.rms_norm_op(4, 16, eps=eps)
    for eps, units in ((0, 0), (1e-12, 1), (1e-6, 10 ** 6), (float(np.float32(1e-5)), 10 ** 7), (1.2345e-8, 12345), (1, 10 ** 12)):
        assert B.rms_norm_op(4, 16, eps=eps).desc().dims[2] == units


def test_coverage_refuses_the_parameters_of_another_operator():
    norm, product = B.rms_norm_op(8, 256), B.scaled_gemm_op(40, 32, 256)
    p, q = (B.trace_validate(op, op.space(), B.default_trace(op.space())) for op in (norm, product))
    for op, params, n in ((norm, q, 8 * 256), (product, p, 40 * 32), (B.gemm_op(40, 32, 64), q, 40 * 32)):
        refused(B.MS_ERR_BAD_ARG, B.variant_coverage, op, params, n)
        refused(B.MS_ERR_BAD_ARG, B.variant_reduction_coverage, op, params)
    for params, op, n in ((p, norm, 8 * 256), (q, product, 40 * 32)):
        params.body_tile = 0
        refused(B.MS_ERR_BAD_ARG, B.variant_coverage, op, params, n)
