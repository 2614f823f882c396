"""Persistent workgroups of 256 x 256 tiles that go on from one whole tile to the next, against the definitions in 64 bits; tolerances as in
test_gpu_layers.py.  Each test counts the whole tiles that the kernel makes of its sizes, two at least for every workgroup."""
import pytest
import torch

from paper_2205_13603_amd import binding as B, devmem
from test_gpu_layers import TYPES, close, offsets_of, variant

pytestmark = pytest.mark.gpu


def whole_tiles_each(rows, cols):
    """Whole tiles of each workgroup, at least, in a product of experts of `rows` rows by `cols` columns: those of more than half a tile's rows, without
    a last round that is made in quarters (40 hundredths of a tile's time each) because these end sooner."""
    grid = torch.cuda.get_device_properties(0).multi_processor_count
    nt = -(-cols // 256)
    whole = sum((r + 127) // 256 for r in rows) * nt
    halves = sum(r > (r + 127) // 256 * 256 for r in rows) * nt * 2
    rest = whole % grid
    if rest and -(-(4 * rest + halves) // grid) * 40 < 100 + -(-halves // grid) * 40:
        whole -= rest
    return whole // grid


def on_device(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return g, lambda *shape: torch.randn(*shape, generator=g, device="cuda")


def blocks_of(x, rows_per_scale, g):
    """[..., rows, cols] in 8-bit floats under scales of rows_per_scale x 128 that differ by a factor of up to 16 from block to block, and the
    values these stand for in 64 bits."""
    rows, cols = x.shape[-2:]
    rb, cb = -(-rows // rows_per_scale), -(-cols // 128)
    s = 4.0 ** torch.randint(-1, 2, (*x.shape[:-2], rb, cb), generator=g, device=x.device) / 448 * (1 + torch.rand(*x.shape[:-2], rb, cb, generator=g, device=x.device))
    q = (x * 100).clamp(-448, 448).to(TYPES["f8"])
    wide = s.repeat_interleave(rows_per_scale, -2)[..., :rows, :].repeat_interleave(128, -1)[..., :cols]
    return q, s.contiguous(), q.double() * wide.double()


def run_twice(v, inputs, c):
    """The output of two launches, equal bit for bit; rows that nobody writes keep 7."""
    outs = []
    for _ in range(2):
        c.fill_(7)
        v.launch([x.data_ptr() for x in inputs], c.data_ptr(), stream=devmem.current_stream())
        torch.cuda.synchronize()
        outs.append(c.clone())
    assert torch.equal(outs[0].view(torch.uint8), outs[1].view(torch.uint8)), "two launches differ"
    return outs[0]


@pytest.mark.parametrize("K,code", [(144, 256256), (1024, 256256), (1040, 256256), (1152, 0), (1280, 256256), (2048, 256256), (2176, 0), (3200, 0)])
def test_scaled_product_of_several_whole_tiles_each(K, code):
    """Depths of 2, 8, 9, 10, 16, 17 and 25 blocks of scales."""
    M, N = 8192 + 300, 8192
    op = B.scaled_gemm_op(M, N, K, "bf16")
    assert B.trace_validate(op, op.space(), B.make_trace(op.space(), [[code]])).body == B.BODY_RAGGED_PHASES
    v = variant(op, code)
    if v is None:
        return
    assert whole_tiles_each([M], N) >= 4
    g, normal = on_device(K)
    a, sa, av = blocks_of(normal(M, K), 1, g)
    b, sb, bv = blocks_of(normal(N, K), 128, g)
    c = run_twice(v, [a, b, sa, sb], torch.empty(M, N, dtype=torch.bfloat16, device="cuda"))
    close(c, av @ bv.t(), av.abs() @ bv.abs().t(), K // 64 + 4, "bf16", f8=True)


@pytest.mark.parametrize("kind,rows_of_k,K", [("f8", True, 272), ("f8", True, 1040), ("f8", True, 1152), ("f8", True, 2064), ("bf16", True, 40), ("bf16", True, 72), ("f16", True, 192),
                                              ("f16", False, 64), ("bf16", False, 328)])
def test_grouped_product_of_several_whole_tiles_each(kind, rows_of_k, K):
    counts, ahead, behind, N = [1948, 0, 1950, 137, 250, 3], 2, 5, 8184
    E, T = len(counts), ahead + sum(counts) + behind
    out = "f16" if kind == "f16" else "bf16"
    v = variant(B.grouped_gemm_op(E, T, N, K, rows_of_k, kind, out), 256256)
    if v is None:
        return
    assert whole_tiles_each(counts, N) >= 2
    g, normal = on_device(K)
    off = offsets_of(counts, ahead)
    a, b, extra = normal(T, K), normal(E, N, K), []
    if kind == "f8":
        a, sa, av = blocks_of(a, 1, g)
        b, sb, bv = blocks_of(b, 128, g)
        extra = [sa, sb]
    else:
        a, b = a.to(TYPES[kind]), b.to(TYPES[kind])
        av, bv = a.double(), b.double()
        if not rows_of_k:
            b = b.transpose(1, 2).contiguous()
    c = run_twice(v, [a, b, off.cuda()] + extra, torch.empty(T, N, dtype=TYPES[out], device="cuda"))
    assert bool((c[:ahead] == 7).all()) and bool((c[T - behind:] == 7).all()), "rows of no expert were written"
    for e in range(E):
        rows = slice(int(off[e]), int(off[e + 1]))
        if counts[e]:
            close(c[rows], av[rows] @ bv[e].t(), av[rows].abs() @ bv[e].abs().t(), K, out, f8=kind == "f8")


def test_weight_gradient_of_several_whole_tiles_each():
    """Tiles of unequal depths, from none and one step up, one after the other in a workgroup."""
    counts, I, J = [700, 1, 0, 64, 65, 130, 3, 256, 0, 40], 2040, 2056
    E, T = len(counts), sum(counts) + 3
    v = variant(B.grouped_wgrad_op(E, T, I, J, "bf16", "bf16"), 256256)
    if v is None:
        return
    assert E * 8 * 9 // torch.cuda.get_device_properties(0).multi_processor_count >= 2
    _, normal = on_device(3)
    p, q, off = normal(T, I).bfloat16(), normal(T, J).bfloat16(), offsets_of(counts, 1)
    d = run_twice(v, [p, q, off.cuda()], torch.empty(E, I, J, dtype=torch.bfloat16, device="cuda"))
    for e in range(E):
        rows = slice(int(off[e]), int(off[e + 1]))
        pv, qv = p[rows].double(), q[rows].double()
        close(d[e], pv.t() @ qv, pv.abs().t() @ qv.abs(), max(1, counts[e]), "bf16")


def test_captured_whole_tiles():
    """A graph of a product of several whole tiles for each workgroup and of the gradient, replayed with other inputs and the program's own work in between."""
    M, N, K, E = 4096, 8192, 1152, 4
    v, w = variant(B.scaled_gemm_op(M, N, K, "bf16"), 256256), variant(B.grouped_wgrad_op(E, M, 2048, 4096, "bf16", "f32"), 256256)
    if v is None:
        return
    v.prepare(), w.prepare()
    g, normal = on_device(5)
    a, sa, _ = blocks_of(normal(M, K), 1, g)
    b, sb, _ = blocks_of(normal(N, K), 128, g)
    c, d = torch.empty(M, N, dtype=torch.bfloat16, device="cuda"), torch.empty(E, 2048, 4096, device="cuda")
    p, off = normal(M, 2048).bfloat16(), torch.tensor([0, 1000, 1000, 1001, 4000], dtype=torch.int32, device="cuda")

    def step():
        v.launch_static([a.data_ptr(), b.data_ptr(), sa.data_ptr(), sb.data_ptr()], c.data_ptr(), stream=devmem.current_stream())
        w.launch_static([p.data_ptr(), c.data_ptr(), off.data_ptr()], d.data_ptr(), stream=devmem.current_stream())

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        a.copy_(blocks_of(normal(M, K), 1, g)[0])
        got = []
        for run in (graph.replay, step):
            c.fill_(3), d.fill_(3)
            run()
            torch.cuda.synchronize()
            got.append((c.clone(), d.clone()))
        assert all(torch.equal(x, y) for x, y in zip(*got))
        assert bool((got[0][1][1] == 0).all())
