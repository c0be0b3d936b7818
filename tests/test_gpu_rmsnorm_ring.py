"""The backward pass of many long rows, which come through a ring in shared memory: other kernels take the sizes of
test_gpu_rmsnorm's tests."""
import pytest
import torch

import paper_1603_05279_b200 as X
from rows_util import EPS, TYPES, U, Guards, gen, half_step, least, norm64, randn, strided
from test_gpu_rmsnorm import backward64

pytestmark = pytest.mark.gpu

#        rows, cols, types: one chunk of columns per thread and two, four; a last thread without columns; as many rows for
#        every block as not; two stages and eight
SIZES = [(593, 2048, "bf16 f16 f32"), (1300, 2056, "bf16 f16 f32"), (2961, 2048, "bf16"), (600, 1032, "f32"), (1201, 8200, "bf16 f16"),
         (700, 8192, "f32"), (2000, 4096, "bf16"), (640, 12296, "f16")]


def kernels_of(call):
    """Names of the kernels that a call launches."""
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA, torch.profiler.ProfilerActivity.CPU]) as p:
        call()
        torch.cuda.synchronize()
    return " ".join(e.name for e in p.events())


def inputs(rows, cols, t, seed, pads=(0, 0, 0)):
    g = gen(seed)
    h, dy, ds = (strided(randn((rows, cols), g, t, k), p) for k, p in zip((2.0, 1.0, 1.0), pads))
    return h, dy, ds, randn((cols,), g, t), norm64(h, None)[0].float()


def backward(dy, ds, h, w, rstd, pad=0):
    T, D = h.shape
    G = Guards()
    dx, dw = G.rows(T, D, h.dtype, pad), G.flat(D, torch.float32)
    work = G.flat(X.xnor_rmsnorm_work_elems(T, D), torch.float32)
    X.xnor_rmsnorm_backward(dy, ds, h, w, rstd, dx, dw, work)
    X.xnor_check_device()
    G.check()
    return dx, dw


def check(dy, ds, h, w, rstd, dx, dw):
    T, D = h.shape
    dx64, mag, dw64, dwmag = backward64(dy, ds, h, w, rstd)
    # a row's sum: a thread adds up to 32 products of two roundings each, then 5 steps of a tree and up to 16 warps; 8
    # operations after it
    off = (dx.double() - dx64).abs() - (half_step(h.dtype) * dx64.abs() + least(h.dtype) + (32 + 2 + 5 + 16 + 8) * U * mag)
    assert (off <= 0).all(), off.max()
    # a column: a block's rows in a chain (at least as many blocks as rows of partial sums per 4: the ring may take a
    # quarter of the most), the blocks' sums in 32 chains joined in 5 steps, two products and the last addition
    parts = X.xnor_rmsnorm_work_elems(T, D) // D
    chain = -(-T // max(1, parts // 4)) + -(-parts // 32) + 5 + 3
    off = (dw.double() - dw64).abs() - chain * U * dwmag
    assert (off <= 0).all(), off.max()


@pytest.mark.parametrize("rows,cols,name", [(r, c, n) for r, c, names in SIZES for n in names.split()])
def test_backward_through_the_ring(rows, cols, name):
    h, dy, ds, w, rstd = inputs(rows, cols, TYPES[name], rows + cols)
    for d, ww in ((None, w), (ds, w.float()), (ds, None)):
        check(dy, d, h, ww, rstd, *backward(dy, d, h, ww, rstd))


@pytest.mark.parametrize("rows,cols,name", [(r, c, n) for r, c, names in SIZES for n in names.split()])
def test_these_sizes_take_the_ring(rows, cols, name):
    h, dy, ds, w, rstd = inputs(rows, cols, TYPES[name], 1)
    dx = torch.empty_like(h)
    for d in (None, ds):
        names = kernels_of(lambda: X.xnor_rmsnorm_backward(dy, d, h, w, rstd, dx, None, None))
        if "rmsnorm_backward" not in names:
            pytest.skip("the profiler names no kernels here")
        assert "rmsnorm_backward_ring_kernel" in names, names


@pytest.mark.parametrize("name", sorted(TYPES))
def test_rows_apart_and_in_place(name):
    """Strides of whole pieces of 16 bytes: bulk copies take them, and nothing between the rows moves."""
    rows, cols, pad = 1300, 2056, 16
    h, dy, ds, w, rstd = inputs(rows, cols, TYPES[name], 5, (pad, 2 * pad, 3 * pad))
    dx, dw = backward(dy, ds, h, w, rstd, pad)
    check(dy, ds, h, w, rstd, dx, dw)
    for over in (dy, ds):                             # later rows of `over` are on their way while earlier ones are written
        keep = over.clone()
        X.xnor_rmsnorm_backward(dy, ds, h, w, rstd, over, None, None)
        assert torch.equal(over, dx)
        over.copy_(keep)


def test_one_gradient_for_all_rows():
    h, _, _, w, rstd = inputs(900, 4096, torch.bfloat16, 6)
    dy = randn((1, 4096), gen(7), torch.bfloat16).expand(900, 4096)
    check(dy, None, h, w, rstd, *backward(dy, None, h, w, rstd))


def test_same_bits_every_time():
    h, dy, ds, w, rstd = inputs(1201, 4096, torch.bfloat16, 8)
    first = backward(dy, ds, h, w, rstd)
    for _ in range(5):
        again = backward(dy, ds, h, w, rstd)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_captured_and_replayed():
    """Replays on new inputs give the bits of direct calls; the workspace is the graph's own."""
    h, dy, ds, w, rstd = inputs(800, 4096, torch.bfloat16, 9)
    dx, (dw, work) = torch.empty_like(h), X.alloc_rmsnorm_backward(800, 4096)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        X.xnor_rmsnorm_backward(dy, ds, h, w, rstd, dx, dw, work)
    for seed in (10, 11):
        h2, dy2, ds2, _, rstd2 = inputs(800, 4096, torch.bfloat16, seed)
        want = backward(dy2, ds2, h2, w, rstd2)
        for a, b in ((h, h2), (dy, dy2), (ds, ds2), (rstd, rstd2)):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
