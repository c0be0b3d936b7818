"""The operators on rows of tokens together, as a decoder's layers use them: runs of calls, graphs, streams, threads."""
import threading

import pytest
import torch

import paper_1603_05279_b200 as X
from paper_1603_05279_b200.runner import TokenBlock
from rows_util import EPS, U, gen, half_step, matmul_bound, norm64, norm_error, randn, unpack_codes, weights64

pytestmark = pytest.mark.gpu


def block(rows, K, N, q, seed, zeros=False, group=128):
    g = gen(seed)
    b = TokenBlock(rows, K, N, group=group, zeros=zeros, quant=q)
    b.weight.copy_(1 + 0.1 * randn((K,), g))
    b.load(randn((N, K), g, torch.bfloat16, 0.02))
    b.x.copy_(randn((rows, K), g, torch.bfloat16))
    b.residual.copy_(randn((rows, K), g, torch.bfloat16))
    return b


def check(b):
    """Each stage from the stage before it as the GPU has it."""
    N, K = b.d.N, b.d.K
    h = (b.x0.float() + b.residual0.float()).to(torch.bfloat16)
    assert torch.equal(b.residual, h)
    y = norm64(h, b.weight)[1]
    e = norm_error(K) + 4 * U
    if b.q is None:
        assert ((b.y.double() - y).abs() <= (half_step(torch.bfloat16) + 2 * e) * y.abs() + 1e-40).all()
        x, each = b.y, 1.0
    else:
        each = b.q_scales.double().repeat_interleave(K // b.q_scales.shape[1], 1)
        step = 0.5 * each if b.q.dtype == torch.int8 else (2.0 ** -4 * y.abs()).clamp(min=2.0 ** -10 * each)
        assert ((b.q.float().double() * each - y).abs() <= step + 3 * e * y.abs() + 2 * U * y.abs()).all()
        x = b.q.float()
    codes = torch.from_numpy(unpack_codes(b.packed, N, K)).cuda()
    W = weights64(codes, b.scales, b.zeros, b.d.group)
    want = (x.double() * each) @ W.t()
    assert ((b.out.double() - want).abs() <= matmul_bound(x, each, W, K, b.d.group, b.out.dtype, want)).all()


@pytest.mark.parametrize("rows", [1, 8, 23, 130])
@pytest.mark.parametrize("q", [None, "i8", "i8_groups", "e4m3", "e4m3_groups"])
def test_norm_then_product(rows, q):
    b = block(rows, 1024, 520, q, rows, zeros=rows == 23)
    b.x0, b.residual0 = b.x.clone(), b.residual.clone()
    b.forward()
    X.xnor_check_device()
    check(b)


def run_layers(layers):
    """Projections one after the other: each adds what the one before gave to the residual stream it keeps."""
    for i, b in enumerate(layers):
        if i:
            b.x.copy_(layers[i - 1].out)
            b.residual.copy_(layers[i - 1].residual)
        b.forward()
    return layers[-1].out


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("q", [None, "i8", "e4m3_groups"])
def test_captured_and_replayed(rows, q):
    """Three layers in a graph, replayed on new inputs: the bits of the same calls made one by one."""
    layers = [block(rows, 512, 512, q, i) for i in range(3)]
    first = layers[0]
    inputs = [(randn((rows, 512), gen(50 + i), torch.bfloat16), randn((rows, 512), gen(90 + i), torch.bfloat16)) for i in range(3)]

    def put(i):
        first.x.copy_(inputs[i][0])
        first.residual.copy_(inputs[i][1])

    want = []
    for i in range(3):
        put(i)
        want.append(run_layers(layers).clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        put(0)
        run_layers(layers)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            run_layers(layers)
    for i in (2, 0, 1):
        put(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(layers[-1].out, want[i])
    X.xnor_check_device()


def test_two_streams_and_two_threads():
    """Blocks that share their weights, run from two threads on two streams at the same time."""
    a, b = block(64, 1024, 1024, "i8", 1), block(64, 1024, 1024, "i8", 2)
    b.packed, b.scales = a.packed, a.scales
    torch.cuda.synchronize()
    want = []
    for s in (a, b):
        s.x0, s.residual0 = s.x.clone(), s.residual.clone()
        s.forward()
        want.append(s.out.clone())
    torch.cuda.synchronize()

    def work(s, errors):
        try:
            stream = torch.cuda.Stream()
            for _ in range(20):
                with torch.cuda.stream(stream):
                    s.residual.copy_(s.residual0)
                s.forward(stream)
            stream.synchronize()
        except Exception as e:                    # handed to the thread that asserts
            errors.append(e)

    errors = []
    threads = [threading.Thread(target=work, args=(s, errors)) for s in (a, b)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors and torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])


def test_training_step_of_the_norm():
    """Forward, backward and an update of the norm's weight, eager and as a captured graph beside it."""
    g = gen(7)
    T, D = 200, 768
    x, r, dy = (randn((T, D), g, torch.bfloat16) for _ in range(3))
    w = 1 + 0.1 * randn((D,), g)
    total, y, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    rstd = torch.empty(T, device="cuda")
    dw, work = X.alloc_rmsnorm_backward(T, D)

    def step():
        X.xnor_rmsnorm(x, r, w, EPS, total, y, rstd)
        X.xnor_rmsnorm_backward(dy, dy, total, w, rstd, dx, dw, work)
        w.sub_(dw, alpha=1e-4)

    w0 = w.clone()
    step()
    step()
    want = (w.clone(), dx.clone())
    w.copy_(w0)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    torch.cuda.synchronize()
    w.copy_(w0)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(w, want[0]) and torch.equal(dx, want[1])


FIRST_CALL = """
import torch
from paper_1603_05279_b200.runner import TokenBlock
import paper_1603_05279_b200 as X
b = TokenBlock(%d, 512, 640, quant=%r)
w = torch.randn(640, 512, device="cuda").bfloat16()
b.x.normal_()
b.residual.normal_()
start = b.residual.clone()
torch.cuda.synchronize()
side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=side):
    b.load(w)
    b.forward()
graph.replay()
torch.cuda.synchronize()
got = b.out.clone()
b.residual.copy_(start)
b.load(w)
b.forward()
X.xnor_check_device()
assert torch.equal(got, b.out) and torch.isfinite(got).all()
"""


@pytest.mark.parametrize("rows,q", [(3, None), (40, "i8"), (300, None)])
def test_first_calls_inside_a_capture(rows, q):
    """What a process's first calls look up and set may happen while a graph is being captured."""
    import subprocess
    import sys
    from test_binding import ROOT
    r = subprocess.run([sys.executable, "-c", FIRST_CALL % (rows, q)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
