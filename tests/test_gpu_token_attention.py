"""A decoder's layer in a run of calls: projection, norms and rotation, cache, attention, projection; graphs, streams and threads."""
import threading
from types import SimpleNamespace

import pytest
import torch

import paper_1603_05279_b200 as X
from kv4_util import Batch, attention64, heads64, heads_error, quantized, stood_for
from paper_1603_05279_b200.runner import TokenAttention, TokenBlock
from rows_util import gen, half_step, least, randn

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, rows, seqs, context, Hq, Hk, D, width, seed, **more):
        g = gen(seed)
        self.qkv = TokenBlock(rows, width, (Hq + 2 * Hk) * D, quant="i8")
        self.attention = TokenAttention(rows, seqs, context, Hq, Hk, D, **more)
        self.o = TokenBlock(rows, Hq * D, width)
        self.qkv.load(randn(((Hq + 2 * Hk) * D, width), g, torch.bfloat16, 0.05))
        self.o.load(randn((width, Hq * D), g, torch.bfloat16, 0.05))
        self.attention.cache.random_(0, 256, generator=g)

    def forward(self, x):
        """x: [rows][width], all of the blocks' rows."""
        self.qkv.x.copy_(x)
        self.qkv.residual.zero_()
        a = self.attention.forward(self.qkv.forward())
        self.o.x.copy_(a)
        self.o.residual.zero_()
        return self.o.forward()


def check_attention(L, lens, new):
    """Attention's output from the projection's rows and the cache as the GPU has them."""
    A, n = L.attention, sum(new)
    Hq, Hk, D = A.q_heads, A.kv_heads, A.dim
    qkv = L.qkv.out[:n]
    pos = torch.cat([torch.arange(a - b, a, device="cuda") for a, b in zip(lens, new)])
    q = qkv[:, :Hq * D].unflatten(1, (Hq, D))
    want, size = heads64(q, A.q_weight, A.eps, A.rope, pos, False)
    h = half_step(torch.bfloat16)
    assert ((A.q[:n].double() - want).abs() <= h * want.abs() + (1 + h) * heads_error() * size + least(torch.bfloat16)).all()
    b = Batch(lens, new, Hk, D, A.d.page, 0)
    b.cache, b.table, b.pages = A.cache, A.table, A.d.pages
    out, _, off, _ = attention64(b, A.q[:n], D ** -0.5)
    assert ((A.out[:n].unflatten(1, (Hq, D)).double() - out).abs() <= off).all()
    k = qkv[:, Hq * D:(Hq + Hk) * D].unflatten(1, (Hk, D))
    k = stood_for(*quantized(heads64(k, A.k_weight, A.eps, A.rope, pos, False)[0].float()))
    v = stood_for(*quantized(qkv[:, (Hq + Hk) * D:].unflatten(1, (Hk, D)).float()))
    row = 0
    for i, (a, m) in enumerate(zip(lens, new)):
        K, V = b.read64(i)
        assert torch.equal(K[a - m:], k[row:row + m]) and torch.equal(V[a - m:], v[row:row + m])
        row += m


@pytest.mark.parametrize("Hq,Hk,D", [(8, 2, 128), (6, 6, 64)])
def test_prompts_then_tokens(Hq, Hk, D):
    """Prompts of three sequences, then token after token, then a few at once: a new token sees all before it."""
    L = Layer(110, 3, 200, Hq, Hk, D, 256, 1, page=16)
    g, lens = gen(2), [0, 0, 0]
    for new in ([60, 1, 49], [1, 1, 1], [1, 1, 1], [5, 0, 2], [1, 30, 1], [0, 0, 1]):
        L.attention.grow(torch.tensor(new, dtype=torch.int32, device="cuda"))
        lens = [a + b for a, b in zip(lens, new)]
        L.forward(randn((110, 256), g, torch.bfloat16))
        X.xnor_check_device()
        check_attention(L, lens, new)


def test_captured_and_replayed():
    """A step in a graph, replayed with other inputs and lengths: the bits of the same calls made one by one."""
    make = lambda: Layer(4, 4, 600, 8, 2, 128, 256, 3, page=32, most=1)
    eager, other = make(), make()
    start = torch.tensor([500, 1, 77, 0], dtype=torch.int32, device="cuda")
    xs = [randn((4, 256), gen(10 + i), torch.bfloat16) for i in range(5)]
    ones = torch.ones(4, dtype=torch.int32, device="cuda")
    for L in (eager, other):
        c = L.attention
        full = TokenAttention(578, 4, 600, 8, 2, 128, page=32)
        full.cache, full.table = c.cache, c.table
        full.grow(start)
        full.forward(randn((578, 12 * 128), gen(9), torch.bfloat16))
        c.lens.copy_(start)
    want = []
    for x in xs:
        eager.attention.grow(ones)
        want.append(eager.forward(x).clone())
    x_in = xs[0].clone()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other.attention.grow(ones)
        other.forward(x_in)
        other.attention.lens.copy_(start)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            other.attention.grow(ones)
            out = other.forward(x_in)
    torch.cuda.synchronize()
    for x, w in zip(xs, want):
        x_in.copy_(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, w)
    assert torch.equal(eager.attention.cache, other.attention.cache)
    X.xnor_check_device()


def test_two_streams_and_two_threads():
    """Attention over one cache from two threads on two streams at the same time, a workspace each."""
    batch = Batch([3000, 100, 640], [2, 2, 2], 2, 128, 16, 4).fill(5)
    d = X.make_kv4_desc(batch.pages, 16, 2, 128)
    qs = [randn((6, 16, 128), gen(i), torch.bfloat16) for i in range(2)]
    works, outs = [X.alloc_kv4_work(d, 6, 16, 3) for _ in range(2)], [torch.empty_like(qs[0]) for _ in range(2)]
    want = []
    for q, w in zip(qs, works):
        o = torch.empty_like(q)
        X.xnor_kv4_attention(q, batch.cache, batch.starts, batch.lens, batch.table, d, 0.1, 2, o, None, w)
        want.append(o)
    torch.cuda.synchronize()
    wrong = []

    def go(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(50):
                X.xnor_kv4_attention(qs[i], batch.cache, batch.starts, batch.lens, batch.table, d, 0.1, 2, outs[i], None, works[i])
            stream.synchronize()
            wrong.append(not torch.equal(outs[i], want[i]))

    threads = [threading.Thread(target=go, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == [False, False]
    X.xnor_check_device()


def test_a_stream_given_by_hand_waits_for_what_is_on_it():
    """Back-to-back calls that overlap their launches: each sees what the one before wrote."""
    L = TokenAttention(2, 2, 100, 4, 2, 64, page=16, most=1)
    ones = torch.ones(2, dtype=torch.int32, device="cuda")
    g = gen(6)
    rows = [randn((2, 8 * 64), g, torch.bfloat16) for _ in range(60)]
    outs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for r in rows:
            L.grow(ones)
            outs.append(L.forward(r, side).clone())
    side.synchronize()
    X.xnor_check_device(side)
    b = Batch([60, 60], [60, 60], 2, 64, 16, 0)
    b.cache, b.table, b.pages = L.cache, L.table, L.d.pages
    q = torch.stack(rows, 1).flatten(0, 1)[:, :4 * 64].unflatten(1, (4, 64))      # by sequence, then token
    pos = torch.arange(60, device="cuda").repeat(2)
    q = heads64(q, None, L.eps, L.rope, pos, False)[0].to(torch.bfloat16)
    want, _, off, _ = attention64(b, q, 64 ** -0.5)
    got = torch.stack(outs, 1).flatten(0, 1).unflatten(1, (4, 64)).double()
    # (queries rounded from fp32 may differ by one rounding here and there: a step of bfloat16 in some of 64 products)
    assert ((got - want).abs() <= off + 2e-2 * want.abs().max()).all()


def test_gradients_through_a_run():
    """Two norms with rotations one after the other, gradients back through both, in a captured graph while eager tensors of the same values live."""
    T, H, D = 40, 3, 128
    g = gen(7)
    x, dy = randn((T, H, D), g), randn((T, H, D), g)
    w = [(1 + 0.2 * randn((D,), g)) for _ in range(2)]
    pos, rope = torch.arange(T, dtype=torch.int32, device="cuda"), X.make_rope(T, D)
    a, b, da, dx = (torch.empty_like(x) for _ in range(4))
    dw = [torch.empty(D, device="cuda") for _ in range(2)]
    work = [X.alloc_qk_backward(T, H, 0, D)[2] for _ in range(2)]

    def go():
        X.xnor_qk_norm_rope(x, None, w[0], None, 1e-6, pos, rope, False, a, None)
        X.xnor_qk_norm_rope(a, None, w[1], None, 1e-6, pos, rope, False, b, None)
        X.xnor_qk_norm_rope_backward(dy, None, a, None, w[1], None, 1e-6, pos, rope, False, da, None, dw[1], None, work[1])
        X.xnor_qk_norm_rope_backward(da, None, x, None, w[0], None, 1e-6, pos, rope, False, dx, None, dw[0], None, work[0])

    go()
    torch.cuda.synchronize()
    eager = [t.clone() for t in (b, dx, *dw)]
    leaf, weights = x.double().requires_grad_(), [v.double().requires_grad_() for v in w]
    y = heads64(heads64(leaf, weights[0], 1e-6, rope, pos, False)[0], weights[1], 1e-6, rope, pos, False)[0]
    y.backward(dy.double())
    for got, want in ((b, y), (dx, leaf.grad), (dw[0], weights[0].grad), (dw[1], weights[1].grad)):
        # two passes of fp32, each within some 100 U of sums of up to 120 terms that are no larger than ten times the largest
        assert (got.double() - want).abs().max() <= 200 * 2.0 ** -24 * 10 * 120 ** 0.5 * want.abs().max()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        go()
    for t in (b, dx, *dw):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(t, e) for t, e in zip((b, dx, *dw), eager))
    X.xnor_check_device()


def test_room_for_many_rows_is_room_for_few():
    """A layer made for prompts of thousands of tokens gets one of 200, whose context is shared by many blocks."""
    A = TokenAttention(5000, 2, 5200, 8, 8, 64, page=16)
    A.grow(torch.tensor([200, 1], dtype=torch.int32, device="cuda"))
    qkv = randn((201, 24 * 64), gen(3), torch.bfloat16)
    A.forward(qkv)
    X.xnor_check_device()
    check_attention(SimpleNamespace(attention=A, qkv=SimpleNamespace(out=qkv)), [200, 1], [200, 1])
