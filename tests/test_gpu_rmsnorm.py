"""Root-mean-square norm of rows, its 8-bit outputs and its backward pass against 64-bit definitions."""
import pytest
import torch

import paper_1603_05279_b200 as X
from rows_util import EPS, TYPES, U, Guards, gen, half_step, least, norm64, norm_error, randn, strided

pytestmark = pytest.mark.gpu

#        rows, cols: one and few, odd, a chunk short or over, every number of chunks per thread, the widest
SIZES = [(1, 1), (3, 7), (2, 8), (5, 33), (1, 2048), (4, 256), (37, 1000), (6, 1001), (9, 4096), (3, 4104), (2, 8200),
         (2, 16392), (3, 32761), (2, 32768)]


def run_forward(x, r, w, eps=EPS, pad=0, want_sum=True):
    g = Guards()
    T, D = x.shape
    total = g.rows(T, D, x.dtype, pad) if want_sum else None
    y, rstd = g.rows(T, D, x.dtype, pad), g.flat(T, torch.float32)
    X.xnor_rmsnorm(x, r, w, eps, total, y, rstd)
    g.check()
    return total, y, rstd


def check_forward(x, r, w, total, y, rstd, eps=EPS):
    t = x.dtype
    h = x if r is None else (x.float() + r.float()).to(t)
    if total is not None:
        assert torch.equal(total, h)
    rstd64, y64 = norm64(h, w, eps)
    e = norm_error(x.shape[1])
    assert ((rstd.double() - rstd64).abs() <= e * rstd64).all()
    off = (y.double() - y64).abs() - ((half_step(t) + e * (1 + half_step(t))) * y64.abs() + least(t))
    assert (off <= 0).all(), off.max()


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_norm(name, rows, cols):
    t, g = TYPES[name], gen(rows * 40000 + cols)
    x, r = randn((rows, cols), g, t, 3.0), randn((rows, cols), g, t)
    for res, w in ((None, randn((cols,), g, t)), (r, randn((cols,), g)), (r, None)):
        check_forward(x, res, w, *run_forward(x, res, w, want_sum=res is not None))


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("cols,pad", [(64, 1), (100, 28), (1000, 8), (1001, 7), (4096, 4)])
def test_norm_of_rows_apart(name, cols, pad):
    """Rows at strides that are and are not multiples of 16 bytes; what lies between them stays."""
    t, g = TYPES[name], gen(cols + pad)
    x, r = strided(randn((5, cols), g, t), pad), strided(randn((5, cols), g, t), 2 * pad)
    w = randn((cols,), g, t)
    check_forward(x, r, w, *run_forward(x, r, w, pad=pad))


def test_norm_of_one_row_for_all():
    g = gen(3)
    x, r, w = randn((1, 520), g).expand(9, 520), randn((9, 520), g), randn((520,), g)
    check_forward(x, r, w, *run_forward(x, r, w))


@pytest.mark.parametrize("name", sorted(TYPES))
def test_norm_in_place(name):
    """sum over the residual and y over x: the residual stream of a model stays in one buffer."""
    t, g = TYPES[name], gen(11)
    for cols in (1001, 4096):
        x, r, w = randn((33, cols), g, t), randn((33, cols), g, t), randn((cols,), g, t)
        total, y, rstd = run_forward(x, r, w)
        x2, r2 = x.clone(), r.clone()
        X.xnor_rmsnorm(x2, r2, w, EPS, r2, x2, None)
        assert torch.equal(r2, total) and torch.equal(x2, y)


def test_norm_of_zeros_nan_and_infinity():
    """A row of zeros is a row of zeros; a row with NaN or infinity spoils itself alone."""
    g = gen(5)
    x, w = randn((6, 1024), g), randn((1024,), g)
    x[1] = 0
    x[2, 77] = float("nan")
    x[4, 5] = float("inf")
    _, y, rstd = run_forward(x, None, w, want_sum=False)
    sound = [0, 3, 5]
    check_forward(x[sound], None, w, None, y[sound], rstd[sound])
    assert (y[1] == 0).all() and y[2].isnan().all() and y[4, 5].isnan() and (y[4, :5] == 0).all()
    q, s = X.alloc_rmsnorm_quant(6, 1024, 128)
    X.xnor_rmsnorm_quant(x, None, w, EPS, 128, None, q, s, None)
    assert (s[1] == 0).all() and (q[1] == 0).all()
    assert s[2].isnan().all() and (q[2] == 0).all()
    assert s[4, 0].isnan() and (q[4] == 0).all() and (s[4, 1:] == 0).all()


def check_quant(x, r, w, group, q, s, total):
    """q and its scales against 64 bits: y is off by norm_error, the scale by that, a constant and a product (2 U); the
    quotient by both errors, those of an approximate reciprocal (2 U) and two products (2 U), relative to its
    magnitude; then half a step of the output."""
    h = x if r is None else (x.float() + r.float()).to(x.dtype)
    if total is not None:
        assert torch.equal(total, h)
    T, D = x.shape
    top = 127.0 if q.dtype == torch.int8 else 448.0
    y = norm64(h, w)[1].view(T, -1, group or D)
    s64 = y.abs().amax(2) / top
    e = norm_error(D) + 2 * U
    assert ((s.double() - s64).abs() <= e * s64).all()
    v = torch.where(s64[:, :, None] > 0, y / s64[:, :, None], 0.0)
    d = (q.float().double().view_as(v) - v).abs()
    if q.dtype == torch.int8:
        bound = 0.5 + (2 * e + 4 * U) * v.abs()
    else:
        bound = (2.0 ** -4 * v.abs()).clamp(min=2.0 ** -10) + (2 * e + 4 * U) * v.abs()      # subnormal below 2^-6
    assert (d <= bound).all(), (d - bound).max()


@pytest.mark.parametrize("qtype", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("rows,cols,groups", [(1, 32, (0, 32)), (3, 64, (32, 64)), (5, 100, (0,)), (7, 1001, (0,)),
                                              (4, 1056, (0, 32)), (33, 4096, (0, 32, 64, 128)), (2, 8320, (64, 128)),
                                              (3, 16512, (0, 128)), (2, 32768, (0, 32, 128)), (2, 32767, (0,))])
def test_quant(qtype, rows, cols, groups):
    for group in groups:
        for name, t in TYPES.items():
            g = gen(cols + group)
            x, r, w = randn((rows, cols), g, t, 2.0), randn((rows, cols), g, t), randn((cols,), g)
            G = Guards()
            q, s = G.rows(rows, cols, qtype), G.rows(rows, cols // group if group else 1, torch.float32)
            total, rstd = G.rows(rows, cols, t), G.flat(rows, torch.float32)
            X.xnor_rmsnorm_quant(x, r, w, EPS, group, total, q, s, rstd)
            G.check()
            check_quant(x, r, w, group, q, s, total)


def test_quant_of_rows_apart_and_tiny_values():
    g = gen(8)
    x = strided(randn((5, 384), g, torch.bfloat16), 3)
    w = randn((384,), g)
    q, s = X.alloc_rmsnorm_quant(5, 384, 128, torch.float8_e4m3fn)
    X.xnor_rmsnorm_quant(x, None, w, EPS, 128, None, q, s, None)
    check_quant(x, None, w, 128, q, s, None)
    # scales whose reciprocal overflows: the weights shrink the norm to subnormal numbers
    tiny = torch.full((384,), 3e-38, device="cuda") * (1 + torch.rand(384, generator=g, device="cuda"))
    q, s = X.alloc_rmsnorm_quant(5, 384, 0)
    X.xnor_rmsnorm_quant(x, None, tiny, EPS, 0, None, q, s, None)
    y = norm64(x, tiny)[1]
    # y is a whole number of the smallest subnormal: off by half of one more than norm_error
    v = y / s.double()
    assert ((q.double() - v).abs() <= 0.5 + 2.0 ** -150 / s.double() + 128 * (norm_error(384) + U)).all()


def backward64(dy, ds, h, w, rstd):
    dy, h, r = dy.double(), h.double(), rstd.double()[:, None]
    u = dy if w is None else dy * w.double()
    dx = r * (u - h * (r * r * (u * h).mean(1, keepdim=True)))
    # magnitudes of the terms that are added: what the errors of the sums are relative to
    mag = r * (u.abs() + h.abs() * (r * r * (u * h).abs().mean(1, keepdim=True)))
    if ds is not None:
        dx, mag = dx + ds.double(), mag + ds.double().abs()
    return dx, mag, (dy * h * r).sum(0), (dy * h * r).abs().sum(0)


def run_backward(dy, ds, h, w, rstd, pad=0):
    T, D = h.shape
    G = Guards()
    dx, dw = G.rows(T, D, h.dtype, pad), G.flat(D, torch.float32)
    work = G.flat(X.xnor_rmsnorm_work_elems(T, D), torch.float32)
    X.xnor_rmsnorm_backward(dy, ds, h, w, rstd, dx, dw, work)
    G.check()
    return dx, dw


def check_backward(dy, ds, h, w, rstd, dx, dw):
    t = h.dtype
    dx64, mag, dw64, dwmag = backward64(dy, ds, h, w, rstd)
    # the row's sum: chains as in the forward pass (69 U) of products of two roundings, then 8 operations
    off = (dx.double() - dx64).abs() - (half_step(t) * dx64.abs() + least(t) + 80 * U * mag)
    assert (off <= 0).all(), off.max()
    # a column: at most rows / blocks in a chain, the blocks' sums in eight chains, 8 to join, two products
    T = h.shape[0]
    chain = T + 148 + 8 + 3
    off = (dw.double() - dw64).abs() - chain * U * dwmag
    assert (off <= 0).all(), off.max()


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("rows,cols", SIZES + [(700, 520), (1300, 64), (400, 8192)])
def test_backward(name, rows, cols):
    t, g = TYPES[name], gen(rows * 40000 + cols + 1)
    h, dy, ds = randn((rows, cols), g, t, 2.0), randn((rows, cols), g, t), randn((rows, cols), g, t)
    rstd = norm64(h, None)[0].float()
    for d, w in ((None, randn((cols,), g, t)), (ds, randn((cols,), g)), (ds, None)):
        check_backward(dy, d, h, w, rstd, *run_backward(dy, d, h, w, rstd))


@pytest.mark.parametrize("name", sorted(TYPES))
def test_backward_of_rows_apart_and_in_place(name):
    t, g = TYPES[name], gen(21)
    for cols, pad in ((100, 28), (1001, 7), (1000, 1)):
        h, dy, ds = (strided(randn((6, cols), g, t), k * pad) for k in (1, 2, 3))
        w, rstd = randn((cols,), g, t), norm64(h, None)[0].float()
        dx, dw = run_backward(dy, ds, h, w, rstd, pad)
        check_backward(dy, ds, h, w, rstd, dx, dw)
        for over in (dy, ds):
            keep = over.clone()
            X.xnor_rmsnorm_backward(dy, ds, h, w, rstd, over, None, None)
            assert torch.equal(over, dx)
            over.copy_(keep)


def test_backward_against_differences():
    """The loss sum(y dy) + sum(h ds) along a random direction, by central differences of the 64-bit definition: the
    error of a step of 1e-4 is of the order of its square times the third derivative, below 1e-6 of the terms."""
    g = gen(4)
    x, r, dy, ds, v = (randn((3, 257), g) for _ in range(5))
    w, dw_dir = randn((257,), g), randn((257,), g)
    h = x + r
    rstd = norm64(h, None)[0].float()
    dx, dw = run_backward(dy, ds, h, w, rstd)

    def loss(step):
        hh = h.double() + step * v.double()
        y = norm64(hh, w.double() + step * dw_dir.double())[1]
        return (y * dy.double()).sum() + (hh * ds.double()).sum()

    slope = (loss(1e-4) - loss(-1e-4)) / 2e-4
    mine = (dx.double() * v.double()).sum() + (dw.double() * dw_dir.double()).sum()
    terms = (dx.double() * v.double()).abs().sum() + (dw.double() * dw_dir.double()).abs().sum()
    assert abs(slope - mine) <= 1e-5 * terms


def test_backward_of_no_rows_and_without_dweight():
    e = torch.empty((0, 96), device="cuda")
    dw = torch.full((96,), 5.0, device="cuda")
    X.xnor_rmsnorm_backward(e, None, e, None, torch.empty(0, device="cuda"), e.clone(), dw, torch.empty(0, device="cuda"))
    assert (dw == 0).all()
    X.xnor_rmsnorm(e, None, None, EPS, None, e.clone(), None)
    q, s = X.alloc_rmsnorm_quant(0, 96, 32)
    X.xnor_rmsnorm_quant(e, None, None, EPS, 32, None, q, s, None)


def test_same_bits_every_time():
    g = gen(6)
    h, dy = randn((2000, 1000), g, torch.bfloat16), randn((2000, 1000), g, torch.bfloat16)
    w, rstd = randn((1000,), g), norm64(h, None)[0].float()
    first = run_backward(dy, None, h, w, rstd)
    for _ in range(5):
        again = run_backward(dy, None, h, w, rstd)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_rows_beyond_32_bits():
    """Two rows 2^31 + 16 elements apart."""
    far = (1 << 31) + 16
    big = torch.zeros(far + 64, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((2, 64), (far, 1))
    g = gen(2)
    x.copy_(randn((2, 64), g, torch.bfloat16))
    w = randn((64,), g)
    keep = x.clone()
    check_forward(keep, None, w, *run_forward(x, None, w, want_sum=False))
    rstd, dy = norm64(keep, None)[0].float(), randn((2, 64), g, torch.bfloat16)
    dx, dw = run_backward(dy, None, x, w, rstd)
    check_backward(dy, None, keep, w, rstd, dx, dw)
    X.xnor_rmsnorm(keep, None, w, EPS, None, x, None)        # and written there
    check_forward(keep, None, w, None, x.clone(), rstd)
    assert int((big != 0).sum()) == int((x != 0).sum())
