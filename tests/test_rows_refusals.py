"""Calls on rows of tokens that are refused before anything is launched (no GPU needed)."""
import ctypes

import pytest

import paper_1603_05279_b200 as X
from paper_1603_05279_b200 import binding as B
from test_binding import run_child

P, ODD, NULL = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004), ctypes.c_void_p(0)
INV, UNS = B.XNOR_ERR_INVALID_ARG, B.XNOR_ERR_UNSUPPORTED


def norm(rows=4, cols=64, type=B.XNOR_BF16, weight_type=B.XNOR_F32, eps=1e-5, stride=64, **more):
    d = B.xnor_norm_desc(rows, cols, type, weight_type, eps, stride, stride, stride, stride)
    for k, v in more.items():
        setattr(d, k, v)
    return ctypes.byref(d)


def test_norm_arguments():
    lib = X.load()
    fwd = lambda d, x=P, r=P, w=P, s=P, y=P, rs=P: lib.xnor_rmsnorm(x, r, w, d, s, y, rs, NULL)
    for kw in (dict(x=NULL), dict(y=NULL), dict(x=ODD), dict(r=ODD), dict(w=ODD), dict(s=ODD), dict(y=ODD), dict(rs=ODD)):
        assert fwd(norm(), **kw) == INV, kw
    for kw in (dict(rows=-1), dict(cols=0), dict(type=B.XNOR_I8), dict(type=9), dict(weight_type=B.XNOR_F16), dict(eps=-1.0),
               dict(eps=float("nan")), dict(x_stride=-64), dict(residual_stride=-1), dict(sum_stride=63), dict(y_stride=0)):
        assert fwd(norm(**kw)) == INV, kw
    assert fwd(None) == INV
    assert fwd(norm(cols=32769, stride=40000)) == UNS
    assert fwd(norm(rows=0), x=NULL, r=NULL, y=NULL, s=NULL, rs=NULL) == B.XNOR_OK       # nothing to do
    q = lambda d, t=B.XNOR_I8, g=32, q=P, s=P: lib.xnor_rmsnorm_quant(P, P, P, d, t, g, P, q, s, P, NULL)
    assert q(norm(), t=B.XNOR_BF16) == INV and q(norm(), g=16) == INV and q(norm(), g=-32) == INV
    assert q(norm(), q=NULL) == INV and q(norm(), s=ODD) == INV
    assert q(norm(cols=80, stride=80)) == UNS and q(norm(), g=128) == UNS
    b = lambda d, dy=P, ds=P, h=P, w=P, rs=P, dx=P, dw=P, wk=P: lib.xnor_rmsnorm_backward(dy, ds, h, w, rs, d, dx, dw, wk, NULL)
    for kw in (dict(dy=NULL), dict(h=NULL), dict(rs=NULL), dict(dx=NULL), dict(wk=NULL), dict(dw=ODD), dict(ds=ODD)):
        assert b(norm(), **kw) == INV, kw
    assert b(norm(sum_stride=10)) == INV
    assert b(norm(cols=40000, stride=40000)) == UNS


def test_work_elems():
    assert X.xnor_rmsnorm_work_elems(0, 64) == 0 and X.xnor_rmsnorm_work_elems(-1, 64) == 0
    assert X.xnor_rmsnorm_work_elems(5, 0) == 0 and X.xnor_rmsnorm_work_elems(5, 32769) == 0
    for rows, cols in ((1, 1), (5, 100), (100000, 4096), (2 ** 31 - 1, 32768)):
        n = X.xnor_rmsnorm_work_elems(rows, cols)
        assert n % cols == 0 and 1 <= n // cols <= min(rows, 8 * 148)


def test_w4_arguments():
    lib = X.load()
    d = lambda N=40, K=100, g=64: ctypes.byref(B.xnor_w4_desc(N, K, g))
    for bad in (d(N=0), d(K=0), d(K=-5), d(g=0), d(g=16), d(g=256), None):
        assert lib.xnor_w4_quantize(P, 1, bad, P, P, P, NULL) == INV
        assert lib.xnor_w4_pack(P, bad, P, NULL) == INV
        assert lib.xnor_w4_dequantize(P, P, P, bad, 1, P, NULL) == INV
        assert lib.xnor_w4_packed_words(bad) == 0
        assert lib.xnor_w4_matmul(P, NULL, P, P, P, bad, ctypes.byref(B.xnor_w4_rows(1, 1, 0, 1, 100, 40)), P, NULL) == INV
    assert lib.xnor_w4_packed_words(d()) == 1 * 2 * 1024
    for big in (d(N=1048449), d(K=(1 << 24) + 1)):
        assert lib.xnor_w4_quantize(P, 1, big, P, P, NULL, NULL) == UNS and lib.xnor_w4_pack(P, big, P, NULL) == UNS
        assert lib.xnor_w4_dequantize(P, P, NULL, big, 1, P, NULL) == UNS and lib.xnor_w4_packed_words(big) == 0
    assert lib.xnor_w4_quantize(P, B.XNOR_I8, d(), P, P, NULL, NULL) == INV
    for a in ((NULL, P, P, P), (P, NULL, P, P), (P, P, NULL, P), (P, P, P, ODD), (ODD, P, P, P)):
        assert lib.xnor_w4_quantize(a[0], 0, d(), a[1], a[2], a[3], NULL) == INV
        assert lib.xnor_w4_dequantize(a[0], a[1], a[3], d(), 0, a[2], NULL) == INV
    rows = lambda rows=3, t=B.XNOR_BF16, xg=0, o=B.XNOR_BF16, xs=100, os=40: ctypes.byref(B.xnor_w4_rows(rows, t, xg, o, xs, os))
    mm = lambda r, x=P, xs=NULL, w=P, s=P, z=P, o=P: lib.xnor_w4_matmul(x, xs, w, s, z, d(), r, o, NULL)
    for kw in (dict(x=NULL), dict(w=NULL), dict(s=NULL), dict(o=NULL), dict(x=ODD), dict(z=ODD), dict(o=ODD), dict(xs=P)):
        assert mm(rows(), **kw) == INV, kw
    for r in (rows(rows=-1), rows(t=7), rows(t=-1), rows(o=B.XNOR_I8), rows(xs=-1), rows(os=39), rows(t=B.XNOR_I8), None):
        assert mm(r) == INV
    assert mm(rows(t=B.XNOR_F32)) == UNS and mm(rows(t=B.XNOR_I8, xg=32), xs=P) == UNS
    assert mm(rows(rows=1048561)) == UNS
    assert mm(rows(rows=0), x=NULL, o=NULL) == B.XNOR_OK


def test_the_binding_checks_tensors_against_each_other():
    run_child("""
bf, u8, i8, e4 = torch.bfloat16, torch.uint8, torch.int8, torch.float8_e4m3fn
f = lambda *s, t=torch.float32: fake(*s, dtype=t)
def no(call, kind=ValueError): raises(kind, call)
N = lambda x=None, r=None, w=None, s=None, y=None, rs=None, eps=1e-5: X.xnor_rmsnorm(
    f(4, 64) if x is None else x, r, w, eps, s, f(4, 64) if y is None else y, rs, stream=0)
no(lambda: N(x=torch.zeros(4, 64)))                       # on the host
no(lambda: N(x=f(4, 64, 1)))
no(lambda: N(x=f(64, 4).t()))                             # columns apart
no(lambda: N(x=f(4, 64, t=torch.float64), y=f(4, 64, t=torch.float64)))
no(lambda: N(y=f(4, 63)))
no(lambda: N(y=f(4, 64, t=bf)))
no(lambda: N(r=f(3, 64)))
no(lambda: N(w=f(63)))
no(lambda: N(w=f(64, t=bf)))                              # neither fp32 nor the rows' type
no(lambda: N(rs=f(5)))
no(lambda: N(eps="a"), TypeError)
no(lambda: N(x=3), AttributeError)
Q = lambda q=None, s=None, g=32: X.xnor_rmsnorm_quant(f(4, 64), None, None, 1e-5, g, None, f(4, 64, t=i8) if q is None else q, f(4, 2) if s is None else s, None, stream=0)
no(lambda: Q(q=f(4, 64, t=u8)))
no(lambda: Q(q=f(4, 64)))
no(lambda: Q(q=f(8, 64, t=i8)[::2]))                      # not dense
no(lambda: Q(s=f(4, 1)))
no(lambda: Q(g=0))
R = lambda dw, wk, h=None: X.xnor_rmsnorm_backward(f(4, 64), None, f(4, 64) if h is None else h, None, f(4), f(4, 64), dw, wk, stream=0)
no(lambda: R(f(64), f(63)))                               # work too small
no(lambda: R(f(63), f(256)))
no(lambda: R(None, None, h=f(4, 64, t=bf)))
d = X.make_w4_desc(40, 100, 64)
pk, sc, z = f(1, 2, 256, 4, t=torch.int32), f(2, 40), f(2, 40, t=u8)
M = lambda x=None, xs=None, p=pk, s=sc, zz=z, d=d, o=None: X.xnor_w4_matmul(f(5, 100, t=bf) if x is None else x, xs, p, s, zz, d, f(5, 40, t=bf) if o is None else o, stream=0)
no(lambda: M(x=f(5, 99, t=bf)))
no(lambda: M(p=f(1, 2, 256, 3, t=torch.int32)))
no(lambda: M(p=f(1, 2, 256, 4)))
no(lambda: M(s=f(40, 2)))
no(lambda: M(zz=f(2, 40)))
no(lambda: M(o=f(5, 41, t=bf)))
no(lambda: M(o=f(4, 40, t=bf)))
no(lambda: M(o=f(5, 40, t=i8)))
no(lambda: M(x=f(5, 100, t=i8), xs=f(5, 3)))
no(lambda: M(x=f(5, 100, t=i8), xs=f(4, 1)))
no(lambda: M(d=(40, 100, 64)), TypeError)
no(lambda: M(d=X.make_w4_desc(0, 100, 64)))
no(lambda: X.xnor_w4_quantize(f(40, 99), d, pk, sc, None, stream=0))
no(lambda: X.xnor_w4_quantize(f(40, 100, t=i8), d, pk, sc, None, stream=0))
no(lambda: X.xnor_w4_quantize(f(100, 40).t(), d, pk, sc, None, stream=0))
no(lambda: X.xnor_w4_pack(f(40, 100, t=i8), d, pk, stream=0))
no(lambda: X.xnor_w4_dequantize(pk, sc, None, d, f(40, 101), stream=0))
""")


RECORD = """
seen = []
vp, ci = ctypes.c_void_p, ctypes.c_int
def record(vp_x, xs, w, s, z, d, r, o, st):
    r, d = ctypes.cast(r, ctypes.POINTER(B.xnor_w4_rows))[0], ctypes.cast(d, ctypes.POINTER(B.xnor_w4_desc))[0]
    seen.append((vp_x, xs, z, (d.N, d.K, d.group), (r.rows, r.x_type, r.x_group, r.out_type, r.x_stride, r.out_stride), o, st))
    return 0
entry = ctypes.CFUNCTYPE(ci, *[vp] * 9)(record)
addresses = [ctypes.cast(getattr(X.load(), "xnor_" + n), vp).value for n in B._MARSHALLED]
addresses[B._MARSHALLED.index("w4_matmul")] = ctypes.cast(entry, vp).value
B._m.bind(addresses, X.xnor_conv_desc, B._address)
class Like:
    is_cuda, device = True, torch.device("cuda", 0)
    def __init__(self, p, dtype, shape, strides): self.p, self.dtype, self.shape, self.strides = p, dtype, shape, strides
    def stride(self): return self.strides
    def data_ptr(self): return self.p
"""


def test_what_the_binding_passes_on():
    """Sizes, types and strides of objects that describe themselves; the stride of a single row is its length."""
    from test_binding import PRELUDE
    run_child("""
d = X.make_w4_desc(40, 100, 64)
pk, sc, z = Like(0x100, torch.int32, (1, 2, 256, 4), (2048, 1024, 4, 1)), Like(0x200, torch.float32, (2, 40), (40, 1)), Like(0x300, torch.uint8, (2, 40), (40, 1))
call = lambda x, xs, o, zz=z: X.xnor_w4_matmul(x, xs, pk, sc, zz, d, o, stream=0x77)
call(Like(0x400, torch.bfloat16, (5, 100), (112, 1)), None, Like(0x500, torch.float32, (5, 40), (48, 1)))
assert seen[-1] == (0x400, None, 0x300, (40, 100, 64), (5, 1, 0, 0, 112, 48), 0x500, 0x77), seen
call(Like(0x400, torch.int8, (1, 100), (7, 1)), Like(0x600, torch.float32, (1, 1), (9, 9)), Like(0x500, torch.float16, (1, 40), (3, 1)), None)
assert seen[-1] == (0x400, 0x600, None, (40, 100, 64), (1, 3, 0, 2, 100, 40), 0x500, 0x77), seen
call(Like(0x400, torch.float8_e4m3fn, (5, 100), (0, 1)), Like(0x600, torch.float32, (5, 2), (2, 1)), Like(0x500, torch.bfloat16, (5, 40), (40, 1)))
assert seen[-1][4] == (5, 4, 64, 1, 0, 40), seen
other = Like(0x500, torch.bfloat16, (5, 40), (40, 1)); other.device = torch.device("cuda", 1)
raises(ValueError, lambda: call(Like(0x400, torch.bfloat16, (5, 100), (100, 1)), None, other))
assert len(seen) == 3
""", PRELUDE + RECORD)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_layout_helpers_agree(group):
    """The tests' own packing is the inverse of their unpacking."""
    import numpy as np
    from rows_util import pack_codes, unpack_codes
    rng = np.random.default_rng(group)
    for N, K in ((1, 1), (17, 65), (40, 200)):
        codes = rng.integers(0, 16, (N, K), dtype=np.uint8)
        assert (unpack_codes(pack_codes(codes), N, K) == codes).all()


def test_the_same_buffer_wants_the_same_rows():
    """Rows of one buffer at two strides would be read after others had been written over them.  (Nothing is launched here:
    calls that are in order are made on a GPU by the tests of the operators.)"""
    lib = X.load()
    a, b, c, e = (ctypes.c_void_p(n << 20) for n in (1, 2, 3, 4))
    fwd = lambda d, s, y: lib.xnor_rmsnorm(a, b, NULL, d, s, y, NULL, NULL)
    for out, stride in ((a, "x_stride"), (b, "residual_stride")):
        for apart in (0, 128):                        # one row for all, or rows apart
            d = norm(**{stride: apart})
            assert fwd(d, c, out) == INV and fwd(d, NULL, out) == INV and fwd(d, out, c) == INV
            assert lib.xnor_rmsnorm_quant(a, b, NULL, d, B.XNOR_I8, 32, out, c, e, NULL, NULL) == INV
    assert fwd(norm(), c, c) == INV                   # two results in one place
    bwd = lambda d, dx: lib.xnor_rmsnorm_backward(a, b, c, NULL, e, d, dx, NULL, NULL, NULL)
    for out, stride in ((a, "y_stride"), (b, "residual_stride")):
        for apart in (0, 128):
            assert bwd(norm(**{stride: apart}), out) == INV


@pytest.mark.parametrize("quant", ["int8", "e4m3_rows", "", "E4M3", 8])
def test_token_block_wants_a_known_kind_of_rows(quant):
    from paper_1603_05279_b200.runner import TokenBlock
    with pytest.raises(ValueError):
        TokenBlock(2, 64, 32, group=32, quant=quant, device="cpu")


def test_token_block_wants_whole_groups():
    from paper_1603_05279_b200.runner import TokenBlock
    for quant in ("i8_groups", "e4m3_groups"):
        with pytest.raises(ValueError):
            TokenBlock(2, 100, 32, group=64, quant=quant, device="cpu")
        assert TokenBlock(2, 128, 32, group=64, quant=quant, device="cpu").q_scales.shape == (2, 2)
    assert TokenBlock(2, 100, 32, group=64, quant="i8", device="cpu").q_scales.shape == (2, 1)


@pytest.mark.parametrize("rows", [1, 40])
def test_a_product_in_the_place_of_its_rows(rows):
    lib = X.load()
    a, b, c, x = (ctypes.c_void_p(n << 20) for n in (1, 2, 3, 4))
    r = ctypes.byref(B.xnor_w4_rows(rows, B.XNOR_BF16, 0, B.XNOR_BF16, 64, 64))
    assert lib.xnor_w4_matmul(x, NULL, a, b, c, ctypes.byref(B.xnor_w4_desc(64, 64, 64)), r, x, NULL) == INV
