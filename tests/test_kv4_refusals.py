"""Calls around the attention over a cache in 4 bits that are refused before anything is launched (no GPU needed)."""
import ctypes

import paper_1603_05279_b200 as X
from paper_1603_05279_b200 import binding as B
from test_binding import run_child

P, Q, ODD, NULL = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000), ctypes.c_void_p(0x1004), ctypes.c_void_p(0)
OK, INV, UNS = B.XNOR_OK, B.XNOR_ERR_INVALID_ARG, B.XNOR_ERR_UNSUPPORTED


def heads(**more):
    d = B.xnor_heads_desc(rows=4, dim=64, q_heads=4, k_heads=2, type=B.XNOR_BF16, weight_type=B.XNOR_F32, norm=1, eps=1e-6, rot=64,
                          pairs=0, positions=10, q_stride=256, k_stride=128, v_stride=128, q_out_stride=256, k_out_stride=128,
                          dq_stride=256, dk_stride=128)
    for k, v in more.items():
        setattr(d, k, v)
    return ctypes.byref(d)


def kv4(**more):
    d = B.xnor_kv4_desc(8, 32, 2, 64, 3, 4)
    for k, v in more.items():
        setattr(d, k, v)
    return ctypes.byref(d)


BAD_HEADS = (dict(rows=-1), dict(dim=0), dict(dim=63), dict(q_heads=-1), dict(k_heads=-1), dict(q_heads=0, k_heads=0), dict(type=B.XNOR_I8),
             dict(type=9), dict(rot=-2), dict(rot=66), dict(rot=3), dict(eps=-1.0), dict(eps=float("nan")), dict(weight_type=B.XNOR_F16),
             dict(positions=0), dict(q_stride=-1), dict(q_out_stride=255))


def test_norm_and_rotation():
    lib = X.load()
    f = lambda d, q=P, k=P, qw=P, kw=P, p=P, r=P, qo=Q, ko=Q: lib.xnor_qk_norm_rope(q, k, qw, kw, p, r, d, qo, ko, NULL)
    b = lambda d, dqo=P, dko=P, q=P, k=P, qw=P, kw=P, p=P, r=P, dq=Q, dk=Q, dqw=P, dkw=P, w=P: \
        lib.xnor_qk_norm_rope_backward(dqo, dko, q, k, qw, kw, p, r, d, dq, dk, dqw, dkw, w, NULL)
    for kw in BAD_HEADS + (dict(k_stride=-1), dict(k_out_stride=127)):
        assert f(heads(**kw)) == INV and b(heads(**kw)) == INV, kw
    assert f(None) == INV and b(None) == INV
    for kw in (dict(q=NULL), dict(k=NULL), dict(qo=NULL), dict(ko=ODD), dict(q=ODD), dict(qw=ODD), dict(kw=ODD), dict(p=NULL), dict(r=NULL), dict(r=ODD)):
        assert f(heads(), **kw) == INV, kw
    for kw in (dict(dqo=NULL), dict(dko=ODD), dict(q=NULL), dict(k=NULL), dict(dq=NULL), dict(dk=ODD), dict(dqw=ODD), dict(w=NULL), dict(p=NULL), dict(r=NULL)):
        assert b(heads(), **kw) == INV, kw
    assert f(heads(q_stride=512), qo=P) == INV and f(heads(k_stride=512), ko=P) == INV           # in place, elsewhere
    assert b(heads(dq_stride=512), dq=P, dqo=P, q=Q) == INV
    for kw in (dict(dim=514, rot=64, q_stride=4000, k_stride=4000, q_out_stride=4000, k_out_stride=4000, dq_stride=4000, dk_stride=4000),
               dict(rows=(1 << 24) + 1), dict(q_heads=65536, q_stride=1 << 23, q_out_stride=1 << 23, dq_stride=1 << 23)):
        assert f(heads(**kw)) == UNS and b(heads(**kw)) == UNS, kw
    assert f(heads(rows=0), q=NULL, k=NULL, qo=NULL, ko=NULL, p=NULL, r=NULL) == OK
    assert b(heads(rows=0), dqo=NULL, dko=NULL, q=NULL, k=NULL, dq=NULL, dk=NULL, dqw=NULL, dkw=NULL, w=NULL, p=NULL, r=NULL) == OK


def test_work():
    assert X.xnor_qk_work_elems(0, 4, 4, 64) == 0 and X.xnor_qk_work_elems(-1, 4, 4, 64) == 0
    assert X.xnor_qk_work_elems(5, 4, 4, 63) == 0 and X.xnor_qk_work_elems(5, 4, 4, 514) == 0 and X.xnor_qk_work_elems((1 << 24) + 1, 4, 4, 64) == 0
    for rows, q, k, dim in ((1, 1, 0, 2), (5, 32, 8, 128), (1 << 24, 128, 128, 512), (1, 0, 65535, 64)):
        n = X.xnor_qk_work_elems(rows, q, k, dim)
        assert n % dim == 0 and 1 <= n // dim <= 2 * 148 + 1
    d = X.make_kv4_desc(8, 32, 2, 64)
    assert X.xnor_kv4_cache_bytes(d) == 8 * 2 * 32 * 72
    assert X.xnor_kv4_work_bytes(d, 10, 5) == 0 and X.xnor_kv4_work_bytes(d, -1, 4) == 0 and X.xnor_kv4_work_bytes(d, 10, 4, type=B.XNOR_F32) == 0
    whole = X.xnor_kv4_work_bytes(d, 100, 8, 4)
    assert all(0 < X.xnor_kv4_work_bytes(d, rows, 8, seqs, most) <= whole for rows in (0, 1, 7, 100) for seqs in (1, 4) for most in (0, 1, 3, 100, 1000))
    for bad in (dict(pages=0), dict(page=8), dict(page=24), dict(page=0), dict(kv_heads=0), dict(dim=0), dict(dim=96), dict(page=65552), dict(kv_heads=4097)):
        d = B.xnor_kv4_desc(8, 32, 2, 64, 3, 4)
        for k, v in bad.items():
            setattr(d, k, v)
        assert X.xnor_kv4_cache_bytes(d) == 0, bad


def test_cache():
    lib = X.load()
    a = lambda h, d, q=P, k=P, v=P, qw=P, kw=P, r=P, s=P, l=P, t=P, qo=Q, c=P: lib.xnor_kv4_append(q, k, v, qw, kw, r, s, l, t, h, d, qo, c, NULL)
    r = lambda d, c=P, s=P, l=P, t=P, ty=B.XNOR_BF16, n=4, k=P, ks=128, v=Q, vs=128: lib.xnor_kv4_read(c, s, l, t, d, ty, n, k, ks, v, vs, NULL)
    m = lambda d, x, q=P, c=P, s=P, l=P, t=P, o=Q, ls=P, w=P: lib.xnor_kv4_attention(q, c, s, l, t, d, x, o, ls, w, NULL)

    def rows(**more):
        x = B.xnor_kv4_rows(4, 4, B.XNOR_BF16, 1, 0.1, 256, 256)
        for k, v in more.items():
            setattr(x, k, v)
        return ctypes.byref(x)

    for kw in (dict(pages=0), dict(page=8), dict(page=24), dict(kv_heads=0), dict(dim=0), dict(seqs=0), dict(table_cols=0)):
        assert a(heads(), kv4(**kw)) == INV and r(kv4(**kw)) == INV and m(kv4(**kw), rows()) == INV, kw
    for kw in (dict(page=65552), dict(seqs=(1 << 20) + 1), dict(page=32768, table_cols=65536), dict(page=16, table_cols=(1 << 27) - 15)):
        assert a(heads(), kv4(**kw)) == UNS and r(kv4(**kw)) == UNS and m(kv4(**kw), rows()) == UNS, kw
    assert a(heads(dim=96, rot=64, q_stride=400, k_stride=400, q_out_stride=400), kv4(dim=96)) == UNS
    assert r(kv4(dim=96), ks=192, vs=192) == UNS and m(kv4(dim=96), rows(q_stride=400, out_stride=400)) == UNS
    assert a(None, kv4()) == INV and a(heads(), None) == INV and r(None) == INV and m(None, rows()) == INV and m(kv4(), None) == INV
    for kw in BAD_HEADS + (dict(k_heads=4, k_stride=256), dict(dim=128, q_stride=512, q_out_stride=512), dict(v_stride=-1), dict(k_stride=-1)):
        assert a(heads(**kw), kv4()) == INV, kw
    for kw in (dict(k=NULL), dict(v=NULL), dict(q=NULL), dict(qo=NULL), dict(k=ODD), dict(v=ODD), dict(kw=ODD), dict(r=NULL), dict(s=NULL),
               dict(l=ODD), dict(t=NULL), dict(c=NULL), dict(c=ODD)):
        assert a(heads(), kv4(), **kw) == INV, kw
    assert a(heads(rot=24), kv4()) == UNS
    assert a(heads(rows=0), kv4(), q=NULL, k=NULL, v=NULL, r=NULL, qo=NULL) == OK
    for kw in (dict(c=NULL), dict(s=ODD), dict(l=NULL), dict(t=NULL), dict(ty=B.XNOR_I8), dict(n=-1), dict(k=NULL), dict(v=ODD), dict(ks=127),
               dict(vs=127), dict(v=P)):
        assert r(kv4(), **kw) == INV, kw
    assert r(kv4(), n=(1 << 24) + 1) == UNS and r(kv4(), n=0, k=NULL, v=NULL) == OK
    for kw in (dict(rows=-1), dict(q_heads=0), dict(q_heads=3), dict(type=7), dict(most=-1), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(q_stride=-1), dict(out_stride=255)):
        assert m(kv4(), rows(**kw)) == INV, kw
    for kw in (dict(q=NULL), dict(q=ODD), dict(c=NULL), dict(s=NULL), dict(l=ODD), dict(t=NULL), dict(o=NULL), dict(o=P), dict(ls=ODD), dict(w=NULL)):
        assert m(kv4(), rows(), **kw) == INV, kw
    assert m(kv4(), rows(type=B.XNOR_F32)) == UNS and m(kv4(), rows(rows=(1 << 24) + 1)) == UNS
    assert m(kv4(), rows(rows=1 << 20, q_heads=2048, q_stride=1 << 17, out_stride=1 << 17)) == UNS
    assert m(kv4(), rows(rows=0), q=NULL, o=NULL, w=NULL) == OK


def test_scratch_of_a_call_is_enough_for_smaller_ones():
    for heads, kv_heads, dim in ((32, 8, 128), (4, 4, 64), (64, 1, 128), (7, 1, 64)):
        d, most_bytes = X.make_kv4_desc(64, 64, kv_heads, dim), {}
        for seqs in (1, 2, 3, 18, 64, 1000):
            for most in (1, 2, 9, 40, 100, 1000, 0):
                before = 0
                for rows in (1, 2, 3, 8, 9, 33, 64, 65, 100, 129, 257, 600, 1025, 4096, 40000):
                    n = X.xnor_kv4_work_bytes(d, rows, heads, seqs, most)
                    key = (rows, most if most else 1 << 30)
                    assert n >= before and all(n >= v for (r, m), v in most_bytes.items() if r <= key[0] and m <= key[1])
                    before = most_bytes[key] = max(n, most_bytes.get(key, 0))
    sizes = [X.xnor_qk_work_elems(rows, 32, 8, 128) for rows in range(1, 3000)]
    assert sizes == sorted(sizes)


def test_the_binding_checks_tensors_against_each_other():
    run_child("""
bf, u8, i32, f32 = torch.bfloat16, torch.uint8, torch.int32, torch.float32
f = lambda *s, t=bf: fake(*s, dtype=t)
def no(call, kind=ValueError): raises(kind, call)
H = lambda q=None, k=None, qw=None, kw=None, eps=1e-6, pos=None, rope=None, qo=None, ko=None: X.xnor_qk_norm_rope(
    f(4, 4, 64) if q is None else q, f(4, 2, 64) if k is None else k, qw, kw, eps, f(4, t=i32) if pos is None else pos,
    f(9, 64, t=f32) if rope is None else rope, False, f(4, 4, 64) if qo is None else qo, f(4, 2, 64) if ko is None else ko, stream=0)
no(lambda: H(q=torch.zeros(4, 4, 64, dtype=bf)))          # on the host
no(lambda: H(q=f(4, 256)))
no(lambda: H(q=f(4, 64, 4).transpose(1, 2)))              # values apart
no(lambda: H(q=f(4, 4, 128)[:, :, :64]))                  # heads apart
no(lambda: H(k=f(5, 2, 64), ko=f(5, 2, 64)))
no(lambda: H(k=f(4, 2, 32), ko=f(4, 2, 32)))
no(lambda: H(k=f(4, 2, 64, t=f32), ko=f(4, 2, 64, t=f32)))
no(lambda: H(qo=f(4, 2, 64)))
no(lambda: H(qo=f(4, 4, 64, t=f32)))
no(lambda: H(qw=f(63)))
no(lambda: H(qw=f(64), kw=f(64, t=f32)))
no(lambda: H(qw=f(64, t=torch.float16)))
no(lambda: H(pos=f(4, t=torch.int64)))
no(lambda: H(pos=f(3, t=i32)))
no(lambda: H(rope=f(9, 66, t=f32)))
no(lambda: H(rope=f(9, 63, t=f32)))
no(lambda: H(rope=f(9, 64)))
no(lambda: H(eps="a"), TypeError)
no(lambda: X.xnor_qk_norm_rope(None, None, None, None, 1e-6, None, None, False, None, None, stream=0))
G = lambda dq=None, dqw=None, w=None: X.xnor_qk_norm_rope_backward(f(4, 4, 64), None, f(4, 4, 64), None, None, None, 1e-6, None, None, False,
    f(4, 4, 64) if dq is None else dq, None, f(64, t=f32) if dqw is None else dqw, None, f(4000, t=f32) if w is None else w, stream=0)
no(lambda: G(dq=f(4, 4, 32)))
no(lambda: G(dqw=f(64)))
no(lambda: G(w=f(63, t=f32)))
d = X.make_kv4_desc(8, 32, 2, 64)
c, st, le, ta = f(8, 2, 2, 16 * 72, t=u8), f(4, t=i32), f(3, t=i32), f(3, 4, t=i32)
A = lambda k=None, v=None, c=c, st=st, le=le, ta=ta, d=d: X.xnor_kv4_append(None, f(4, 2, 64) if k is None else k, f(4, 2, 64) if v is None else v,
    None, None, None, None, False, st, le, ta, d, None, c, stream=0)
R = lambda k=None, v=None, c=c: X.xnor_kv4_read(c, st, le, ta, d, f(4, 2, 64) if k is None else k, f(4, 2, 64) if v is None else v, stream=0)
w = f(X.xnor_kv4_work_bytes(d, 4, 4, 3), t=u8)
M = lambda q=None, o=None, ls=None, w=w, c=c, st=st, scale=0.1, most=1: X.xnor_kv4_attention(f(4, 4, 64) if q is None else q, c, st, le, ta, d, scale, most,
    f(4, 4, 64) if o is None else o, ls, w, stream=0)
no(lambda: A(k=f(4, 4, 64), v=f(4, 4, 64)))
no(lambda: A(v=f(4, 2, 64, t=f32)))
no(lambda: A(c=f(8, 2, 1, 16 * 72, t=u8)))
no(lambda: A(c=f(8, 2, 2, 16 * 72, t=torch.int8)))
no(lambda: A(st=f(3, t=i32)))
no(lambda: A(le=f(3, t=torch.int64)))
no(lambda: A(ta=f(12, t=i32)))
no(lambda: A(ta=f(3, 8, t=i32)[:, ::2]))
no(lambda: A(d=X.make_kv4_desc(8, 24, 2, 64)))
no(lambda: A(d=X.make_w4_desc(8, 24, 32)), TypeError)
no(lambda: X.xnor_kv4_append(None, None, None, None, None, None, None, False, st, le, ta, d, None, c, stream=0))
no(lambda: R(k=f(4, 2, 128), v=f(4, 2, 128)))
no(lambda: R(v=f(5, 2, 64)))
no(lambda: M(q=f(4, 3, 64), o=f(4, 3, 64)))
no(lambda: M(q=f(4, 4, 128), o=f(4, 4, 128)))
no(lambda: M(o=f(4, 4, 64, t=f32)))
no(lambda: M(ls=f(4, 4)))
no(lambda: M(w=f(100, t=u8)))
no(lambda: M(st=f(5, t=i32)))
no(lambda: M(scale="a"), TypeError)
no(lambda: M(most=1.5), TypeError)
for call in (lambda: M(scale=float("nan")), lambda: M(most=-1), lambda: M(q=f(4, 4, 64, t=f32), o=f(4, 4, 64, t=f32))):
    no(call, (X.XnorError, ValueError))
""")
