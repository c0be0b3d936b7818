"""Norms and rotation of heads, and their gradients, against the definition in 64 bits."""
import pytest
import torch

import paper_1603_05279_b200 as X
from paper_1603_05279_b200 import binding as B
from kv4_util import TYPES, backward_error, heads64, heads_backward64, heads_error, pair_columns, weight_error
from rows_util import Guards, gen, half_step, least, randn

pytestmark = pytest.mark.gpu

# rows, queries' heads, keys' heads, dim, rot, pairs, type, norm
CASES = [
    (1, 32, 8, 128, 128, False, "bf16", True),
    (1, 1, 0, 64, 64, True, "f32", True),
    (3, 0, 5, 128, 64, False, "f16", True),
    (70, 7, 3, 64, 32, True, "bf16", True),
    (33, 5, 2, 256, 256, False, "f16", True),
    (33, 3, 1, 256, 96, True, "f32", True),
    (130, 8, 8, 128, 128, False, "f32", False),
    (5, 4, 4, 64, 0, False, "bf16", True),
    (2, 300, 300, 64, 64, False, "bf16", True),
    (700, 6, 2, 128, 96, False, "bf16", True),
    (4000, 2, 1, 64, 64, False, "f16", True),
    # value by value: heads of other sizes, rotated parts of no whole chunks
    (17, 12, 4, 80, 80, False, "f32", True),
    (17, 3, 2, 80, 40, True, "bf16", True),
    (9, 2, 2, 96, 24, False, "f16", True),
    (9, 4, 4, 2, 2, False, "f32", True),
    (9, 4, 4, 8, 0, False, "bf16", True),
    (5, 1, 1, 512, 512, False, "bf16", True),
    (5, 1, 1, 510, 254, True, "f32", False),
    (40, 2, 2, 128, 20, False, "bf16", True),
    (600, 5, 5, 100, 100, True, "f16", True),
]


def rows_of(T, H, D, t, g, scale=1.0, pad=0):
    """[T][H][D] whose rows lie `pad` values further apart."""
    x = torch.full((T, H * D + pad), float("nan"), device="cuda").to(t)
    x[:, :H * D] = randn((T, H * D), g, t, scale)
    return x[:, :H * D].unflatten(1, (H, D))


def make(case, seed=0, pad=0):
    T, Hq, Hk, D, rot, pairs, t, norm = case
    g, t = gen(seed), TYPES[t]
    s = {"q": rows_of(T, Hq, D, t, g, 2.0, pad) if Hq else None, "k": rows_of(T, Hk, D, t, g, 0.3, pad) if Hk else None}
    wt = t if seed % 2 else torch.float32
    s["qw"], s["kw"] = ((1 + 0.3 * randn((D,), g)).to(wt), (0.3 * randn((D,), g)).to(wt)) if norm else (None, None)
    s["eps"] = 1e-6 if norm else None
    s["rope"] = X.make_rope(T + 50, rot) if rot else None
    s["pos"] = torch.randint(0, T + 50, (T,), generator=g, device="cuda", dtype=torch.int32)
    return s


def new_rows(guards, T, H, D, t, pad):
    return guards.rows(T, H * D, t, pad).unflatten(1, (H, D)) if H else None


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("pad", [0, 8, 3])
def test_forward(case, pad):
    T, Hq, Hk, D, rot, pairs, t, norm = case
    s, guards = make(case, pad, pad), Guards()
    q, k = new_rows(guards, T, Hq, D, TYPES[t], pad), new_rows(guards, T, Hk, D, TYPES[t], pad)
    X.xnor_qk_norm_rope(s["q"], s["k"], s["qw"], s["kw"], s["eps"], s["pos"], s["rope"], pairs, q, k)
    X.xnor_check_device()
    guards.check()
    for got, x, w in ((q, s["q"], s["qw"]), (k, s["k"], s["kw"])):
        if x is None:
            continue
        want, size = heads64(x, w, s["eps"], s["rope"], s["pos"], pairs)
        h = half_step(TYPES[t])
        assert ((got.double() - want).abs() <= h * want.abs() + (1 + h) * heads_error() * size + least(TYPES[t])).all()


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("pad", [0, 8, 3])
def test_backward(case, pad):
    T, Hq, Hk, D, rot, pairs, t, norm = case
    s, guards, g = make(case, pad, pad), Guards(), gen(77)
    dy = {"q": rows_of(T, Hq, D, TYPES[t], g, 0.1, pad) if Hq else None, "k": rows_of(T, Hk, D, TYPES[t], g, 1.0, pad) if Hk else None}
    dx = {"q": new_rows(guards, T, Hq, D, TYPES[t], pad), "k": new_rows(guards, T, Hk, D, TYPES[t], pad)}
    dw = {n: guards.flat(D, torch.float32) for n in "qk"}
    work = guards.flat(max(1, X.xnor_qk_work_elems(T, Hq, Hk, D)), torch.float32)
    call = lambda: X.xnor_qk_norm_rope_backward(dy["q"], dy["k"], s["q"], s["k"], s["qw"], s["kw"], s["eps"], s["pos"], s["rope"],
                                                pairs, dx["q"], dx["k"], dw["q"], dw["k"], work)
    call()
    X.xnor_check_device()
    guards.check()
    for n, H in (("q", Hq), ("k", Hk)):
        if not H or not norm:
            assert (dw[n] == 0).all()
        if not H:
            continue
        want, size, w64, w_size = heads_backward64(dy[n], s[n], s[n + "w"], s["eps"], s["rope"], s["pos"], pairs)
        h = half_step(TYPES[t])
        assert ((dx[n].double() - want).abs() <= h * want.abs() + (1 + h) * backward_error() * size + least(TYPES[t])).all()
        if norm:
            assert ((dw[n].double() - w64).abs() <= weight_error(T, H) * w_size).all()
    first = [v.clone() for v in (*dx.values(), *dw.values()) if v is not None]
    call()
    assert all(torch.equal(a, b) for a, b in zip(first, [v for v in (*dx.values(), *dw.values()) if v is not None]))


def test_gradient_against_differences():
    """Of sum(y c) with respect to x and the weight, by central differences of the formula in 64 bits."""
    for case in ((3, 2, 1, 64, 32, False, "f32", True), (3, 2, 1, 10, 6, True, "f32", True)):
        T, Hq, Hk, D, rot, pairs, t, norm = case
        s, g = make(case, 3), gen(5)
        c = randn((T, Hq, D), g)
        dq, dk = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        dqw, dkw, work = X.alloc_qk_backward(T, Hq, Hk, D)
        X.xnor_qk_norm_rope_backward(c, torch.zeros_like(dk), s["q"], s["k"], s["qw"], s["kw"], s["eps"], s["pos"], s["rope"], pairs,
                                     dq, dk, dqw, dkw, work)
        f = lambda x, w: (heads64(x, w, s["eps"], s["rope"], s["pos"], pairs)[0] * c.double()).sum()
        x, w, e = s["q"].double(), s["qw"].double(), 1e-5
        scale = c.abs().sum().item()
        for at in ((0, 0, 0), (1, 1, D - 1), (2, 0, D // 2), (2, 1, 1)):
            d = torch.zeros_like(x)
            d[at] = e
            # the difference's own error: e^2 times a third derivative (of order 1 / |x|^2 <= 100), and fp32's of the gradient
            assert abs((f(x + d, w) - f(x - d, w)) / (2 * e) - dq[at]).item() <= (1e-7 + 80 * 2.0 ** -24 * 4) * scale
        for at in (0, D // 2, D - 1):
            d = torch.zeros_like(w)
            d[at] = e
            assert abs((f(x, w + d) - f(x, w - d)) / (2 * e) - dqw[at]).item() <= (1e-7 + 100 * 2.0 ** -24 * 4) * scale
        assert (dk == 0).all() and (dkw == 0).all()


@pytest.mark.parametrize("D", [128, 80])
def test_in_place_and_views_of_a_product(D):
    """Queries and keys side by side in one product's rows, rotated where they are."""
    T, Hq, Hk = 50, 4, 2
    g = gen(8)
    rows = randn((T, (Hq + 2 * Hk) * D), g, torch.bfloat16)
    q, k = rows[:, :Hq * D].unflatten(1, (Hq, D)), rows[:, Hq * D:(Hq + Hk) * D].unflatten(1, (Hk, D))
    rope, pos = X.make_rope(T, D), torch.arange(T, dtype=torch.int32, device="cuda").flip(0).contiguous()
    before, q2, k2 = rows.clone(), torch.empty(T, Hq, D, device="cuda", dtype=rows.dtype), torch.empty(T, Hk, D, device="cuda", dtype=rows.dtype)
    X.xnor_qk_norm_rope(q, k, None, None, 1e-6, pos, rope, False, q2, k2)
    assert torch.equal(rows, before)
    X.xnor_qk_norm_rope(q, k, None, None, 1e-6, pos, rope, False, q, k)
    assert torch.equal(q, q2) and torch.equal(k, k2) and torch.equal(rows[:, (Hq + Hk) * D:], before[:, (Hq + Hk) * D:])
    # gradients in the place of those that arrive
    x, d1, d2 = randn((T, Hq, D), g, torch.bfloat16), torch.empty(T, Hq, D, device="cuda", dtype=rows.dtype), q2.clone()
    X.xnor_qk_norm_rope_backward(q2, None, x, None, None, None, 1e-6, pos, rope, False, d1, None, None, None, None)
    X.xnor_qk_norm_rope_backward(d2, None, x, None, None, None, 1e-6, pos, rope, False, d2, None, None, None, None)
    assert torch.equal(d1, d2)


def test_one_row_for_all_and_no_rows():
    x = randn((1, 4, 128), gen(1), torch.bfloat16).expand(9, 4, 128)
    pos, rope = torch.arange(9, dtype=torch.int32, device="cuda"), X.make_rope(9, 128)
    y, z = torch.empty(9, 4, 128, device="cuda", dtype=x.dtype), torch.empty(9, 4, 128, device="cuda", dtype=x.dtype)
    X.xnor_qk_norm_rope(x, None, None, None, 1e-6, pos, rope, False, y, None)
    X.xnor_qk_norm_rope(x.contiguous(), None, None, None, 1e-6, pos, rope, False, z, None)
    assert torch.equal(y, z)
    e = torch.empty(0, 4, 128, device="cuda", dtype=x.dtype)
    X.xnor_qk_norm_rope(e, None, None, None, 1e-6, pos[:0], rope, False, e.clone(), None)
    dw, _, _ = X.alloc_qk_backward(1, 4, 0, 128)
    dw.fill_(7)
    X.xnor_qk_norm_rope_backward(e, None, e, None, None, None, 1e-6, pos[:0], rope, False, e.clone(), None, dw, None, None)
    assert (dw == 0).all()


@pytest.mark.parametrize("D", [64, 80])
def test_positions_outside_the_table(D):
    """Such tokens are left as they are, add nothing to the weight's gradient, and the next check says so once."""
    T, H = 6, 3
    g = gen(4)
    x, dy = randn((T, H, D), g), randn((T, H, D), g)
    rope = X.make_rope(10, D)
    pos = torch.tensor([0, -1, 9, 10, 2 ** 31 - 1, 3], dtype=torch.int32, device="cuda")
    good = torch.tensor([0, 2, 5], device="cuda")
    bad = torch.tensor([1, 3, 4], device="cuda")
    y = torch.full((T, H, D), 123.0, device="cuda")
    X.xnor_qk_norm_rope(x, None, None, None, 1e-6, pos, rope, False, y, None)
    with pytest.raises(X.XnorError) as e:
        X.xnor_check_device()
    assert e.value.status == B.XNOR_ERR_BOUNDS
    X.xnor_check_device()
    assert (y[bad] == 123).all()
    want, size = heads64(x[good], None, 1e-6, rope, pos[good], False)
    assert ((y[good].double() - want).abs() <= 2.0 ** -24 * want.abs() + 1.1 * heads_error() * size).all()
    dx = torch.full((T, H, D), 123.0, device="cuda")
    dw, _, work = X.alloc_qk_backward(T, H, 0, D)
    X.xnor_qk_norm_rope_backward(dy, None, x, None, None, None, 1e-6, pos, rope, False, dx, None, dw, None, work)
    with pytest.raises(X.XnorError):
        X.xnor_check_device()
    assert (dx[bad] == 123).all()
    w64, size = heads_backward64(dy[good], x[good], None, 1e-6, rope, pos[good], False)[2:]
    assert ((dw.double() - w64).abs() <= weight_error(T, H) * size).all()


def test_zeros_infinities_and_far_positions():
    x = torch.zeros(4, 2, 128, device="cuda")
    x[1, 0, 3], x[2, 1, 70] = float("inf"), float("nan")
    rope, pos = X.make_rope(1 << 20, 128), torch.tensor([0, 5, (1 << 20) - 1, 9], dtype=torch.int32, device="cuda")
    y = torch.empty_like(x)
    X.xnor_qk_norm_rope(x, None, None, None, 1e-6, pos, rope, False, y, None)
    assert (y[0] == 0).all() and (y[3] == 0).all() and (y[1, 1] == 0).all() and (y[2, 0] == 0).all()
    assert y[1, 0, 3].isnan() and y[2, 1].isnan().all()
    x = randn((4, 2, 128), gen(2))
    X.xnor_qk_norm_rope(x, None, None, None, None, pos, rope, False, y, None)
    a, b = pair_columns(128, 128, False)
    angle = pos.double()[:, None, None] * 10000.0 ** (-torch.arange(64, device="cuda").double() / 64)
    want = x[..., a].double() * angle.cos() - x[..., b].double() * angle.sin()
    assert ((y[..., a].double() - want).abs() <= 4 * 2.0 ** -24 * (x[..., a].abs() + x[..., b].abs()).double()).all()
