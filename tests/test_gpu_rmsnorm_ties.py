"""The 8-bit norm where a quotient lies exactly between two outputs: rounded to even, whatever the row's root.

q = top y / max|y| and y = h rstd weight, so that rstd divides out: q is the rounding of top h weight / max|h weight|.  With
16-bit h and weight both products are exact in 64 bits (22 bits, and 9 more), and so is a border (5 or 8 bits) times the
maximum: comparing the two decides every rounding without one of its own.

The quotient is rounded to fp32 and then to 8 bits.  So one that is off a border b by no more than half a step of fp32,
at most 2^-24 |b|, counts as on it and may go either way.  Of bfloat16 values there is none: with h weight and its maximum in
whole units, at most 2^16 of them, top h weight and b max|h weight| are whole numbers (twice that for the halves of int8) and differ by 1
or more, and the latter is below 31 2^16 (e4m3, powers of two aside) or 255 2^16 (int8), that is below 2^24.  Of
16-bit floats, whose products have 22 bits, there are a few in a million."""
import pytest
import torch

import paper_1603_05279_b200 as X
from rows_util import EPS, TYPES, U, gen, norm64, norm_error, randn

pytestmark = pytest.mark.gpu


def rounded_exactly(h, w, group, qtype):
    """q in 64 bits, [rows][cols], how many quotients lie exactly between two values, and which lie within 2^-24 of that
    without being there."""
    T, D = h.shape
    i8 = qtype == torch.int8
    u = h.double() * (1.0 if w is None else w.double())
    u = u.view(T, -1, group or D)
    m = u.abs().amax(2, keepdim=True)
    n = (127.0 if i8 else 448.0) * u.abs()
    v = torch.where(m > 0, n / m, 0.0)
    step = torch.ones_like(v) if i8 else torch.exp2(torch.floor(torch.log2(v.clamp(min=2.0 ** -6))) - 3)
    low = torch.floor(v / step)                       # (where v is within its rounding of a value, so is the one below)
    twice, border = 2 * n, (2 * low + 1) * step * m
    tie = (twice == border) & (m > 0)
    up = (twice > border) | (tie & (low % 2 == 1))
    q = (low + up) * step * torch.sign(u)
    near = ((twice - border).abs() <= 2.0 ** -24 * border) & ~tie & (m > 0)
    return q.view(T, D), int(tie.sum()), near.view(T, D)


def rows_with_ties(T, D, t, seed, kind):
    g = gen(seed)
    if kind == "normal":                              # as a model has them: few ties, but some
        return randn((T, D), g, t), randn((D,), g, t)
    top = 254 if kind == "halves" else 448            # quotients of int8 are halves; those of e4m3 whole numbers
    h = torch.randint(-top // 2, top // 2 + 1, (T, D), generator=g, device="cuda").float()
    h[:, ::32] = top
    h = (h * torch.exp2(torch.randint(-3, 4, (T, 1), generator=g, device="cuda").float())).to(t)
    return h, None if seed % 2 else torch.full((D,), 0.75, device="cuda").to(t)


@pytest.mark.parametrize("qtype", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("kind", ["normal", "halves", "whole"])
@pytest.mark.parametrize("rows,cols,groups", [(512, 1024, (0, 32, 64, 128)), (64, 4096, (0, 128)), (33, 8320, (0, 64)), (9, 1001, (0,)),
                                              (5, 16512, (0, 128))])
def test_ties_are_decided_exactly(kind, name, qtype, rows, cols, groups):
    ties = 0
    for group in groups:
        h, w = rows_with_ties(rows, cols, TYPES[name], rows + group, kind)
        q, s = X.alloc_rmsnorm_quant(rows, cols, group, qtype)
        rstd = torch.empty(rows, device="cuda")
        X.xnor_rmsnorm_quant(h, None, w, EPS, group, None, q, s, rstd)
        want, n, near = rounded_exactly(h, w, group, qtype)
        ties += n
        assert name == "f16" or not near.any()
        wrong = int(((q.double() != want) & ~near).sum())
        assert wrong == 0, (wrong, n, group)
        # the scale: the maximum is off by the root's error and a product, the scale by a division more
        y = norm64(h, w)[1].view(rows, -1, group or cols).abs().amax(2) / (127.0 if qtype == torch.int8 else 448.0)
        assert ((s.double() - y).abs() <= (norm_error(cols) + U) * y).all()
    if (kind, qtype) in (("halves", torch.int8), ("whole", torch.float8_e4m3fn)) or (kind, name) == ("normal", "bf16"):
        assert ties > 0 or rows * cols < 1 << 18      # the case is what it says


@pytest.mark.parametrize("wname", ["f32", "none"])
def test_ties_of_32_bit_rows_and_weights(wname):
    """Values of few bits in 32-bit rows, and in 32-bit weights beside 16-bit rows."""
    for name, t in TYPES.items():
        w = None if wname == "none" else torch.full((1024,), 1.25, device="cuda")
        for qtype, kind in ((torch.int8, "halves"), (torch.float8_e4m3fn, "whole")):
            h = rows_with_ties(64, 1024, torch.bfloat16, 3, kind)[0].to(t)
            q, s = X.alloc_rmsnorm_quant(64, 1024, 32, qtype)
            X.xnor_rmsnorm_quant(h, None, w, EPS, 32, None, q, s, None)
            want, n, _ = rounded_exactly(h, w, 32, qtype)
            assert torch.equal(q.double(), want) and n > 0, name


@pytest.mark.parametrize("qtype", [torch.int8, torch.float8_e4m3fn])
def test_largest_and_smallest_magnitudes(qtype):
    """Norms up to the end of fp32's range and down to where the scale is subnormal: q stands for y within its step."""
    g = gen(17)
    h = randn((4, 512), g)
    for size in (4e37, 1e37, 1e30, 1.0, 1e-25, 1e-28, 1e-33, 1e-36):
        w = size * (0.5 + torch.rand(512, generator=g, device="cuda"))
        q, s = X.alloc_rmsnorm_quant(4, 512, 128, qtype)
        X.xnor_rmsnorm_quant(h, None, w, EPS, 128, None, q, s, None)
        y = norm64(h, w)[1]
        each = s.double().repeat_interleave(128, 1)
        step = 0.5 * each if qtype == torch.int8 else (2.0 ** -4 * y.abs()).clamp(min=2.0 ** -10 * each)
        # beside the rounding to 8 bits: y's error, the scale's, and half of fp32's least number for y and 128 or 448 of the scale's
        slack = (norm_error(512) + 4 * U) * 2 * y.abs() + 2.0 ** -150 * (1 + 448)
        assert ((q.double() * each - y).abs() <= step + slack).all(), size
