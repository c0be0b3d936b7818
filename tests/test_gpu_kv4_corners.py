"""Attention over the cache in 4 bits where a token or a page spoils a row, against the definition in 64 bits."""
import copy

import pytest
import torch

import paper_1603_05279_b200 as X
from paper_1603_05279_b200 import binding as B
from kv4_util import TYPES, Batch, attention64
from rows_util import U, gen, half_step, least, randn

pytestmark = pytest.mark.gpu

INF = float("inf")


def attend(batch, q, scale, most, table=None):
    T, Hq, D = q.shape
    out, lse = torch.full_like(q, 3.0), torch.full((T, Hq), 3.0, device="cuda")
    d = X.make_kv4_desc(batch.pages, batch.page, batch.heads, D)
    X.xnor_kv4_attention(q, batch.cache, batch.starts, batch.lens, batch.table if table is None else table, d, scale, most, out, lse,
                         X.alloc_kv4_work(d, T, Hq, len(batch.len_list)))
    return out, lse


# lens, new, sequence and token that is NaN.  The first: two blocks' shares of five records are cut before the only one that has the token.
NAN_CASES = [
    ([33, 17], [1, 1], 0, 32),
    ([33, 17], [1, 1], 0, 3),
    ([5000], [1], 0, 4999),
    ([5000], [1], 0, 0),
    ([3000, 1, 40], [2, 1, 3], 0, 2998),
    ([3000], [300], 0, 2700),
]


@pytest.mark.parametrize("case", NAN_CASES, ids=lambda c: "%s-%s-%d-%d" % c)
@pytest.mark.parametrize("D,t", [(64, "f16"), (128, "bf16")])
@pytest.mark.parametrize("which", ["key", "value"])
def test_nan_reaches_every_row_that_sees_it(case, D, t, which):
    """However the context is cut: the outputs of rows that see a key or a value of NaN are NaN; lse is with keys."""
    lens, new, b, p = case
    H, G = 1, 4
    batch = Batch(lens, new, H, D, 16, 201).fill(202)
    q = randn((batch.T, H * G, D), gen(203), TYPES[t])
    want, x, off, lse_off = attention64(batch, q, 0.1)
    page, slot = batch.place(b, torch.tensor(p, device="cuda"))
    batch.cache[..., 16 * D:].view(torch.int32)[page, 0, slot // 16, (0 if which == "key" else 16) + slot % 16] = 0x7FFFFFF8
    out, lse = attend(batch, q, 0.1, max(new))
    X.xnor_check_device()
    r0, first = sum(new[:b]), max(0, p - (lens[b] - new[b]))
    hit = torch.zeros(batch.T, dtype=torch.bool, device="cuda")
    hit[r0 + first:r0 + new[b]] = True
    assert out[hit].isnan().all()
    assert ((out.double() - want).abs() <= off)[~hit].all() and ((lse.double() - x).abs() <= lse_off)[~hit].all()
    assert lse[hit].isnan().all() if which == "key" else ((lse.double() - x).abs() <= lse_off)[hit].all()


@pytest.mark.parametrize("lens,new", [([5000], [1]), ([33, 17], [1, 1]), ([3000], [300])])
def test_a_query_of_nan(lens, new):
    batch = Batch(lens, new, 1, 64, 16, 211).fill(212)
    q = randn((batch.T, 2, 64), gen(213), torch.bfloat16)
    q[0, 1, 7] = float("nan")
    out, lse = attend(batch, q, 0.1, max(new))
    X.xnor_check_device()
    bad = torch.zeros(batch.T, 2, dtype=torch.bool, device="cuda")
    bad[0, 1] = True
    assert torch.equal(lse.isnan(), bad) and torch.equal(out.isnan(), bad[..., None].expand_as(out))


# lens, new, kv heads, queries a head, the pages of sequence 0 that are in the cache (from the end; 0: none)
BLIND_CASES = [
    ([20], [1], 1, 4, 0),
    ([5000], [1], 2, 4, 0),                    # cut among blocks
    ([33, 17], [1, 1], 1, 4, 0),
    ([300, 50], [6, 2], 2, 2, 0),
    ([100], [40], 2, 2, 1),                    # rows before the page that is there
    ([200], [200], 2, 2, 0),
    ([200], [200], 2, 2, 5),
    ([3000, 30], [300, 1], 1, 8, 0),           # cut among blocks
    ([3000], [300], 1, 8, 4),
]


@pytest.mark.parametrize("case", BLIND_CASES, ids=str)
@pytest.mark.parametrize("D,t", [(64, "bf16"), (128, "f16")])
def test_rows_whose_visible_tokens_are_all_outside_the_cache(case, D, t):
    """They see nothing: zeros and -infinity.  The others see what is there."""
    lens, new, H, G, there = case
    batch = Batch(lens, new, H, D, 16, 221).fill(222)
    q = randn((batch.T, H * G, D), gen(223), TYPES[t])
    pages = -(-lens[0] // 16)
    table = batch.table.clone()
    table[0, :pages - there] = torch.where(torch.arange(pages - there, device="cuda") % 2 == 0, batch.pages, -1).int()
    out, lse = attend(batch, q, 0.1, max(new), table)
    with pytest.raises(X.XnorError) as e:
        X.xnor_check_device()
    assert e.value.status == B.XNOR_ERR_BOUNDS
    X.xnor_check_device()
    n, first = new[0], (pages - there) * 16
    blind = torch.arange(lens[0] - n, lens[0], device="cuda") < first
    assert (out[:n][blind] == 0).all() and (lse[:n][blind] == -INF).all()
    if there:
        # a sequence of the tokens that are there, whose first rows come before them
        rest = copy.copy(batch)
        rest.table, rest.len_list, rest.new_list = batch.table[:, pages - there:], [lens[0] - first] + lens[1:], new
        want, x, off, lse_off = attention64(rest, q, 0.1)
        assert ((out.double() - want).abs() <= off)[:n].all() and ((lse.double() - x).abs() <= lse_off)[:n][~blind].all()
    want, x, off, lse_off = attention64(batch, q, 0.1)
    assert ((out.double() - want).abs() <= off)[n:].all() and ((lse.double() - x).abs() <= lse_off)[n:].all()


def row_by_row(batch, q, scale):
    """attention64 of each row with the tokens that it sees, and no others, in its sequence."""
    got = []
    for b, (length, n) in enumerate(zip(batch.len_list, batch.new_list)):
        for i in range(n):
            one = copy.copy(batch)
            one.len_list, one.new_list, one.table, one.gap = [length - n + i + 1], [1], batch.table[b:b + 1], 0
            row = sum(batch.new_list[:b]) + i
            got.append(attention64(one, q[row:row + 1], scale))
    return [torch.cat(v) for v in zip(*got)]


def set_value_scales(batch, b, first, factors):
    """Values of tokens first .. of sequence b times powers of two."""
    page, slot = batch.place(b, first + torch.arange(factors.numel(), device="cuda"))
    words = batch.cache[..., 16 * batch.dim:].view(torch.int32)
    at = (page, slice(None), slot // 16, 16 + slot % 16)
    w = words[at]
    words[at] = ((w & ~15).view(torch.float32) * factors[:, None]).view(torch.int32) | (w & 15)


# lens, new, kv heads, queries a head, token of sequence 0 whose values are large
FEW = [
    ([16], [16], 1, 1, 9),
    ([400], [4], 2, 4, 398),
    ([400], [4], 2, 4, 399),
    ([403, 20], [16, 16], 1, 1, 400),
    ([400, 90], [8, 2], 2, 2, 393),
    ([5000], [3], 1, 5, 4998),
]
MANY = [
    ([150], [150], 2, 1, 70),
    ([150], [150], 2, 4, 149),
    ([400], [200], 2, 4, 290),
    ([400, 30], [200, 3], 1, 16, 399),
    ([300], [300], 1, 1, 140),
    ([3000], [130], 1, 8, 2999),
]


@pytest.mark.parametrize("case", FEW + MANY, ids=lambda c: "%s-%s-%d-%d-%d" % c)
@pytest.mark.parametrize("D", [64, 128])
def test_values_of_later_tokens(case, D):
    """A row is as exact as if the tokens behind it did not exist, however large their values are: one of them 2^40 times the
    others, and all of them growing from token to token."""
    lens, new, H, G, p = case
    first = lens[0] - new[0]
    grow = 2.0 ** (3.0 * torch.arange(new[0], device="cuda")).clamp(max=80)
    for at, factors in ((p, torch.full((1,), 2.0 ** 40, device="cuda")), (first, grow)):
        batch = Batch(lens, new, H, D, 16, 231).fill(232, v_scale=2.0 ** -10)
        set_value_scales(batch, 0, at, factors)
        q = randn((batch.T, H * G, D), gen(233), torch.bfloat16)
        out, lse = attend(batch, q, 0.1, max(new))
        X.xnor_check_device()
        want, x, off, lse_off = row_by_row(batch, q, 0.1)
        assert ((lse.double() - x).abs() <= lse_off).all()
        worst = ((out.double() - want).abs() / off).amax((1, 2))
        assert (worst <= 1).all(), (worst.argmax(), worst.max())


# lens, new, kv heads, queries a head, most
FINE = [
    ([1, 2, 3, 5, 17], [1] * 5, 2, 1, 1),
    ([4, 1, 9], [4, 1, 5], 2, 4, 5),
    ([40, 700], [2, 1], 3, 8, 2),
    ([3000], [1], 1, 2, 1),                      # cut among blocks
    ([150, 130], [150, 130], 1, 1, 150),
    ([130, 200], [130, 4], 2, 4, 130),
    ([2500], [200], 1, 4, 200),                  # cut among blocks
]


@pytest.mark.parametrize("case", FINE, ids=str)
@pytest.mark.parametrize("D", [64, 128])
def test_outputs_in_f16_are_off_by_their_own_rounding(case, D):
    """As attention64 derives it, but weights times scales are rounded in two parts: what F16 leaves of a value x, at most 2^-11 x and exact in
    fp32, is rounded to F16 in its turn, so that 2^-22 x is left, or half a step of the least numbers, 2^-32 of the largest scale.
    Small logits, so that fp32's share is small too."""
    lens, new, H, G, most = case
    batch = Batch(lens, new, H, D, 16, 241).fill(242)
    q = randn((batch.T, H * G, D), gen(243), torch.float16, 0.05)
    scale = 0.125
    out, lse = attend(batch, q, scale, most)
    X.xnor_check_device()
    for b, (length, n) in enumerate(zip(lens, new)):
        K, V = batch.read64(b)
        rows = slice(sum(new[:b]), sum(new[:b]) + n)
        Q = q[rows].double().unflatten(1, (H, G))
        S = torch.einsum("nhgd,lhd->nhgl", Q, K) * scale
        size = torch.einsum("nhgd,lhd->nhgl", Q.abs(), K.abs()).amax(-1) * scale
        hidden = torch.arange(length, device="cuda") > torch.arange(length - n, length, device="cuda")[:, None]
        w = torch.softmax(S.masked_fill(hidden[:, None, None], -INF), -1)
        want, mass = torch.einsum("nhgl,lhd->nhgd", w, V), torch.einsum("nhgl,lhd->nhgd", w, V.abs())
        # logits (2 D + 4) U of their size, their distances below 10: 4 U each, exp2 2^-21; twice, and the sums' chains
        e = 2 * (size * (2 * D + 4) * U + 40 * U + 2.0 ** -21) + (length / 64 + 64) * 2 * U
        off = mass * (e[..., None] + 2.0 ** -22 + (length / 16 + 64) * 2 * U) + 2.0 ** -32 * 2 * 15 * length * V.abs().amax()
        off = off + half_step(torch.float16) * (want.abs() + off) + least(torch.float16)
        worst = ((out[rows].double().unflatten(1, (H, G)) - want).abs() / off).max().item()
        assert worst <= 1, (b, worst)
