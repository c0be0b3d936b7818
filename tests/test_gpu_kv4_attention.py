"""Attention over the cache in 4 bits, against the definition in 64 bits."""
import pytest
import torch

import paper_1603_05279_b200 as X
from paper_1603_05279_b200 import binding as B
from kv4_util import TYPES, Batch, attention64, put, quantized
from rows_util import Guards, U, gen, half_step, randn

pytestmark = pytest.mark.gpu

# lens, new, kv heads, queries a head, dim, page, type, most
CASES = [
    ([1], [1], 1, 1, 64, 16, "bf16", 1),
    ([2], [2], 1, 1, 128, 16, "f16", 2),
    ([16], [1], 1, 8, 128, 16, "bf16", 1),
    ([17, 15, 33], [1, 1, 1], 2, 4, 128, 16, "bf16", 1),
    ([5000], [1], 8, 4, 128, 16, "bf16", 1),
    ([5000], [1], 1, 1, 64, 64, "f16", 1),
    ([700, 1, 0, 300, 64], [1, 1, 0, 1, 1], 5, 7, 64, 32, "bf16", 1),
    ([300, 31, 2000], [5, 31, 3], 4, 4, 64, 32, "f16", 0),
    ([90, 1000], [1, 9], 2, 1, 128, 48, "f16", 9),
    ([2, 40, 0, 9], [5, 3, 2, 9], 3, 2, 64, 16, "bf16", 9),                   # more rows than tokens
    ([30] * 70, [1, 2] * 35, 2, 8, 128, 16, "bf16", 2),
    ([12] * 1100, [1] * 1100, 1, 2, 64, 16, "f16", 1),
    ([100], [100], 2, 4, 128, 64, "bf16", 100),
    ([333, 700], [333, 20], 1, 16, 128, 128, "bf16", 333),
    ([400, 50], [130, 50], 2, 5, 64, 16, "f16", 0),
    ([3000], [300], 1, 8, 128, 64, "bf16", 300),
    ([1500, 1500, 129], [1500, 1, 129], 2, 2, 128, 256, "f16", 1500),
    ([600, 128], [600, 128], 4, 1, 64, 64, "bf16", 1),                        # most too small
    ([40, 20], [40, 20], 1, 100, 64, 16, "bf16", 40),
]


def run(batch, q, scale, most, pad=0, guards=None, lse=True, fill=3.0):
    T, Hq, D = q.shape
    guards = guards or Guards()
    out = guards.rows(T, Hq * D, q.dtype, pad)
    out.fill_(fill)
    stats = guards.rows(T, Hq, torch.float32) if lse else None
    if lse:
        stats.fill_(fill)
    d = X.make_kv4_desc(batch.pages, batch.page, batch.heads, D)
    work = guards.flat(X.xnor_kv4_work_bytes(d, T, Hq, len(batch.len_list), most), torch.uint8)
    X.xnor_kv4_attention(q, batch.cache, batch.starts, batch.lens, batch.table, d, scale, most, out.unflatten(1, (Hq, D)), stats, work)
    X.xnor_check_device()
    guards.check()
    return out.unflatten(1, (Hq, D)), stats


def check(batch, q, scale, out, lse, fill=3.0):
    want, x, off, lse_off = attention64(batch, q, scale)
    n = batch.T
    assert (out[:batch.gap] == fill).all() and (out[n:] == fill).all() and (lse is None or (lse[:batch.gap] == fill).all())
    rows = slice(batch.gap, n)
    worst = ((out.double() - want).abs() / off)[rows].max().item() if n > batch.gap else 0.0
    assert worst <= 1, worst
    if lse is not None:
        assert (lse[n:] == fill).all()
        blind = x[rows] == -float("inf")
        assert torch.equal(lse[rows] == -float("inf"), blind)
        assert ((lse[rows].double() - x[rows]).abs() <= lse_off[rows])[~blind].all()


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%s-%d-%d-%d-%d-%s-%d" % (str(c[0])[:16], str(c[1])[:16], *c[2:]))
@pytest.mark.parametrize("pad", [0, 3])
def test_attention(case, pad):
    lens, new, H, G, D, page, t, most = case
    batch = Batch(lens, new, H, D, page, 11, gap=1 if pad else 0).fill(12)
    g = gen(13)
    q = torch.full((batch.T + 2, H * G * D + pad), float("nan"), device="cuda").to(TYPES[t])
    q[:, :H * G * D] = randn((batch.T + 2, H * G * D), g, TYPES[t])
    q = q[:, :H * G * D].unflatten(1, (H * G, D))
    scale = D ** -0.5 * (3 if pad else 1)
    check(batch, q, scale, *run(batch, q, scale, most, pad))


@pytest.mark.parametrize("new,most", [(1, 1), (4, 4), (200, 200)])
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_peaked_and_scaled(new, most, t):
    """Logits of hundreds, maxima that rise on the way, values of any size, a scale below zero and of zero."""
    for scale, k_scale, v_scale in ((1.0, 3.0, 1.0), (0.1, 1.0, 1e-5), (-0.3, 1.0, 1e4), (0.0, 1.0, 1.0), (0.3, 1e-8, 1e-20 if t == "bf16" else 1e-3)):
        batch = Batch([400, 1000], [new, min(3, new)], 2, 64, 16, 21).fill(22, k_scale, v_scale)
        q = randn((batch.T, 8, 64), gen(23), TYPES[t])
        out, lse = run(batch, q, scale, most)
        check(batch, q, scale, out, lse)
    # growing keys: every record has a new maximum
    batch = Batch([900], [new], 1, 64, 16, 24).fill(25)
    words = batch.cache[..., 16 * 64:].view(torch.int32)
    for p in range(0, 900, 16):
        page, slot = batch.place(0, torch.tensor(p, device="cuda"))
        s = torch.full((16,), 1e-3 * (1 + p), device="cuda").view(torch.int32) & ~15
        words[page, 0, slot // 16, :16] = s | 7
    q = randn((batch.T, 4, 64), gen(26), TYPES[t])
    check(batch, q, 0.5, *run(batch, q, 0.5, most))


@pytest.mark.parametrize("new,most", [(3, 3), (150, 150)])
@pytest.mark.parametrize("D", [64, 128])
def test_what_is_not_seen_may_stand_for_anything(new, most, D):
    """Tokens behind the last, in the same record and page, whose scales are NaN, infinite or huge; queries of blind rows that are NaN;
    and later tokens, NaN, which earlier rows do not see."""
    batch = Batch([150, 40, 1], [new, 2, 4], 2, D, 32, 31).fill(32)
    last = [150, 40, 1]
    odd = torch.tensor([float("nan"), float("inf"), 1e38, -1e38], device="cuda").view(torch.int32) & ~15
    words = batch.cache[..., 16 * D:].view(torch.int32)
    for b, n in enumerate(last):
        for p in range(n, -(-n // 32) * 32):
            page, slot = batch.place(b, torch.tensor(p, device="cuda"))
            words[page, :, slot // 16, slot % 16] = odd[p % 4]
            words[page, :, slot // 16, 16 + slot % 16] = odd[(p + 1) % 4]
    q = randn((batch.T, 8, D), gen(33), torch.bfloat16)
    q[new + 2:new + 5] = float("nan")                    # three rows come before their sequence's first token
    out, lse = run(batch, q, 0.1, most)
    check(batch, q.nan_to_num(0.0), 0.1, out, lse)
    # the last token of sequence 0 is NaN: only its last row sees it
    page, slot = batch.place(0, torch.tensor(149, device="cuda"))
    words[page, 1, slot // 16, slot % 16] = 0x7FFFFFF8
    out2, lse2 = run(batch, q, 0.1, most)
    seen = torch.zeros(batch.T, 8, dtype=torch.bool, device="cuda")
    seen[new - 1, 4:] = True
    assert out2[seen].isnan().all() and torch.equal(out2[~seen], out[~seen]) and torch.equal(lse2[~seen], lse[~seen])


@pytest.mark.parametrize("new,most", [(1, 1), (140, 140)])
def test_lengths_tables_and_pages_that_are_wrong(new, most):
    """A page outside the cache and tokens outside the table are not seen, and the next check says so once."""
    H, D = 2, 64
    batch = Batch([300, 200], [new, new], H, D, 16, 41).fill(42)
    q = randn((batch.T, 4, D), gen(43), torch.bfloat16)
    d = X.make_kv4_desc(batch.pages, 16, H, D)
    out, lse, work = torch.empty_like(q), torch.empty(batch.T, 4, device="cuda"), X.alloc_kv4_work(d, batch.T, 4, 2)
    call = lambda lens, table: X.xnor_kv4_attention(q, batch.cache, batch.starts, lens, table, d, 0.1, most, out, lse, work)
    bad = batch.table.clone()
    bad[0, 2], bad[0, 5] = batch.pages, -3
    call(batch.lens, bad)
    with pytest.raises(X.XnorError) as e:
        X.xnor_check_device()
    assert e.value.status == B.XNOR_ERR_BOUNDS
    X.xnor_check_device()
    K, V = batch.read64(0)
    keep = torch.ones(300, dtype=torch.bool, device="cuda")
    keep[32:48] = keep[80:96] = False
    S = torch.einsum("hgd,lhd->hgl", q[new - 1].double().unflatten(0, (H, 2)), K[keep]) * 0.1
    want = torch.einsum("hgl,lhd->hgd", torch.softmax(S, -1), V[keep]).flatten(0, 1)
    assert (out[new - 1].double() - want).abs().max() < 2e-2 * want.abs().max()
    assert (lse[new - 1].double() - torch.logsumexp(S, -1).flatten()).abs().max() < 1e-4
    # the other sequence; how sums are shared out, so their last bits, goes by all lengths
    other, _, off, _ = attention64(batch, q, 0.1)
    same = lambda: ((out.double() - other).abs() <= off)[new:].all()
    assert same()
    call(torch.tensor([2 ** 31 - 1, 200], dtype=torch.int32, device="cuda"), batch.table)     # a length that no table has
    with pytest.raises(X.XnorError):
        X.xnor_check_device()
    assert same()
    call(torch.tensor([-5, 200], dtype=torch.int32, device="cuda"), batch.table)
    X.xnor_check_device()
    assert (out[:new] == 0).all() and same()


def test_no_rows_no_lse_and_the_same_bits():
    batch = Batch([1000, 50], [3, 2], 2, 128, 16, 51).fill(52)
    q = randn((5, 8, 128), gen(53), torch.bfloat16)
    a, lse = run(batch, q, 0.1, 3)
    b, _ = run(batch, q, 0.1, 3, lse=False)
    assert torch.equal(a, b)
    d = X.make_kv4_desc(batch.pages, 16, 2, 128)
    X.xnor_kv4_attention(q[:0], batch.cache, batch.starts, batch.lens, batch.table, d, 0.1, 0, q[:0].clone(), None,
                         torch.empty(X.xnor_kv4_work_bytes(d, 0, 8), dtype=torch.uint8, device="cuda"))
    X.xnor_check_device()


def test_sequences_that_share_pages():
    """Two sequences whose first pages are the same ones: both read them."""
    batch = Batch([200, 200], [1, 1], 2, 64, 16, 61).fill(62)
    batch.table[1, :10] = batch.table[0, :10]
    q = randn((2, 4, 64), gen(63), torch.bfloat16)
    check(batch, q, 0.2, *run(batch, q, 0.2, 1))


@pytest.mark.parametrize("new,most", [(3, 3), (150, 150)])
@pytest.mark.parametrize("D", [64, 128])
def test_logits_of_any_size(new, most, D):
    """Keys of 10^30, and the largest of them ever later: a row is then the value of one token."""
    L, H, G = 700, 2, 2
    for rising in (False, True):
        batch = Batch([L], [new], H, D, 16, 71).fill(72)
        words = batch.cache[..., 16 * D:].view(torch.int32)
        page, slot = batch.place(0, torch.arange(L, device="cuda"))
        size = 1e30 * (1 + torch.arange(L, device="cuda")) ** 2 if rising else torch.full((L,), 1e30, device="cuda")
        words[page, :, slot // 16, slot % 16] = (size.float().view(torch.int32) & ~15)[:, None] | (words[page, :, slot // 16, slot % 16] & 15)
        q = randn((new, H * G, D), gen(73), torch.bfloat16)
        out, lse = run(batch, q, 0.1, most)
        assert out.isfinite().all() and lse.isfinite().all()
        K, V = batch.read64(0)
        S = 0.1 * torch.einsum("nhgd,lhd->nhgl", q.double().unflatten(1, (H, G)), K)
        mass = 0.1 * torch.einsum("nhgd,lhd->nhgl", q.double().abs().unflatten(1, (H, G)), K.abs())
        hidden = torch.arange(L, device="cuda") > torch.arange(L - new, L, device="cuda")[:, None]
        S = S.masked_fill(hidden[:, None, None], -float("inf"))
        two, at = S.topk(2, -1)
        # a logit's products and sums are off by (2 D + 5) U of their magnitudes' sum: where the first is ahead by more than both are off, and 100
        clear = two[..., 0] - two[..., 1] > 100 + 2 * (2 * D + 5) * U * mass.masked_fill(hidden[:, None, None], 0.0).amax(-1)
        assert clear.float().mean() > 0.9
        want = V[at[..., 0], torch.arange(H, device="cuda")[:, None]]                 # [new][H][G][D]
        # a weight of 1 (the rest together below 700 e^-100) times the scale, to 11 bits: off by 2^-11
        off = want.abs() * (2.0 ** -11 + 64 * U)
        off = off + half_step(torch.bfloat16) * (want.abs() + off)
        assert ((out.double().unflatten(1, (H, G)) - want).abs() <= off)[clear].all()
        assert ((lse.double().unflatten(1, (H, G)) - two[..., 0]).abs() <= (2 * D + 10) * U * mass.masked_fill(hidden[:, None, None], 0.0).amax(-1)).all()


@pytest.mark.parametrize("new,most", [(4, 4), (150, 150)])
def test_queries_of_a_wide_range(new, most):
    """bfloat16 queries with values 2^26 apart, the large ones where all keys are zero; rows of very small ones."""
    batch, D, H = Batch([300], [new], 2, 64, 16, 81).fill(82), 64, 2
    page, slot = batch.place(0, torch.arange(300, device="cuda"))
    x = randn((300, H, D), gen(83))
    x[..., 5] = x[..., 40] = 0
    put(batch.cache, D, False, page, slot, *quantized(x))
    q = randn((new, 4, D), gen(84), torch.bfloat16)
    q[0] *= 2.0 ** -60
    q[1] *= 2.0 ** -126
    q[..., 5] = 2.0 ** 20
    q[2:, :, 40] = -1.5 * 2.0 ** 26
    q[1, :, 5] = 0
    check(batch, q, 0.3, *run(batch, q, 0.3, most))


@pytest.mark.parametrize("seqs,heads", [(3, 2), (40, 4)])
def test_sequences_of_all_sizes_in_one_call(seqs, heads):
    """Some of a batch's sequences have few new tokens, some many, on both sides of where the kernels meet."""
    new = [(1, 130, 16, 47, 33, 48, 0, 17, 49)[i % 9] for i in range(seqs)]
    batch = Batch([n + 150 - 3 * i for i, n in enumerate(new)], new, heads, 64, 16, 91).fill(92)
    q = randn((batch.T, 2 * heads, 64), gen(93), torch.float16)
    check(batch, q, 0.2, *run(batch, q, 0.2, 0))


@pytest.mark.parametrize("most", [0, 700])
def test_short_sequences_beside_long_prompts(most):
    """Rows of short ones, whose context many blocks share, next to prompts that make up nearly all of the call's rows."""
    lens, new = [700, 3000, 1, 650, 2500, 0], [700, 1, 1, 650, 24, 0]
    batch = Batch(lens, new, 2, 64, 32, 101).fill(102)
    q = randn((batch.T, 8, 64), gen(103), torch.bfloat16)
    check(batch, q, 0.2, *run(batch, q, 0.2, most))
