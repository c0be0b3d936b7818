"""The cache in 4 bits: storing with norm and rotation, and reading back, against the definition in 64 bits."""
import pytest
import torch

import paper_1603_05279_b200 as X
from paper_1603_05279_b200 import binding as B
from kv4_util import TYPES, Batch, cache_parts, heads64, heads_error, quantized, stood_for
from rows_util import Guards, gen, half_step, least, randn

pytestmark = pytest.mark.gpu

# lens, new, kv heads, queries a head, dim, page, rot, pairs, norm, type
CASES = [
    ([1], [1], 1, 1, 64, 16, 64, False, True, "bf16"),
    ([5, 40, 17, 1], [1, 1, 1, 1], 8, 4, 128, 16, 128, False, True, "bf16"),
    ([100, 3, 64, 65], [100, 3, 64, 65], 5, 2, 64, 32, 32, True, True, "f16"),
    ([300, 31], [7, 31], 2, 7, 128, 64, 64, False, False, "f32"),
    ([50, 0, 33, 20], [50, 0, 0, 20], 4, 1, 128, 48, 0, False, True, "bf16"),
    ([2, 40, 0, 9], [5, 3, 2, 9], 3, 2, 64, 16, 64, False, True, "f32"),      # more rows than tokens
    ([1000], [1000], 1, 8, 128, 256, 128, True, True, "f16"),
    ([30] * 70, [1, 2] * 35, 2, 1, 64, 16, 16, False, True, "bf16"),
    ([3] * 33, [1] * 33, 1, 1, 64, 16, 16, False, True, "bf16"),              # how sequences are found: 32 at a time
    ([2] * 1100, [1, 0, 2, 0] * 275, 1, 1, 64, 16, 16, False, True, "f16"),
]


def inputs(batch, group, t, seed, pad=0, rot=0, norm=True):
    g, T, H, D = gen(seed), batch.T + 4, batch.heads, batch.dim       # four rows behind the last sequence
    rows = torch.full((T, (H * group + 2 * H) * D + pad), float("nan"), device="cuda").to(t)
    rows[:, :(H * group + 2 * H) * D] = randn((T, (H * group + 2 * H) * D), g, t, 1.5)
    cut = [H * group * D, (H * group + H) * D, (H * group + 2 * H) * D]
    q, k, v = (rows[:, a:b].unflatten(1, (-1, D)) for a, b in zip([0] + cut, cut))
    k += 1.0                                                          # (ranges that zero does not halve)
    w = [(1 + 0.3 * randn((D,), g)).to(t) for _ in "qk"] if norm else [None, None]
    return q, k, v, w, 1e-6 if norm else None, X.make_rope(max(batch.len_list) + 1, rot) if rot else None


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("pad", [0, 3])
def test_append(case, pad):
    lens, new, H, group, D, page, rot, pairs, norm, t = case
    batch, guards = Batch(lens, new, H, D, page, 1, gap=2 if pad else 0), Guards()
    q, k, v, w, eps, rope = inputs(batch, group, TYPES[t], 3, pad, rot, norm)
    q_out = guards.rows(q.shape[0], H * group * D, TYPES[t], pad)
    q_out.fill_(77)
    cache = guards.rows(1, batch.cache.numel(), torch.uint8).view(batch.cache.shape)
    cache.copy_(batch.cache)
    d = X.make_kv4_desc(batch.pages, page, H, D)
    X.xnor_kv4_append(q, k, v, *w, eps, rope, pairs, batch.starts, batch.lens, batch.table, d, q_out.unflatten(1, (-1, D)), cache)
    X.xnor_check_device()
    guards.check()
    row, seq, pos = batch.rows()
    left = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
    left[row] = False
    assert (q_out[left] == 77).all()                                  # rows that have no place
    if row.numel() == 0:
        assert torch.equal(cache, batch.cache)
        return
    want, size = heads64(q[row], w[0], eps, rope, pos, pairs)
    h = half_step(TYPES[t])
    assert ((q_out[row].unflatten(1, (-1, D)).double() - want).abs() <= h * want.abs() + (1 + h) * heads_error() * size + least(TYPES[t])).all()
    # codes and words exactly, and nothing else in the cache
    at = torch.stack([torch.stack(batch.place(b, p)) for b, p in zip(seq.tolist(), pos)], 1)
    parts, before = cache_parts(cache, D), cache_parts(batch.cache, D)
    x = [heads64(k[row], w[1], eps, rope, pos, pairs)[0].float(), v[row].float()]
    for (codes, words), (codes0, words0), y in zip(parts, before, x):
        c, p = quantized(y)
        codes0[at[0], :, at[1]], words0[at[0], :, at[1]] = c, p
        assert torch.equal(codes, codes0) and torch.equal(words, words0)
    # read back
    k_out, v_out = (guards.rows(q.shape[0], H * D, TYPES[t], pad) for _ in "kv")
    k_out.fill_(55), v_out.fill_(55)
    X.xnor_kv4_read(cache, batch.starts, batch.lens, batch.table, d, k_out.unflatten(1, (H, D)), v_out.unflatten(1, (H, D)))
    X.xnor_check_device()
    guards.check()
    for got, y in ((k_out, x[0]), (v_out, x[1])):
        assert (got[left] == 55).all()
        want = stood_for(*quantized(y))
        assert torch.equal(got[row].unflatten(1, (H, D)), want.float().to(TYPES[t]))


@pytest.mark.parametrize("D", [64, 128])
def test_values_at_borders_and_extremes(D):
    """Quotients that are ties, heads of zeros, of one sign, of one value, of the least numbers, infinities and NaN."""
    T = 12
    batch = Batch([T], [T], 1, D, 16, 2)
    x = torch.zeros(T, 1, D, device="cuda")
    i = torch.arange(D, device="cuda")
    x[1, 0] = (i % 31 - 15) / 2                      # scale 1: half of the quotients are ties
    x[2, 0] = 3.0 + i / D
    x[3, 0] = -5.0
    x[4, 0] = (i % 16) * 2.0 ** -149                 # below what is left of a scale
    x[5, 0] = (i % 16) * 2.0 ** -142
    x[6, 0, 5], x[7, 0, 6], x[8, 0, 7] = float("inf"), float("-inf"), float("nan")
    x[9, 0] = torch.where(i % 2 == 0, 3.4e38, -3.4e38)
    x[10, 0] = torch.where(i == 3, 1e30, 1e-30)
    x[11, 0] = (i % 16 - 7.5) * (1 + 2.0 ** -23)
    d = X.make_kv4_desc(batch.pages, 16, 1, D)
    X.xnor_kv4_append(None, x, x, None, None, None, None, False, batch.starts, batch.lens, batch.table, d, None, batch.cache)
    X.xnor_check_device()
    page, slot = batch.place(0, torch.arange(T, device="cuda"))
    for codes, words in cache_parts(batch.cache, D):
        c, p = quantized(x)
        assert torch.equal(codes[page, :, slot], c) and torch.equal(words[page, :, slot], p)
    k, v = torch.empty_like(x), torch.empty_like(x)
    X.xnor_kv4_read(batch.cache, batch.starts, batch.lens, batch.table, d, k, v)
    assert torch.equal(k.isnan(), v.isnan()) and k[6:9].isnan().all() and not k[:6].isnan().any() and not k[9:].isnan().any()
    assert (k[0] == 0).all()


def test_rotated_keys_are_those_of_the_other_call():
    """One rounding apart: keys stored as they come from xnor_qk_norm_rope in fp32."""
    batch = Batch([40], [40], 2, 128, 16, 3)
    q, k, v, w, eps, rope = inputs(batch, 1, torch.float32, 5, 0, 128)
    d = X.make_kv4_desc(batch.pages, 16, 2, 128)
    X.xnor_kv4_append(q, k, v, *w, eps, rope, False, batch.starts, batch.lens, batch.table, d, torch.empty_like(q), batch.cache)
    (codes, words), _ = cache_parts(batch.cache, 128)
    r = torch.empty_like(k)
    pos = torch.arange(k.shape[0], dtype=torch.int32, device="cuda").clamp(max=40)
    X.xnor_qk_norm_rope(None, k, None, w[1], eps, pos, rope, False, None, r)
    page, slot = batch.place(0, torch.arange(40, device="cuda"))
    got, want = stood_for(codes[page, :, slot], words[page, :, slot]), stood_for(*quantized(r[:40]))
    step = (words[page, :, slot] & ~15).view(torch.float32).double()
    assert ((got - want).abs() <= 1.001 * step[..., None]).all() and ((got - want).abs() > 1e-4 * step[..., None]).double().mean() < 1e-3


def test_places_outside_the_table_and_the_cache():
    """They are left out, everything else is stored, and the next check says so once."""
    H, D = 2, 64
    batch = Batch([40, 20, 33], [40, 20, 33], H, D, 16, 4)
    q, k, v, w, eps, rope = inputs(batch, 1, torch.bfloat16, 6, 0, 64)
    d = X.make_kv4_desc(batch.pages, 16, H, D)
    row, seq, pos = batch.rows()
    good_table = batch.table.clone()
    batch.table[0, 1], batch.table[1, 0] = batch.pages, -1
    cut = batch.table[:, :2].contiguous()                             # the third column is missing
    q_out = torch.full_like(q, 7.0)
    cache = batch.cache.clone()
    X.xnor_kv4_append(q, k, v, *w, eps, rope, False, batch.starts, batch.lens, cut, d, q_out, cache)
    with pytest.raises(X.XnorError) as e:
        X.xnor_check_device()
    assert e.value.status == B.XNOR_ERR_BOUNDS
    X.xnor_check_device()
    stored = (pos < 32) & ~((seq == 0) & (pos >= 16)) & ~((seq == 1) & (pos < 16))
    want = batch.cache.clone()
    batch.table = good_table
    parts = cache_parts(want, D)
    x = [heads64(k[row], w[1], eps, rope, pos, False)[0].float(), v[row].float()]
    at = torch.stack([torch.stack(batch.place(b, p)) for b, p in zip(seq.tolist(), pos)], 1)[:, stored]
    for (codes, words), (codes0, words0), y in zip(cache_parts(cache, D), parts, x):
        codes0[at[0], :, at[1]], words0[at[0], :, at[1]] = quantized(y[stored])
        assert torch.equal(codes, codes0) and torch.equal(words, words0)
    assert not (q_out[row] == 7).all(2).any()                         # queries are rotated all the same
    # a table of rotations that ends early
    X.xnor_kv4_append(q, k, v, *w, eps, rope[:10].contiguous(), False, batch.starts, batch.lens, batch.table, d, q_out.fill_(7.0), cache)
    with pytest.raises(X.XnorError):
        X.xnor_check_device()
    assert (q_out[row][pos >= 10] == 7).all() and not (q_out[row][pos < 10] == 7).all(2).any()


def test_a_cache_of_more_than_four_gigabytes():
    H, D, page = 8, 128, 256
    pages = (5 << 30) // (page * H * (D + 8))
    d = X.make_kv4_desc(pages, page, H, D)
    cache = X.alloc_kv4(d)
    assert cache.numel() == X.xnor_kv4_cache_bytes(d) > 1 << 32
    ids = [pages - 1, 0, pages // 2, pages - 2]
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    n = 3 * page + 17
    g = gen(7)
    k, v = randn((n, H, D), g, torch.bfloat16), randn((n, H, D), g, torch.bfloat16)
    starts, lens = torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    X.xnor_kv4_append(None, k, v, None, None, None, None, False, starts, lens, table, d, None, cache)
    a, b = torch.empty_like(k), torch.empty_like(v)
    X.xnor_kv4_read(cache, starts, lens, table, d, a, b)
    for got, x in ((a, k), (b, v)):
        assert torch.equal(got, stood_for(*quantized(x)).float().to(torch.bfloat16))
    out, lse, work = torch.empty(n, H, D, device="cuda", dtype=k.dtype), torch.empty(n, H, device="cuda"), X.alloc_kv4_work(d, n, H)
    X.xnor_kv4_attention(k, cache, starts, lens, table, d, 0.05, n, out, lse, work)
    X.xnor_check_device()
    # the last token of all, from what was read back: the stored values are a's and b's before their rounding
    K, V = (stood_for(*quantized(x)) for x in (k, v))
    S = torch.einsum("hd,lhd->hl", k[-1].double(), K) * 0.05
    want = torch.einsum("hl,lhd->hd", torch.softmax(S, 1), V)
    assert ((out[-1].double() - want).abs().max() <= 2e-2 * want.abs().max()) and (lse[-1].double() - torch.logsumexp(S, 1)).abs().max() < 1e-3
