"""Plain 64-bit definitions of norms and rotations of heads, of the cache in 4 bits and of the attention over it."""
import math

import torch

from rows_util import U, gen, half_step, least, randn

HEADS_EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---- norms and rotation -----------------------------------------------------------------------
def pair_columns(dim, rot, pairs):
    """Columns of the first and the second of each pair."""
    i = torch.arange(rot // 2, device="cuda")
    return (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)


def rotated(x, cos, sin, rot, pairs, size=False):
    """x [rows][heads][dim] turned; size: the sum of the magnitudes that are added instead."""
    a, b = pair_columns(x.shape[2], rot, pairs)
    u, v, y = x[..., a], x[..., b], x.clone()
    if size:
        y = y.abs()
        y[..., a], y[..., b] = (u * cos).abs() + (v * sin).abs(), (v * cos).abs() + (u * sin).abs()
    else:
        y[..., a], y[..., b] = u * cos - v * sin, v * cos + u * sin
    return y


def angles(rope, positions):
    c, s = rope[positions.long()].double().chunk(2, 1)
    return c[:, None], s[:, None]


def heads64(x, weight, eps, rope, positions, pairs):
    """(values, their size) in 64 bits of stored values x."""
    y = x.double()
    if eps is not None:
        eps = torch.tensor(eps, dtype=torch.float32).double().item()
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * (1.0 if weight is None else weight.double())
    if rope is None or rope.shape[1] == 0:
        return y, y.abs()
    c, s = angles(rope, positions)
    return rotated(y, c, s, rope.shape[1], pairs), rotated(y, c, s, rope.shape[1], pairs, True)


def heads_error():
    """Of a value in fp32, relative to its size.  The squares' sum: chains of up to 16 products added, a tree of 5 steps
    and at most two more roundings for the mean and eps, so 24 U, half of it for the root; root and reciprocal 2 U,
    the products with weight and value 2 U, two products and their sum 2 U."""
    return (12 + 2 + 2 + 2) * U


def heads_backward64(dy, x, weight, eps, rope, positions, pairs):
    """(dx, its size, dweight, its size) in 64 bits."""
    g, gs = dy.double(), dy.double().abs()
    if rope is not None:
        c, s = angles(rope, positions)
        g, gs = rotated(g, c, -s, rope.shape[1], pairs), rotated(g, c, s, rope.shape[1], pairs, True)
    if eps is None:
        return g, gs, None, None
    x, w = x.double(), torch.ones(x.shape[2], device="cuda").double() if weight is None else weight.double()
    eps = torch.tensor(eps, dtype=torch.float32).double().item()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    dx = r * (g * w - x * (r * r * (g * w * x).mean(-1, keepdim=True)))
    size = r * (gs * w.abs() + x.abs() * (r * r * (gs * w.abs() * x.abs()).mean(-1, keepdim=True)))
    return dx, size, (g * x * r).sum((0, 1)), (gs * (x * r).abs()).sum((0, 1))


def backward_error():
    """The turned gradient 2 U, the products in the sum of u x 2 U, its chain of 16, tree of 5, mean 1 U: 26 U; rstd 14 U (as
    above without the value's products) three times, and five products and sums: 26 + 42 + 5, rounded up."""
    return 80 * U


def weight_error(rows, heads):
    """Each term: the turned gradient 2 U, rstd 14 U, two products 2 U; then additions, of which no value passes more than there are rows of heads, and
    the block's (32) and the grid's (up to 8 + 8 + 32)."""
    return (18 + rows * heads + 80) * U


# ---- the cache --------------------------------------------------------------------------------
def quantized(x):
    """(codes, words) of stored fp32 values [..][dim]: the definition, in 64 bits."""
    x = x.float().double()
    lo, hi = x.amin(-1).clamp(max=0), x.amax(-1).clamp(min=0)
    word = ((hi - lo) / 15).float().view(torch.int32) & ~15
    s = word.view(torch.float32).double()
    sound = torch.isfinite(x).all(-1) & (s > 0)
    z = torch.where(sound, torch.round(-lo / s).clamp(0, 15), 8.0)
    q = torch.where(sound[..., None], torch.round(x / s[..., None]) + z[..., None], 8.0).clamp(0, 15)
    word = torch.where(torch.isfinite(x).all(-1), word, torch.full_like(word, 0x7FFFFFF0))
    return q.to(torch.uint8), word | z.to(torch.int32)


def stood_for(codes, words):
    return (codes.double() - (words & 15).double()[..., None]) * (words & ~15).view(torch.float32).double()[..., None]


def cache_parts(cache, dim):
    """(codes [pages][heads][page][dim], words [pages][heads][page]) of keys, and of values, by the documented layout."""
    pages, heads, records, _ = cache.shape
    got = []
    for first, word in ((0, 16 * dim), (8 * dim, 16 * dim + 64)):
        b = cache[..., first:first + 8 * dim].reshape(pages, heads, records * 16, dim // 8, 4).int()
        w = b[..., 0] | b[..., 1] << 8 | b[..., 2] << 16 | b[..., 3] << 24
        codes = torch.stack([(w >> (4 * (c // 2) + 16 * (c % 2))) & 15 for c in range(8)], -1).flatten(-2).to(torch.uint8)
        got.append((codes, cache[..., word:word + 64].contiguous().view(torch.int32).flatten(2)))
    return got


def put(cache, dim, values, page, slot, codes, words):
    """Codes [n][heads][dim] and words [n][heads] into places (page, slot) [n], by the documented layout."""
    w = torch.zeros(codes.shape[:-1] + (dim // 8,), dtype=torch.int64, device="cuda")
    c = codes.long().unflatten(-1, (-1, 8))
    for i in range(8):
        w |= c[..., i] << (4 * (i // 2) + 16 * (i % 2))
    b = torch.stack([(w >> (8 * i)) & 255 for i in range(4)], -1).flatten(-2).to(torch.uint8)
    first = 8 * dim if values else 0
    cache[..., first:first + 8 * dim].unflatten(3, (16, dim // 2))[page, :, slot // 16, slot % 16] = b
    cache[..., 16 * dim:].view(torch.int32)[page, :, slot // 16, (16 if values else 0) + slot % 16] = words


class Batch:
    """Sequences with `new` new tokens of `lens` in all, in a cache whose other bytes are anything."""

    def __init__(self, lens, new, heads, dim, page, seed, spare=3, gap=0):
        g = gen(seed)
        self.len_list, self.new_list, self.heads, self.dim, self.page = list(lens), list(new), heads, dim, page
        cols = max(1, -(-max(lens) // page))
        need = [-(-n // page) for n in lens]
        self.pages = sum(need) + spare
        free = torch.randperm(self.pages, generator=g, device="cuda").int()
        self.table = torch.full((len(lens), cols), -7, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = free[at:at + n]
            at += n
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.starts = torch.tensor([gap + sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
        self.gap, self.T = gap, gap + sum(new)
        self.cache = torch.randint(0, 256, (self.pages, heads, page // 16, 16 * (dim + 8)), generator=g, dtype=torch.uint8, device="cuda")

    def place(self, b, p):
        """(page, slot) of tokens p of sequence b."""
        return self.table[b, p // self.page].long(), p % self.page

    def rows(self):
        """(row, sequence, token) of each new token that has a place."""
        got = []
        for b, (length, n) in enumerate(zip(self.len_list, self.new_list)):
            for i in range(n):
                if length - n + i >= 0:
                    got.append((self.gap + sum(self.new_list[:b]) + i, b, length - n + i))
        return torch.tensor(got, dtype=torch.int64, device="cuda").view(-1, 3).t()

    def fill(self, seed, k_scale=1.0, v_scale=1.0):
        """All tokens' keys and values, stored by the definition."""
        g = gen(seed)
        for b, n in enumerate(self.len_list):
            if n == 0:
                continue
            page, slot = self.place(b, torch.arange(n, device="cuda"))
            for values, scale in ((False, k_scale), (True, v_scale)):
                put(self.cache, self.dim, values, page, slot, *quantized(randn((n, self.heads, self.dim), g, scale=scale)))
        return self

    def read64(self, b):
        """Keys and values of sequence b in 64 bits, [tokens][heads][dim]."""
        n = self.len_list[b]
        page, slot = self.place(b, torch.arange(n, device="cuda"))
        return [stood_for(codes[page, :, slot], words[page, :, slot]) for codes, words in cache_parts(self.cache, self.dim)]


def attention64(batch, q, scale):
    """(out, lse, how far out may be off, lse) in 64 bits of rows q; rows of no sequence: zeros, and NaN for lse.

    Off by: a logit's products are exact and added one by one (2 U each, cut off), then scaled (4 U), of sums of magnitudes; the exponent's argument, up
    to its size x, 4 U x, and exp2 itself 2^-21; so a weight's relative error e, twice (its sum's too), with the sum's chain of up to L/64 + 64 additions.
    A weight times the value's scale is rounded to F16's 11 bits, off by half a step, torch.finfo(torch.float16).eps / 2 = 2^-11, or by 2^-32 of the largest scale (half a step of
    F16's subnormals, 2^-25, after the product with 2^7), times codes up to 15.  O's additions like the logits', 2 U each."""
    T, Hq, D = q.shape
    G = Hq // batch.heads
    out, lse = torch.zeros(T, Hq, D, dtype=torch.float64, device="cuda"), torch.full((T, Hq), math.nan, dtype=torch.float64, device="cuda")
    off, lse_off = torch.zeros_like(out), torch.zeros_like(lse)
    scale = torch.tensor(scale, dtype=torch.float32).double().item()
    for b, (length, n) in enumerate(zip(batch.len_list, batch.new_list)):
        r0 = batch.gap + sum(batch.new_list[:b])
        if n == 0:
            continue
        lse[r0:r0 + n] = -math.inf
        seen = torch.arange(length - n, length, device="cuda")
        if length == 0:
            continue
        K, V = batch.read64(b)
        words = cache_parts(batch.cache, D)[1][1]
        page, slot = batch.place(b, torch.arange(length, device="cuda"))
        top = torch.nan_to_num((words[page, :, slot] & ~15).view(torch.float32).double(), 0.0, 0.0, 0.0).amax(0)      # [heads]
        Q = q[r0:r0 + n].double().unflatten(1, (batch.heads, G))
        S = torch.einsum("nhgd,lhd->nhgl", Q, K) * scale
        size = torch.einsum("nhgd,lhd->nhgl", Q.abs(), K.abs()) * abs(scale)
        hidden = torch.arange(length, device="cuda") > seen[:, None]
        S = S.masked_fill(hidden[:, None, None], -math.inf)
        has = seen >= 0
        x = torch.logsumexp(S, -1)
        w = torch.exp(S - torch.where(has[:, None, None], x, 0.0)[..., None])
        o = torch.einsum("nhgl,lhd->nhgd", w, torch.where(hidden.all(0)[:, None, None], 0.0, V))
        sz = torch.einsum("nhgl,lhd->nhgd", w, torch.where(hidden.all(0)[:, None, None], 0.0, V).abs())
        es = torch.where(hidden[:, None, None], 0.0, size).amax(-1) * (2 * D + 4) * U
        reach = torch.where(w > 1e-12, (x[..., None] - S) * 1.5, 0.0).amax(-1) + 10
        e = 2 * (es + 4 * U * reach + 2.0 ** -21) + (length / 64 + 64) * 2 * U
        rows = slice(r0, r0 + n)
        lse[rows] = torch.where(has[:, None, None], x, -math.inf).flatten(1, 2)
        lse_off[rows] = (e + 4 * U * x.abs().nan_to_num(0, 0, 0)).flatten(1, 2)
        out[rows] = torch.where(has[:, None, None, None], o, 0.0).flatten(1, 2)
        step = 2.0 ** -32 * 2 * 15 * top[None, :, None] * length
        off[rows] = (sz * (e[..., None] + 2.0 ** -11 + (length / 16 + 64) * 2 * U) + step[..., None]).flatten(1, 2)
    t = q.dtype
    off += half_step(t) * (out.abs() + off) + least(t)
    return out, lse, off, lse_off
