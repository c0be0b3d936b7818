"""Timed cases of the operators around a language model's attention over a cache in 4 bits.

A case is one pass of

  heads      root-mean-square norm of the queries' and keys' heads, with the position rotation
  headsbwd   its backward pass: gradients of queries, keys and both weights
  append     new tokens: queries rotated, keys rotated and with the values quantised to 4 bits and put into the pages
             of their sequences; then read back, so that what was stored comes out as the values it stands for
  attend     attention of the new tokens' queries over the cache, causal, with grouped heads
  step       append, then attention: what a layer does with one token of each sequence

`run` computes it plainly where `own` is false, and through the library's calls where it is true.

The cache is bytes [pages][kv_heads][page / 16][16 (dim + 8)]: for 16 tokens the keys' codes (dim / 2 bytes a token), the
values', then a word for each token's keys and one for its values: the scale in fp32, whose last four bits are the zero
point instead.  Column 2 i + h of eight is in bits 4 i + 16 h and up of their word.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-6
_BASE = 10000.0


def _X():
    import paper_1603_05279_b200 as X
    return X


# ---- the cases ------------------------------------------------------------------------------
def listed():
    return [
        # one token between projection and attention while an answer is written: latency alone
        {"name": "heads_1x32x128_bf16", "kind": "heads", "T": 1, "Hq": 32, "Hk": 8, "D": 128, "rot": 128, "pairs": False,
         "norm": True, "type": "bf16"},
        # a long prompt, or a training batch
        {"name": "heads_8192x32x128_bf16", "kind": "heads", "T": 8192, "Hq": 32, "Hk": 8, "D": 128, "rot": 128,
         "pairs": False, "norm": True, "type": "bf16"},
        # a small model in full precision: heads of no power of two, half of each rotated, neighbours paired
        {"name": "heads_333x12x80_f32", "kind": "heads", "T": 333, "Hq": 12, "Hk": 12, "D": 80, "rot": 40, "pairs": True,
         "norm": True, "type": "f32"},
        # training: the gradient on its way from attention to the projections
        {"name": "headsbwd_4096x32x128_bf16", "kind": "headsbwd", "T": 4096, "Hq": 32, "Hk": 8, "D": 128, "rot": 128,
         "pairs": False, "norm": True, "type": "bf16"},
        # the same for a short sequence of a small model
        {"name": "headsbwd_100x12x80_f32", "kind": "headsbwd", "T": 100, "Hq": 12, "Hk": 4, "D": 80, "rot": 80,
         "pairs": False, "norm": True, "type": "f32"},
        # 64 answers written side by side: one token each
        {"name": "append_64x8x128_bf16", "kind": "append", "B": 64, "least": 1, "most": 4096, "new": 1, "Hq": 32, "Hk": 8,
         "D": 128, "page": 16, "rot": 128, "pairs": False, "norm": True, "type": "bf16"},
        # several prompts of different lengths at once
        {"name": "append_prompts_8x64_f16", "kind": "append", "B": 16, "least": 100, "most": 1000, "new": 0, "Hq": 32,
         "Hk": 8, "D": 64, "page": 64, "rot": 32, "pairs": False, "norm": False, "type": "f16"},
        # one answer after a middling context: latency, and few rows for the whole GPU
        {"name": "attend_1x5000_bf16", "kind": "attend", "B": 1, "least": 5000, "most": 5000, "new": 1, "Hq": 32, "Hk": 8,
         "D": 128, "page": 16, "type": "bf16"},
        # many answers side by side, contexts from short to long: the cache is read once
        {"name": "attend_64x8192_bf16", "kind": "attend", "B": 64, "least": 300, "most": 8192, "new": 1, "Hq": 32, "Hk": 8,
         "D": 128, "page": 64, "type": "bf16"},
        # five guessed tokens of each answer checked at once, another head layout
        {"name": "attend_16x2000x5_f16", "kind": "attend", "B": 16, "least": 500, "most": 2000, "new": 5, "Hq": 16,
         "Hk": 4, "D": 64, "page": 32, "type": "f16"},
        # whole prompts: tensor-core work
        {"name": "attend_prompts_4096_bf16", "kind": "attend", "B": 2, "least": 4000, "most": 4096, "new": 0, "Hq": 32,
         "Hk": 8, "D": 128, "page": 64, "type": "bf16"},
        # a layer's work between two projections for 16 answers
        {"name": "step_16x1500_bf16", "kind": "step", "B": 16, "least": 100, "most": 1500, "new": 1, "Hq": 32, "Hk": 8,
         "D": 128, "page": 16, "rot": 128, "pairs": False, "norm": True, "type": "bf16"},
    ]


_MAX_HEADS = 8192 * 40 * 128       # values of a heads case, the listed prompt's
_MAX_NEW = 9000 * 48 * 64          # values of an append, the listed prompts'
_MAX_CACHE = 64 * 8192 * 8 * 128   # padded keys of an attention, the listed batch's
_MAX_SCORES = 2 * 32 * 4096 * 4096


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["heads", "heads", "headsbwd", "append", "append", "attend", "attend", "attend", "step"])
    while True:
        c = {"kind": kind}
        c["Hk"] = rng.choice([1, 2, 4, 8, 8, 5])
        c["Hq"] = c["Hk"] * rng.choice([1, 2, 4, 4, 7, 8])
        if kind.startswith("heads"):
            c["T"], c["D"] = _log_int(rng, 1, 8192), rng.choice([32, 64, 80, 96, 128, 128, 128, 256])
            c["rot"] = rng.choice([c["D"], c["D"], c["D"] // 2])
            c["pairs"], c["norm"] = rng.random() < 0.3, kind == "headsbwd" or rng.random() < 0.8
            c["type"] = rng.choice(["bf16", "bf16", "f16", "f32"])
            if c["T"] * (c["Hq"] + c["Hk"]) * c["D"] <= _MAX_HEADS * (0.5 if c["type"] == "f32" or kind == "headsbwd" else 1.0):
                return c
            continue
        c["D"], c["page"] = rng.choice([64, 128, 128]), rng.choice([16, 16, 32, 64, 128])
        c["type"] = rng.choice(["bf16", "bf16", "f16"])
        if kind != "attend":
            c["rot"] = rng.choice([c["D"], c["D"], c["D"] // 2])
            c["pairs"], c["norm"] = rng.random() < 0.3, rng.random() < 0.7
        c["B"] = _log_int(rng, 1, 128)
        c["most"] = _log_int(rng, 1, 30000)
        c["least"] = max(1, int(c["most"] * rng.uniform(0.05, 1.0)))
        c["new"] = rng.choice([1, 1, 0, 2, 5, _log_int(rng, 1, 1000)]) if kind != "step" else rng.choice([1, 1, 2, 3])
        longest = min(c["new"] or c["most"], c["most"])
        if kind != "attend" and c["B"] * longest * (c["Hq"] + 2 * c["Hk"]) * c["D"] > _MAX_NEW:
            continue
        if c["B"] * c["most"] * c["Hk"] * c["D"] <= _MAX_CACHE * (0.25 if kind == "append" else 1.0) and \
                (kind == "append" or c["B"] * c["Hq"] * longest * c["most"] <= _MAX_SCORES):
            return c


def _lengths(c):
    """(tokens of each sequence after the new ones, how many of them are new): the case's own."""
    rng = random.Random("%d %d %d" % (c["B"], c["least"], c["most"]))
    lens = [rng.randint(c["least"], c["most"]) for _ in range(c["B"])]
    lens[-1] = c["most"]
    return lens, [min(n, c["new"] or n) for n in lens]


# ---- inputs ---------------------------------------------------------------------------------
def _heads(rows, heads, dim, gen, loud=0.0):
    """Rows of heads: normal values, a few columns of each head larger than the others."""
    x = torch.randn(rows, heads, dim, generator=gen, device="cuda")
    if loud:
        x *= torch.where(torch.rand(heads, dim, generator=gen, device="cuda") < loud, 5.0, 1.0)
    return x


def _rope(positions, rot):
    """cos and sin of position * base^(-2 i / rot), rounded once."""
    f = _BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _views(cache, c):
    """Codes [pages][heads][blocks][16][dim / 2] and words [..][16] of keys and of values, inside the cache."""
    D, lead = c["D"], cache.shape[:3]
    word = cache[..., 16 * D:].view(torch.int32)
    return (cache[..., :8 * D].unflatten(3, (16, D // 2)), cache[..., 8 * D:16 * D].unflatten(3, (16, D // 2)),
            word[..., :16], word[..., 16:])


def _quantize(x):
    """Codes in bytes [..][dim / 2] and words of rows in fp32.  Quotients are rounded from 64 bits: with values of few
    bits many lie next to a border between two codes."""
    x = x.float().double()
    lo, hi = x.amin(-1).clamp(max=0), x.amax(-1).clamp(min=0)
    s = ((hi - lo) / 15).float().view(torch.int32) & -16
    step = s.view(torch.float32).double()
    z = torch.where(step > 0, torch.round(-lo / step), 8.0).clamp(0, 15)
    q = torch.where(step[..., None] > 0, torch.round(x / step[..., None]), 0.0) + z[..., None]
    q = q.clamp(0, 15).to(torch.uint8).unflatten(-1, (-1, 2, 2, 2)).movedim(-1, -3)       # [..][8s][h][r][n]
    return (q[..., 0] | q[..., 1] << 4).flatten(-3), s | z.to(torch.int32)


def _values(codes, words):
    """fp32 rows that bytes [..][dim / 2] and words stand for."""
    q = torch.stack([codes & 15, codes >> 4], -1).unflatten(-2, (-1, 2, 2))                # [..][8s][h][r][n]
    q = q.movedim(-3, -1).flatten(-4).float()
    return (q - (words & 15).float()[..., None]) * (words & -16).view(torch.float32)[..., None]


def _place(c, table, seq, pos):
    """Page, block in it and slot in that of places of sequences."""
    return table[seq, pos // c["page"]].long(), pos % c["page"] // 16, pos % 16


def _store(cache, c, at, k, v):
    page, block, slot = at
    kc, vc, kw, vw = _views(cache, c)
    for x, codes, words in ((k, kc, kw), (v, vc, vw)):
        q, w = _quantize(x)
        codes[page, :, block, slot] = q
        words[page, :, block, slot] = w


def _fetch(cache, c, at):
    page, block, slot = at
    kc, vc, kw, vw = _views(cache, c)
    return (_values(kc[page, :, block, slot], kw[page, :, block, slot]),
            _values(vc[page, :, block, slot], vw[page, :, block, slot]))


def _rows(s):
    """Sequence and place in it of each new token."""
    row = torch.arange(s["T"], device="cuda")
    seq = torch.searchsorted(s["starts"][1:].contiguous(), row.int(), right=True)
    return seq, (s["lens"][seq] - (s["starts"][seq + 1] - row)).long()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 29)
    c, t = case, _TYPES[case["type"]]
    s = {"case": c}
    if not c["kind"].startswith("heads"):
        lens, new = _lengths(c)
        s["T"], s["longest"], s["most_new"] = sum(new), max(lens), max(new)
        cols = -(-s["longest"] // c["page"])
        pages = sum(-(-n // c["page"]) for n in lens) + 3
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["starts"] = torch.tensor([sum(new[:i]) for i in range(c["B"] + 1)], dtype=torch.int32, device="cuda")
        s["table"] = torch.zeros(c["B"], cols, dtype=torch.int32, device="cuda")
        free = torch.randperm(pages, generator=gen, device="cuda").int()
        used = (torch.arange(cols, device="cuda") * c["page"] < s["lens"][:, None]).nonzero()
        s["table"][used[:, 0], used[:, 1]] = free[:used.shape[0]]
        # pages hold whatever was there before, and the sequences' tokens
        s["cache"] = torch.randint(0, 256, (pages, c["Hk"], c["page"] // 16, 16 * (c["D"] + 8)), generator=gen,
                                   dtype=torch.uint8, device="cuda")
        if c["kind"] != "append":
            at = (torch.arange(s["longest"], device="cuda") < s["lens"][:, None]).nonzero()
            for part in at.split(1 << 17):
                _store(s["cache"], c, _place(c, s["table"], part[:, 0], part[:, 1]),
                       _heads(part.shape[0], c["Hk"], c["D"], gen, 0.02), _heads(part.shape[0], c["Hk"], c["D"], gen))
    T = c.get("T") or s["T"]
    s["q"] = _heads(T, c["Hq"], c["D"], gen).to(t)
    if c["kind"] != "attend":
        s["k"] = _heads(T, c["Hk"], c["D"], gen, 0.02).to(t)
        s["v"] = _heads(T, c["Hk"], c["D"], gen).to(t)
        s["q_weight"] = s["k_weight"] = None
        if c["norm"]:
            s["q_weight"] = (1 + 0.1 * torch.randn(c["D"], generator=gen, device="cuda")).to(t)
            s["k_weight"] = (1 + 0.1 * torch.randn(c["D"], generator=gen, device="cuda")).to(t)
        s["eps"] = _EPS if c["norm"] else None
        s["rope"] = _rope(s["longest"] if "longest" in s else T + 1000, c["rot"])
    if c["kind"].startswith("heads"):
        s["positions"] = torch.randint(0, T + 1000, (T,), generator=gen, dtype=torch.int32, device="cuda")
        s["dq_out"] = 1e-2 * torch.randn(T, c["Hq"], c["D"], generator=gen, device="cuda")
        s["dk_out"] = 1e-2 * torch.randn(T, c["Hk"], c["D"], generator=gen, device="cuda")
        s["dq_out"], s["dk_out"] = s["dq_out"].to(t), s["dk_out"].to(t)
    s["scale"] = c["D"] ** -0.5
    if own:                                 # the buffers that a program keeps
        X = _X()
        s["q_out"] = torch.empty_like(s["q"])
        if c["kind"].startswith("heads"):
            s["k_out"] = torch.empty_like(s["k"])
            if c["kind"] == "headsbwd":
                s["dq_weight"], s["dk_weight"], s["work"] = X.alloc_qk_backward(T, c["Hq"], c["Hk"], c["D"])
        else:
            s["d"] = X.make_kv4_desc(s["cache"].shape[0], c["page"], c["Hk"], c["D"])
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(T, c["Hq"], dtype=torch.float32, device="cuda")
            if c["kind"] == "append":
                s["k_read"], s["v_read"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
            else:
                s["work"] = X.alloc_kv4_work(s["d"], T, c["Hq"], c["B"])
    return s


# ---- one pass -------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    X, c = _X(), s["case"]
    kind = c["kind"]
    if kind == "heads":
        X.xnor_qk_norm_rope(s["q"], s["k"], s["q_weight"], s["k_weight"], s["eps"], s["positions"], s["rope"], c["pairs"],
                            s["q_out"], s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if kind == "headsbwd":
        X.xnor_qk_norm_rope_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["eps"],
                                     s["positions"], s["rope"], c["pairs"], s["q_out"], s["k_out"], s["dq_weight"],
                                     s["dk_weight"], s["work"])
        return {"dq": s["q_out"], "dk": s["k_out"], "dq_weight": s["dq_weight"], "dk_weight": s["dk_weight"]}
    if kind != "attend":
        X.xnor_kv4_append(s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["eps"], s["rope"], c["pairs"],
                          s["starts"], s["lens"], s["table"], s["d"], s["q_out"], s["cache"])
    if kind == "append":
        X.xnor_kv4_read(s["cache"], s["starts"], s["lens"], s["table"], s["d"], s["k_read"], s["v_read"])
        return {"q": s["q_out"], "k": s["k_read"], "v": s["v_read"]}
    X.xnor_kv4_attention(s["q"] if kind == "attend" else s["q_out"], s["cache"], s["starts"], s["lens"], s["table"], s["d"],
                         s["scale"], s["most_new"], s["out"], s["lse"], s["work"])
    return {"out": s["out"], "lse": s["lse"]}


def _rotate(x, cos, sin, rot, pairs):
    """x [rows][heads][dim], cos and sin [rows][1][rot / 2]."""
    if pairs:
        a, b = x[..., :rot:2], x[..., 1:rot:2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([r, x[..., rot:]], -1)


def _angles(s, positions, t):
    cos, sin = s["rope"][positions.long()].to(t).chunk(2, -1)
    return cos[:, None], sin[:, None]


def _norm_rope(s, x, weight, positions, t):
    c, x = s["case"], x.to(t)
    if c["norm"]:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + _EPS) * weight.to(t)
    return _rotate(x, *_angles(s, positions, t), c["rot"], c["pairs"])


def _norm_rope_backward(s, dy, x, weight):
    c, x, w = s["case"], x.float(), weight.float()
    cos, sin = _angles(s, s["positions"], torch.float32)
    g = _rotate(dy.float(), cos, -sin, c["rot"], c["pairs"])
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + _EPS)
    u = g * w
    return (r * (u - x * (r * r * (u * x).mean(-1, keepdim=True)))).to(dy.dtype), (g * x * r).sum((0, 1))


def _append(s):
    """Rotated queries; the cache has the new tokens.  Keys in 64 bits: their codes lie next to borders."""
    c = s["case"]
    seq, pos = _rows(s)
    q = _norm_rope(s, s["q"], s["q_weight"], pos, torch.float32).to(s["q"].dtype)
    _store(s["cache"], c, _place(c, s["table"], seq, pos), _norm_rope(s, s["k"], s["k_weight"], pos, torch.float64), s["v"])
    return q


def _attend(s, q):
    c, B, L, n = s["case"], s["case"]["B"], s["longest"], s["most_new"]
    seq, pos = _rows(s)
    at = torch.arange(L, device="cuda")
    k, v = _fetch(s["cache"], c, _place(c, s["table"], torch.arange(B, device="cuda")[:, None], at[None]))
    there = (at < s["lens"][:, None])[:, :, None, None]
    k, v = torch.where(there, k, 0.0), torch.where(there, v, 0.0)        # [B][L][Hk][D]
    row = torch.arange(s["T"], device="cuda") - s["starts"][seq]
    Q = torch.zeros(B, n, c["Hq"], c["D"], device="cuda")
    Q[seq, row] = q.float()
    limit = torch.full((B, n), -1, device="cuda")
    limit[seq, row] = pos
    Q = Q.unflatten(2, (c["Hk"], -1)).movedim(1, 3).flatten(2, 3)        # [B][Hk][group * n][D]
    S = (Q @ k.permute(0, 2, 3, 1)).unflatten(2, (-1, n)) * s["scale"]   # [B][Hk][group][n][L]
    S = S.masked_fill_(at > limit[:, None, None, :, None], -math.inf)
    top = S.amax(-1, keepdim=True).clamp(min=-3e38)
    S = S.sub_(top).exp_()
    total = S.sum(-1, keepdim=True)
    out = (S.flatten(2, 3) @ v.permute(0, 2, 1, 3)).unflatten(2, (-1, n)) / total
    out, lse = out.movedim(3, 1).flatten(2, 3), (total.log() + top).squeeze(-1).movedim(3, 1).flatten(2, 3)
    return {"out": out[seq, row].to(q.dtype), "lse": lse[seq, row]}


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "heads":
        return {n: _norm_rope(s, s[n], s[n + "_weight"], s["positions"], torch.float32).to(s[n].dtype) for n in ("q", "k")}
    if c["kind"] == "headsbwd":
        dq, dqw = _norm_rope_backward(s, s["dq_out"], s["q"], s["q_weight"])
        dk, dkw = _norm_rope_backward(s, s["dk_out"], s["k"], s["k_weight"])
        return {"dq": dq, "dk": dk, "dq_weight": dqw, "dk_weight": dkw}
    if c["kind"] == "attend":
        return _attend(s, s["q"])
    q = _append(s)
    if c["kind"] == "step":
        return _attend(s, q)
    k, v = _fetch(s["cache"], c, _place(c, s["table"], *_rows(s)))
    return {"q": q, "k": k.to(q.dtype), "v": v.to(q.dtype)}


# ---- what a pass cannot do without ----------------------------------------------------------
def work(case):
    c = case
    e, D = 4 if c["type"] == "f32" else 2, c["D"]
    if c["kind"].startswith("heads"):
        n = c["T"] * (c["Hq"] + c["Hk"]) * D
        rope = 4 * c["T"] * (1 + c["rot"])
        if c["kind"] == "heads":
            return {"bytes": 2 * e * n + rope, "flops": 7 * n}
        return {"bytes": 3 * e * n + rope + 8 * D, "flops": 14 * n}
    lens, new = _lengths(c)
    T, token = sum(new), c["Hk"] * (D + 8)                        # token: its bytes in the cache
    got = {"bytes": 0, "flops": 0}
    if c["kind"] != "attend":
        got["bytes"] += e * T * D * 2 * (c["Hq"] + c["Hk"]) + T * token + 4 * T * c["rot"]
        got["flops"] += T * D * (7 * (c["Hq"] + c["Hk"]) + 12 * c["Hk"])
    if c["kind"] == "append":
        got["bytes"] += T * token + 2 * e * T * c["Hk"] * D
        got["flops"] += 4 * T * c["Hk"] * D
        return got
    seen = sum(n * (length - n) + n * (n + 1) // 2 for length, n in zip(lens, new))
    got["bytes"] += sum(lens) * token + T * c["Hq"] * (2 * e * D + 4)
    got["flops"] += 4 * seen * c["Hq"] * D
    return got


# ---- the definitions in 64 bits -------------------------------------------------------------
def _exact_heads(c, x, weight, eps, table, positions):
    """Complex numbers: a pair is one, a rotation a product."""
    y = x.to(torch.float64)
    if c["norm"]:
        y = torch.einsum("thd,th,d->thd", y, torch.rsqrt((y * y).sum(2) / y.shape[2] + eps), weight.to(torch.float64))
    half = c["rot"] // 2
    turn = torch.complex(*table[positions.long()].to(torch.float64).split(half, 1))[:, None, :]
    part = y[:, :, :c["rot"]]
    z = torch.view_as_complex(part.unflatten(2, (half, 2)).contiguous()) if c["pairs"] else \
        torch.complex(part[:, :, :half].contiguous(), part[:, :, half:].contiguous())
    z = z * turn
    y[:, :, :c["rot"]] = torch.view_as_real(z).flatten(2) if c["pairs"] else torch.cat([z.real, z.imag], 2)
    return y


def _exact_backward(c, dy, x, weight, eps, table, positions):
    half = c["rot"] // 2
    cos, sin = (v[:, None, :] for v in table[positions.long()].to(torch.float64).split(half, 1))
    g, x, w = dy.to(torch.float64), x.to(torch.float64), weight.to(torch.float64)
    first = torch.arange(half, device="cuda") * (2 if c["pairs"] else 1)
    second = first + (1 if c["pairs"] else half)
    a, b = g[:, :, first], g[:, :, second]
    g[:, :, first], g[:, :, second] = a * cos + b * sin, b * cos - a * sin
    r = torch.rsqrt((x * x).sum(2) / x.shape[2] + eps)
    dot = torch.einsum("thd,thd,d->th", g, x, w) * r ** 3 / x.shape[2]
    dx = torch.einsum("thd,d,th->thd", g, w, r) - torch.einsum("thd,th->thd", x, dot)
    return dx, torch.einsum("thd,thd,th->d", g, x, r)


def _exact_codes(x):
    """The values that rows stand for once they are in 4 bits."""
    lo = torch.minimum(x.min(2).values, torch.zeros((), dtype=x.dtype, device="cuda"))
    hi = torch.maximum(x.max(2).values, torch.zeros((), dtype=x.dtype, device="cuda"))
    mantissa, exponent = torch.frexp(((hi - lo) / 15.0).float().to(torch.float64))
    step = torch.ldexp(torch.floor(mantissa * 2.0 ** 20), exponent - 20)       # 20 bits are kept of the scale's 24
    zero = torch.round(-lo / step).clamp(0, 15)
    return (torch.clamp(torch.round(x / step[..., None]) + zero[..., None], 0, 15) - zero[..., None]) * step[..., None]


def _exact_read(c, cache, pages, count):
    """Keys and values of a sequence's first `count` tokens, 64 bits, [heads][count][dim]."""
    raw, D = cache[pages.long()].movedim(1, 0).flatten(1, 2), c["D"]           # [heads][blocks][bytes]
    column = torch.arange(D, device="cuda") % 8
    bit = 4 * (column // 2) + 16 * (column % 2)
    byte = torch.arange(D, device="cuda") // 8 * 4 + bit // 8
    got = []
    for first, word in ((0, 16 * D), (8 * D, 16 * D + 64)):
        rows = raw[:, :, first:first + 8 * D].unflatten(2, (16, D // 2)).flatten(1, 2)[:, :count]
        q = (rows[..., byte].int() >> (bit % 8)) & 15
        p = raw[:, :, word:word + 64].contiguous().view(torch.int32).flatten(1, 2)[:, :count]
        step = (p - (p & 15)).view(torch.float32).to(torch.float64)
        got.append((q - (p & 15)[..., None]).to(torch.float64) * step[..., None])
    return got


def exact(case, seed):
    global own
    mine, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    c, f = case, torch.float64
    if c["kind"] == "heads":
        return {n: _exact_heads(c, s[n], s[n + "_weight"], _EPS, s["rope"], s["positions"]) for n in ("q", "k")}
    if c["kind"] == "headsbwd":
        dq, dqw = _exact_backward(c, s["dq_out"], s["q"], s["q_weight"], _EPS, s["rope"], s["positions"])
        dk, dkw = _exact_backward(c, s["dk_out"], s["k"], s["k_weight"], _EPS, s["rope"], s["positions"])
        return {"dq": dq, "dk": dk, "dq_weight": dqw, "dk_weight": dkw}
    lens, new = _lengths(c)
    q, first, outs, lses = s["q"].to(f), 0, [], []
    if c["kind"] != "attend":
        at = torch.cat([torch.arange(n - m, n, device="cuda") for n, m in zip(lens, new)])
        q = _exact_heads(c, s["q"], s["q_weight"], _EPS, s["rope"], at)
        k = _exact_codes(_exact_heads(c, s["k"], s["k_weight"], _EPS, s["rope"], at).float().to(f))
        v = _exact_codes(s["v"].to(f))
        if c["kind"] == "append":
            return {"q": q, "k": k, "v": v}
        q = q.to(s["q"].dtype).to(f)                              # attention reads them as they were stored
    for b, (length, n) in enumerate(zip(lens, new)):
        K, V = _exact_read(c, s["cache"], s["table"][b, :-(-length // c["page"])], length)
        if c["kind"] == "step":
            K[:, length - n:], V[:, length - n:] = k[first:first + n].movedim(1, 0), v[first:first + n].movedim(1, 0)
        Q = q[first:first + n].unflatten(1, (c["Hk"], -1))
        first += n
        out, lse = [], []
        for h in range(c["Hk"]):                                  # a head at a time: 64 bits of all scores would not fit
            S = torch.einsum("ngd,ld->ngl", Q[:, h], K[h]) * c["D"] ** -0.5
            S += torch.where(torch.arange(length, device="cuda") > torch.arange(length - n, length, device="cuda")[:, None],
                             -math.inf, 0.0)[:, None]
            lse.append(torch.logsumexp(S, 2))
            out.append(torch.einsum("ngl,ld->ngd", torch.softmax(S, 2), V[h]))
        outs.append(torch.cat(out, 1))
        lses.append(torch.cat(lse, 1))
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
