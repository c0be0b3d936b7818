"""Timed cases of the operators of a language model's low-bit block.

A case is one pass of

  norm       root-mean-square norm of rows, with the residual's addition
  normq      the same with an output in 8 bits (e4m3) and a scale for each group of a row
  normbwd    its backward pass: gradients of the input (and with it of the residual) and of the weight
  fake4      a weight matrix quantised to 4 bits with a scale for each group, and dequantised: what a
             training step that is aware of the quantisation computes with
  w4         rows of tokens times a matrix of 4-bit weights
  block      norm with an 8-bit output (int8, one scale for each row), then the product that reads it

`run` computes it plainly where `own` is false, and through the library's calls where it is true.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-5


def _X():
    import paper_1603_05279_b200 as X
    return X


# ---- the cases ------------------------------------------------------------------------------
def listed():
    return [
        # one token between two layers while an answer is written: latency alone
        {"name": "norm_1x2048_bf16", "kind": "norm", "T": 1, "D": 2048, "type": "bf16", "residual": True},
        # a long prompt, or a training batch, between two layers
        {"name": "norm_8192x4096_bf16", "kind": "norm", "T": 8192, "D": 4096, "type": "bf16", "residual": True},
        # a small model in full precision, rows of odd number and size
        {"name": "norm_333x1001_f32", "kind": "norm", "T": 333, "D": 1001, "type": "f32", "residual": False},
        # a prompt on its way into a product of 8-bit operands
        {"name": "normq_2048x4096_e4m3", "kind": "normq", "T": 2048, "D": 4096, "type": "bf16", "residual": True,
         "group": 128},
        # training: the gradient through the norm, and past it along the residual
        {"name": "normbwd_4096x4096_bf16", "kind": "normbwd", "T": 4096, "D": 4096, "type": "bf16", "residual": True},
        # the same for few rows of odd size in full precision, as in fine-tuning of a small model
        {"name": "normbwd_100x1001_f32", "kind": "normbwd", "T": 100, "D": 1001, "type": "f32", "residual": False},
        # training that is aware of the quantisation: a square projection
        {"name": "fake4_4096x4096_bf16", "kind": "fake4", "N": 4096, "K": 4096, "type": "bf16", "group": 128,
         "zeros": False},
        # a classifier of 1000 classes from full-precision weights, small groups with zero points
        {"name": "fake4_1000x4096_f32", "kind": "fake4", "N": 1000, "K": 4096, "type": "f32", "group": 32,
         "zeros": True},
        # one token through the widest fully connected layer of AlexNet
        {"name": "w4_1x4096x9216_bf16", "kind": "w4", "T": 1, "N": 4096, "K": 9216, "type": "bf16", "group": 128,
         "zeros": False},
        # 16 answers written side by side through a wide layer, weights from a checkpoint with zero points
        {"name": "w4_16x16384x4096_f16", "kind": "w4", "T": 16, "N": 16384, "K": 4096, "type": "f16", "group": 64,
         "zeros": True},
        # a short prompt through norm and projection with 8-bit rows
        {"name": "block_100x4096x4096", "kind": "block", "T": 100, "N": 4096, "K": 4096, "type": "bf16", "group": 128,
         "zeros": False},
        # a long prompt through a wide layer: tensor-core work
        {"name": "w4_2048x8192x8192_bf16", "kind": "w4", "T": 2048, "N": 8192, "K": 8192, "type": "bf16", "group": 128,
         "zeros": False},
    ]


_MAX_VALUES = 33e6                 # rows x columns of a norm, the listed prompt's
_MAX_WEIGHTS = 67e6                # of a matrix, the listed wide layer's
_MAX_MACS = 137e9                  # of a product, the listed prompt's


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.35 else max(32, n // 64 * 64)      # most models' are round


def draw(rng):
    kind = rng.choice(["norm", "norm", "normq", "normbwd", "fake4", "w4", "w4", "w4", "block"])
    while True:
        c = {"kind": kind, "type": rng.choice(["bf16", "bf16", "f16", "f32"])}
        if kind.startswith("norm"):
            c["T"], c["D"] = _log_int(rng, 1, 8192), _size(rng, 64, 16384)
            c["residual"] = rng.random() < 0.6
            if kind == "normq":
                c["group"] = rng.choice([32, 64, 128, 128])
                c["D"] = max(1, c["D"] // c["group"]) * c["group"]
            if c["T"] * c["D"] <= _MAX_VALUES * (0.5 if c["type"] == "f32" else 1.0):
                return c
            continue
        c["N"], c["K"] = _size(rng, 64, 16384), _size(rng, 64, 16384)
        c["group"], c["zeros"] = rng.choice([32, 64, 128, 128]), rng.random() < 0.4
        if kind != "fake4":
            c["T"] = rng.choice([1, 1, 2, 5, 8, _log_int(rng, 1, 64), _log_int(rng, 1, 4096)])
            c["type"] = "bf16" if c["type"] == "f32" else c["type"]
        if c["N"] * c["K"] <= _MAX_WEIGHTS * (0.5 if kind == "fake4" else 1.0) and \
                c["N"] * c["K"] * c.get("T", 1) <= _MAX_MACS:
            return c


# ---- inputs ---------------------------------------------------------------------------------
def _rows(T, D, gen):
    """Hidden states: normal values, a few columns far larger than the others."""
    x = torch.randn(T, D, generator=gen, device="cuda")
    loud = torch.rand(D, generator=gen, device="cuda") < 0.004
    return x * torch.where(loud, 12.0, 1.0)


def _groups(w, group):
    """[N][K] -> [N][G][group], the last group filled with zeros."""
    N, K = w.shape
    G = -(-K // group)
    if G * group != K:
        w = torch.cat([w, w.new_zeros(N, G * group - K)], 1)
    return w.view(N, G, group)


def _quantize4(w, group, zeros):
    """codes uint8 [N][K], scales fp32 [G][N], zero points uint8 [G][N] or None, of real weights.  Quotients are
    rounded from 64 bits: with weights of few bits many lie next to a border between two codes."""
    g = _groups(w.double(), group)
    if zeros:
        lo, hi = g.amin(2).clamp(max=0), g.amax(2).clamp(min=0)
        s = ((hi - lo) / 15).float()
        z = torch.where(s > 0, torch.round(-lo / s.double()), 8.0).clamp(0, 15)
    else:
        s = (g.abs().amax(2) / 7).float()
        z = torch.full_like(s, 8.0, dtype=torch.float64)
    q = torch.where(s[:, :, None] > 0, torch.round(g / s.double()[:, :, None]), 0.0) + z[:, :, None]
    q = q.clamp(0, 15).to(torch.uint8).view(w.shape[0], -1)[:, :w.shape[1]].contiguous()
    return q, s.t().contiguous(), z.to(torch.uint8).t().contiguous() if zeros else None


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 17)
    c, t = case, _TYPES[case["type"]]
    s = {"case": c}
    if c["kind"] in ("norm", "normq", "normbwd", "block"):
        D = c["K"] if c["kind"] == "block" else c["D"]
        s["x"] = _rows(c["T"], D, gen).to(t)
        s["weight"] = (1 + 0.1 * torch.randn(D, generator=gen, device="cuda")).to(t)
        residual = c.get("residual", True)
        s["residual"] = _rows(c["T"], D, gen).to(t) if residual else None
        if c["kind"] == "normbwd":          # what the forward pass kept, and the gradients that arrive
            h = s["x"].float()
            s["rstd"] = torch.rsqrt(h.square().mean(1) + _EPS)
            s["dy"] = (1e-2 * torch.randn(c["T"], D, generator=gen, device="cuda")).to(t)
            s["dsum"] = (1e-2 * torch.randn(c["T"], D, generator=gen, device="cuda")).to(t) if residual else None
            del s["residual"]
    if c["kind"] in ("fake4", "w4", "block"):
        w = 0.02 * torch.randn(c["N"], c["K"], generator=gen, device="cuda")
        if c["kind"] == "fake4":
            s["w"] = w.to(t)
        else:
            s["codes"], s["scales"], s["zeros"] = _quantize4(w, c["group"], c["zeros"])
            if c["kind"] == "w4":
                s["x"] = _rows(c["T"], c["K"], gen).to(t)
    if own:                                 # the buffers that a program keeps, and the weights laid out once
        X = _X()
        if c["kind"] in ("norm", "normq", "block"):
            s["sum"] = torch.empty_like(s["x"]) if s["residual"] is not None else None
            s["rstd"] = torch.empty(c["T"], dtype=torch.float32, device="cuda")
        if c["kind"] == "norm":
            s["y"] = torch.empty_like(s["x"])
        elif c["kind"] == "normq":
            s["q"], s["q_scales"] = X.alloc_rmsnorm_quant(c["T"], c["D"], c["group"], torch.float8_e4m3fn)
        elif c["kind"] == "normbwd":
            s["dx"] = torch.empty_like(s["x"])
            s["dweight"], s["work"] = X.alloc_rmsnorm_backward(c["T"], c["D"])
        elif c["kind"] == "fake4":
            s["d"] = X.make_w4_desc(c["N"], c["K"], c["group"])
            s["packed"], s["scales"], s["zeros"] = X.alloc_w4(s["d"], zeros=c["zeros"])
            s["out"] = torch.empty_like(s["w"])
        else:
            s["d"] = X.make_w4_desc(c["N"], c["K"], c["group"])
            s["packed"] = X.alloc_w4(s["d"])[0]
            X.xnor_w4_pack(s["codes"], s["d"], s["packed"])
            s["out"] = torch.empty(c["T"], c["N"], dtype=t, device="cuda")
            if c["kind"] == "block":
                s["q"], s["q_scales"] = X.alloc_rmsnorm_quant(c["T"], c["K"], 0, torch.int8)
    return s


# ---- one pass -------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    X, c = _X(), s["case"]
    kind = c["kind"]
    if kind == "norm":
        X.xnor_rmsnorm(s["x"], s["residual"], s["weight"], _EPS, s["sum"], s["y"], s["rstd"])
        return {"y": s["y"], "sum": s["sum"], "rstd": s["rstd"]}
    if kind == "normq":
        X.xnor_rmsnorm_quant(s["x"], s["residual"], s["weight"], _EPS, c["group"], s["sum"], s["q"], s["q_scales"],
                             s["rstd"])
        return {"q": s["q"], "scales": s["q_scales"], "sum": s["sum"]}
    if kind == "normbwd":
        X.xnor_rmsnorm_backward(s["dy"], s["dsum"], s["x"], s["weight"], s["rstd"], s["dx"], s["dweight"], s["work"])
        return {"dx": s["dx"], "dweight": s["dweight"]}
    if kind == "fake4":
        X.xnor_w4_quantize(s["w"], s["d"], s["packed"], s["scales"], s["zeros"])
        X.xnor_w4_dequantize(s["packed"], s["scales"], s["zeros"], s["d"], s["out"])
        return {"w": s["out"], "scales": s["scales"]}
    if kind == "w4":
        X.xnor_w4_matmul(s["x"], None, s["packed"], s["scales"], s["zeros"], s["d"], s["out"])
        return {"y": s["out"]}
    X.xnor_rmsnorm_quant(s["x"], s["residual"], s["weight"], _EPS, 0, s["sum"], s["q"], s["q_scales"], s["rstd"])
    X.xnor_w4_matmul(s["q"], s["q_scales"], s["packed"], s["scales"], s["zeros"], s["d"], s["out"])
    return {"y": s["out"], "sum": s["sum"]}


def _plain_norm(s):
    """sum (rounded to its type), its fp32 values, rstd, and the norm in fp32."""
    x, t = s["x"].float(), s["x"].dtype
    total = None
    if s["residual"] is not None:
        total = (x + s["residual"].float()).to(t)
        x = total.float()
    rstd = 1 / torch.sqrt(x.square().mean(1) + _EPS)
    return total, rstd, x * rstd[:, None] * s["weight"].float()


def _plain_weights(s):
    """fp32 [N][K] that the codes stand for."""
    c = s["case"]
    q = s["codes"].float() - 8 if s["zeros"] is None else \
        s["codes"].float() - s["zeros"].float().t().repeat_interleave(c["group"], 1)[:, :c["K"]]
    return q * s["scales"].t().repeat_interleave(c["group"], 1)[:, :c["K"]]


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "norm":
        total, rstd, y = _plain_norm(s)
        return {"y": y.to(s["x"].dtype), "sum": total, "rstd": rstd}
    if kind == "normq":
        total, _, y = _plain_norm(s)
        g = y.view(c["T"], -1, c["group"])
        scales = g.abs().amax(2) / 448
        q = torch.where(scales[:, :, None] > 0, g / scales[:, :, None], 0.0).clamp(-448, 448)
        return {"q": q.to(torch.float8_e4m3fn).view(c["T"], c["D"]), "scales": scales, "sum": total}
    if kind == "normbwd":
        h, dy, r = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
        u = dy * s["weight"].float()
        dx = r * (u - h * (r * r * (u * h).mean(1, keepdim=True)))
        if s["dsum"] is not None:
            dx = dx + s["dsum"].float()
        return {"dx": dx.to(s["x"].dtype), "dweight": (dy * h * r).sum(0)}
    if kind == "fake4":
        codes, scales, zeros = _quantize4(s["w"], c["group"], c["zeros"])
        w = _plain_weights({"case": c, "codes": codes, "scales": scales, "zeros": zeros})
        return {"w": w.to(s["w"].dtype), "scales": scales}
    if kind == "w4":
        return {"y": (s["x"].float() @ _plain_weights(s).t()).to(s["x"].dtype)}
    total, _, y = _plain_norm(s)
    scale = y.abs().amax(1, keepdim=True) / 127
    q = torch.where(scale > 0, torch.round(y / scale), 0.0).clamp(-127, 127)
    return {"y": ((q @ _plain_weights(s).t()) * scale).to(s["x"].dtype), "sum": total}


# ---- what a pass cannot do without ----------------------------------------------------------
def work(case):
    c = case
    e = 4 if c["type"] == "f32" else 2
    if c["kind"].startswith("norm"):
        n, r = c["T"] * c["D"], c["residual"]
        if c["kind"] == "norm":
            return {"bytes": e * n * (4 if r else 2) + e * c["D"] + 4 * c["T"], "flops": 4 * n}
        if c["kind"] == "normq":
            return {"bytes": e * n * (3 if r else 1) + n + 4 * n // c["group"] + e * c["D"], "flops": 6 * n}
        return {"bytes": e * n * (4 if r else 3) + (e + 4) * c["D"] + 4 * c["T"], "flops": 10 * n}
    N, K, G = c["N"], c["K"], -(-c["K"] // c["group"])
    w4 = N * K // 2 + N * G * (5 if c["zeros"] else 4)
    if c["kind"] == "fake4":
        return {"bytes": 2 * e * N * K + 4 * N * G, "flops": 4 * N * K}
    if c["kind"] == "w4":
        return {"bytes": w4 + e * c["T"] * (N + K), "flops": 2 * c["T"] * N * K}
    return {"bytes": w4 + e * c["T"] * (N + 3 * K), "flops": 2 * c["T"] * N * K}


# ---- the definitions in 64 bits -------------------------------------------------------------
def exact(case, seed):
    global own
    mine, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    c, f = case, torch.float64
    out = {}
    if c["kind"] in ("norm", "normq", "block"):
        h = s["x"].to(f)
        out["sum"] = None
        if s["residual"] is not None:
            out["sum"] = h + s["residual"].to(f)
            h = out["sum"].to(s["x"].dtype).to(f)           # the norm is of the stored sum
        root = torch.sqrt((h * h).sum(1) / h.shape[1] + _EPS)
        y = h / root.unsqueeze(1) * s["weight"].to(f)
        if c["kind"] == "norm":
            return {"y": y, "sum": out["sum"], "rstd": 1 / root}
    if c["kind"] == "normq":
        G = c["D"] // c["group"]
        top = y.reshape(c["T"], G, c["group"]).abs().max(2).values
        scaled = y / torch.repeat_interleave(top / 448.0, c["group"], 1)
        return {"q": scaled.to(torch.float8_e4m3fn).to(f), "scales": top / 448.0, "sum": out["sum"]}
    if c["kind"] == "normbwd":
        h, dy, w = s["x"].to(f), s["dy"].to(f), s["weight"].to(f)
        r = s["rstd"].to(f)
        dot = torch.einsum("td,td,d->t", h, dy, w) * r ** 3 / h.shape[1]
        dx = torch.einsum("td,d,t->td", dy, w, r) - torch.einsum("td,t->td", h, dot)
        return {"dx": dx if s["dsum"] is None else dx + s["dsum"].to(f), "dweight": torch.einsum("td,td,t->d", dy, h, r)}
    if c["kind"] == "fake4":
        w = s["w"].to(f)
        parts, scales = [], []
        for k in range(0, c["K"], c["group"]):
            p = w[:, k:k + c["group"]]
            if c["zeros"]:
                lo = torch.minimum(p.min(1).values, torch.zeros((), dtype=f, device="cuda"))
                hi = torch.maximum(p.max(1).values, torch.zeros((), dtype=f, device="cuda"))
                step = ((hi - lo) / 15.0).float().to(f)     # scales are held in 32 bits
                z = torch.round(-lo / step)
                code = torch.clamp(torch.round(p / step[:, None]) + z[:, None], 0, 15) - z[:, None]
            else:
                step = (p.abs().max(1).values / 7.0).float().to(f)
                code = torch.round(p / step[:, None])
            parts.append(code * step[:, None])
            scales.append(step)
        return {"w": torch.cat(parts, 1), "scales": torch.stack(scales)}
    n = torch.arange(c["K"], device="cuda") // c["group"]
    q = s["codes"].to(f) - (8.0 if s["zeros"] is None else s["zeros"].to(f)[n].t())
    W = q * s["scales"].to(f)[n].t()
    if c["kind"] == "w4":
        return {"y": torch.einsum("tk,nk->tn", s["x"].to(f), W)}
    step = y.abs().max(1).values / 127.0
    return {"y": torch.einsum("tk,nk->tn", torch.round(y / step[:, None]) * step[:, None], W), "sum": out["sum"]}
