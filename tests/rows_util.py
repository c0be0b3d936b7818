"""Helpers of the tests on rows of tokens: guarded buffers of any type and plain 64-bit definitions."""
import math

import numpy as np
import torch

U = 2.0 ** -24                       # half a step of fp32
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def half_step(t):
    """A rounding to type t is off by at most this, relative to the value."""
    return torch.finfo(t).eps / 2


def least(t):
    """... or by this, where the value is subnormal."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


class Guards:
    """Outputs inside larger allocations of a byte pattern: [rows][cols], rows `pad` elements apart."""

    def __init__(self):
        self.items = []

    def rows(self, rows, cols, dtype, pad=0):
        n = max(0, rows * (cols + pad) - pad)
        e = torch.empty((), dtype=dtype).element_size()
        raw = torch.full((512 + -(-n * e // 16) * 16 + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        t = raw[512:512 + n * e].view(dtype)
        t = t.as_strided((rows, cols), (cols + pad, 1), t.storage_offset())
        self.items.append((raw, n, e, rows, cols, pad))
        return t

    def flat(self, n, dtype):
        return self.rows(1, n, dtype).view(-1)

    def check(self):
        torch.cuda.synchronize()
        for raw, n, e, rows, cols, pad in self.items:
            b = raw.cpu().numpy()
            assert (b[:512] == 0xA5).all() and (b[512 + n * e:] == 0xA5).all(), "write outside the buffer"
            if pad and rows > 1:
                body = np.concatenate([b[512:512 + n * e], np.full(pad * e, 0xA5, np.uint8)])
                assert (body.reshape(rows, (cols + pad) * e)[:, cols * e:] == 0xA5).all(), "write between the rows"


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(shape, g, t=torch.float32, scale=1.0):
    return (scale * torch.randn(shape, generator=g, device="cuda")).to(t)


def strided(t, pad):
    """A copy of t whose rows lie `pad` elements further apart, NaN between them."""
    if not pad:
        return t
    big = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=torch.float32, device="cuda").to(t.dtype) \
        if t.dtype.is_floating_point else torch.full((t.shape[0], t.shape[1] + pad), 77, dtype=t.dtype, device="cuda")
    big[:, :t.shape[1]] = t
    return big[:, :t.shape[1]]


def norm64(h, w, eps=EPS):
    """(rstd, y) of the norm in 64 bits, of stored values h."""
    h = h.double()
    rstd = 1 / torch.sqrt((h * h).mean(1) + eps)
    return rstd, h * rstd[:, None] * (1.0 if w is None else w.double())


def norm_error(D):
    """Relative error of y before its rounding, of fp32 sums and products.

    A row's squares are added by a thread in chains of up to 32, then by a tree of 5 steps and a chain over up to
    32 warps, each addition and product off by U at most: 69 U for the sum; the rounded reciprocal of D, its
    product and the addition of eps: 3 U more.  Half of that for the root, which is within 2 U itself; two products: 2 U."""
    return (72 / 2 + 4) * U


def unpack_codes(packed, N, K):
    """Codes [N][K] of the packed tiles, by the documented layout alone."""
    p = packed.cpu().numpy().view(np.uint32)
    panels, ct = p.shape[:2]
    p = p.reshape(panels, ct, 8, 32, 4).transpose(0, 2, 1, 3, 4).reshape(panels * 8, ct, 32, 4)
    out = np.zeros((panels * 128, ct * 64), np.uint8)
    for place in range(32):
        g = place // 4
        t = (place % 4) ^ (g // 2 % 4)
        for word in range(4):
            row, col = g + 8 * (word // 2), 32 * (word % 2) + 8 * t
            for i in range(8):
                out[row::16, col + i::64] = (p[:, :, place, word] >> np.uint32(4 * (i // 2) + 16 * (i % 2))) & 15
    return out[:N, :K]


def pack_codes(codes):
    """The packed tiles of codes [N][K] (numpy), by the documented layout alone; 8 beyond the matrix."""
    N, K = codes.shape
    panels, ct = -(-N // 128), -(-K // 64)
    full = np.full((panels * 128, ct * 64), 8, np.uint32)
    full[:N, :K] = codes
    p = np.zeros((panels * 8, ct, 32, 4), np.uint32)
    for place in range(32):
        g = place // 4
        t = (place % 4) ^ (g // 2 % 4)
        for word in range(4):
            row, col = g + 8 * (word // 2), 32 * (word % 2) + 8 * t
            for i in range(8):
                p[:, :, place, word] |= full[row::16, col + i::64] << np.uint32(4 * (i // 2) + 16 * (i % 2))
    p = np.ascontiguousarray(p.reshape(panels, 8, ct, 32, 4).transpose(0, 2, 1, 3, 4)).reshape(panels, ct, 256, 4)
    return torch.from_numpy(p.view(np.int32))


def weights64(codes, scales, zeros, group):
    """[N][K] in 64 bits from codes [N][K], scales and zeros [G][N]."""
    K = codes.shape[1]
    z = 8.0 if zeros is None else zeros.double().t().repeat_interleave(group, 1)[:, :K]
    return (codes.double() - z) * scales.double().t().repeat_interleave(group, 1)[:, :K]


def matmul_bound(x, xs, W, K, group, out_type, out64):
    """How far a product may be off: the operands are exact, so additions and the scaling are all that rounds.

    Inside a group every addition of a tensor core may be cut off instead of rounded (2 U each, at most `group`
    of them); the groups are added in a chain (G), then warps and blocks (16), and a scale costs 3 products.
    All relative to the sum of magnitudes; then one rounding of the result."""
    G = math.ceil(K / group)
    mag = (x.double().abs() * xs) @ W.abs().t()
    return half_step(out_type) * out64.abs() + least(out_type) + (2 * group + G + 19) * U * mag
