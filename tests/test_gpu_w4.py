"""4-bit weights: quantisation, layout and dequantisation exactly; products with rows against 64 bits."""
import pytest
import torch

import paper_1603_05279_b200 as X
from rows_util import (TYPES, Guards, gen, matmul_bound, pack_codes, randn, strided, unpack_codes, weights64)

pytestmark = pytest.mark.gpu

#        N, K: less than a tile, ragged in both, many groups; K short of, at and past a group and a tile
MATRICES = [(1, 1), (15, 31), (16, 32), (17, 33), (5, 63), (33, 65), (48, 128), (100, 129), (1000, 257), (64, 1000),
            (130, 1024), (31, 4099), (256, 4096)]


def quantize64(w, group, zeros):
    """codes, scales (fp32) and zeros of the definition: quotients rounded from 64 bits, which is exact (quotients of
    two 24-bit numbers that are no ties are at least 2^-29 of their size away from one)."""
    N, K = w.shape
    G = -(-K // group)
    g = torch.zeros((N, G * group), dtype=torch.float64, device=w.device)
    g[:, :K] = w.double()
    g = g.view(N, G, group)
    if zeros:
        lo, hi = g.amin(2).clamp(max=0), g.amax(2).clamp(min=0)
        s = ((hi - lo) / 15).float()
        z = torch.where(s > 0, torch.round(-lo / s.double()), 8.0).clamp(0, 15)
    else:
        s = (g.abs().amax(2) / 7).float()
        z = torch.full_like(s, 8.0, dtype=torch.float64)
    q = torch.where(s[:, :, None] > 0, torch.round(g / s.double()[:, :, None]), 0.0) + z[:, :, None]
    codes = q.clamp(0, 15).view(N, -1)[:, :K].to(torch.uint8)
    return codes, s.t().contiguous(), z.t().to(torch.uint8).contiguous() if zeros else None


def quantized(w, group, zeros):
    N, K = w.shape
    d, G = X.make_w4_desc(N, K, group), Guards()
    shapes = X.alloc_w4(d, zeros=True)
    packed = G.flat(shapes[0].numel(), torch.int32).view(shapes[0].shape)
    scales = G.flat(shapes[1].numel(), torch.float32).view(shapes[1].shape)
    zs = G.flat(shapes[2].numel(), torch.uint8).view(shapes[2].shape) if zeros else None
    X.xnor_w4_quantize(w, d, packed, scales, zs)
    G.check()
    return d, packed, scales, zs


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantize_and_dequantize(group, zeros, name):
    for N, K in MATRICES:
        g = gen(N * 5000 + K)
        w = randn((N, K), g, TYPES[name], 0.02)
        if K > 40:
            w[0, :40] = 0                         # a group of zeros
            w[-1] = w[-1].abs()                   # one sign only
        if K > 64 and N > 2:
            w[1, 33] = 100 * w[1, 33]             # one large value
        codes, scales, zs = quantize64(w, group, zeros)
        d, packed, s, z = quantized(w, group, zeros)
        assert torch.equal(s, scales)
        assert z is None or torch.equal(z, zs)
        assert (unpack_codes(packed, N, K) == codes.cpu().numpy()).all()
        for out in TYPES.values():
            G = Guards()
            back = G.rows(N, K, out)
            X.xnor_w4_dequantize(packed, s, z, d, back)
            G.check()
            # code - zero times scale in 64 bits is exact; the library rounds it to fp32 and then to the type
            want = weights64(codes, scales, zs, group).float().to(out)
            assert torch.equal(back, want)


@pytest.mark.parametrize("zeros", [False, True])
def test_quantize_at_borders(zeros):
    """Weights at and next to the middle between two codes, at every size of scale, down to subnormal ones."""
    g = gen(1)
    for top in (7.0, 0.0123, 1e-30, 3e-38, 1e-41, 3e38):
        w = torch.zeros((48, 128), device="cuda")
        w[:, 0], w[:, 1] = top, (-top if not zeros else -top * 0.4)
        half = torch.randint(-6, 7, (48, 126), generator=g, device="cuda") + 0.5
        w[:, 2:] = (half * (top / 7)).float()
        near = torch.randint(-1, 2, (48, 126), generator=g, device="cuda", dtype=torch.int32)
        w[:, 2:] = (w[:, 2:].contiguous().view(torch.int32) + near).view(torch.float32)
        w = w.clamp(-top, top)
        codes, scales, zs = quantize64(w, 128, zeros)
        d, packed, s, z = quantized(w, 128, zeros)
        if not torch.isfinite(scales).all():
            continue
        assert torch.equal(s, scales) and (z is None or torch.equal(z, zs))
        assert (unpack_codes(packed, 48, 128) == codes.cpu().numpy()).all(), top


def test_quantize_nan_and_infinity():
    g = gen(2)
    w = randn((20, 256), g)
    w[3, 5], w[4, 200] = float("nan"), float("-inf")
    for zeros in (False, True):
        d, packed, s, z = quantized(w, 128, zeros)
        back = torch.empty_like(w)
        X.xnor_w4_dequantize(packed, s, z, d, back)
        assert s[0, 3].isnan() and s[1, 4].isinf()
        assert back[3, :128].isnan().all() and back[4, 128:].isnan().all()
        rest = torch.ones(20, 2, dtype=torch.bool, device="cuda")
        rest[3, 0] = rest[4, 1] = False
        assert torch.isfinite(back.view(20, 2, 128)[rest]).all()


def test_pack():
    g = gen(3)
    for N, K in MATRICES:
        codes = torch.randint(0, 16, (N, K), generator=g, device="cuda").to(torch.uint8)
        d, G = X.make_w4_desc(N, K, 64), Guards()
        shape = X.alloc_w4(d)[0].shape
        packed = G.flat(shape.numel(), torch.int32).view(shape)
        X.xnor_w4_pack(codes | 0xE0, d, packed)                  # higher bits are ignored
        G.check()
        assert (unpack_codes(packed, N, K) == codes.cpu().numpy()).all()
        assert X.xnor_w4_packed_words(d) == packed.numel()


# ---- products -------------------------------------------------------------------------------
def operands(T, N, K, group, zeros, xname, seed, x_groups=False):
    """x (as stored), its scales or None, those of every value in 64 bits, and the matrix."""
    g = gen(seed)
    G = -(-K // group)
    codes = torch.randint(0, 16, (N, K), generator=g, device="cuda").to(torch.uint8)
    scales = 0.01 + torch.rand((G, N), generator=g, device="cuda")
    zs = torch.randint(0, 16, (G, N), generator=g, device="cuda").to(torch.uint8) if zeros else None
    xs = None
    if xname in ("bf16", "f16"):
        x = randn((T, K), g, TYPES[xname], 2.0)
    else:
        xs = 0.01 + torch.rand((T, G if x_groups else 1), generator=g, device="cuda")
        x = torch.randint(-128, 128, (T, K), generator=g, device="cuda").to(torch.int8) if xname == "i8" else \
            randn((T, K), g, torch.float32, 60.0).clamp(-448, 448).to(torch.float8_e4m3fn)
    each = 1.0 if xs is None else xs.double() if xs.shape[1] == 1 else \
        xs.double().repeat_interleave(group, 1)[:, :K]
    return x, xs, each, codes, scales, zs


def product(x, xs, codes, scales, zs, group, out_type, pad=0):
    N, K = codes.shape
    d, G = X.make_w4_desc(N, K, group), Guards()
    if N * K > 1 << 20:                          # (the library's own layout, which test_pack compares)
        packed = X.alloc_w4(d)[0]
        X.xnor_w4_pack(codes, d, packed)
    else:
        packed = pack_codes(codes.cpu().numpy()).cuda()
    out = G.rows(x.shape[0], N, out_type, pad)
    X.xnor_w4_matmul(x, xs, packed, scales, zs, d, out)
    X.xnor_check_device()
    G.check()
    return out


def check_product(x, each, codes, scales, zs, group, out):
    W = weights64(codes, scales, zs, group)
    x64 = x.float().double()
    want = (x64 * each) @ W.t()
    off = (out.double() - want).abs() - matmul_bound(x.float(), each, W, codes.shape[1], group, out.dtype, want)
    assert (off <= 0).all(), (off.max(), out.dtype)


ROWS = [1, 2, 7, 8, 9, 16, 17, 33, 65, 100]


@pytest.mark.parametrize("xname", ["bf16", "f16", "i8", "e4m3"])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_product_sizes(xname, group):
    """Every number of rows on ragged matrices, with and without zero points and scales of groups."""
    for i, (N, K) in enumerate(MATRICES + [(300, 520), (129, 2112)]):
        for j, T in enumerate(ROWS):
            if (i + j) % 3 and not (T == 1 or K == 129):
                continue
            x, xs, each, codes, scales, zs = operands(T, N, K, group, (i + j) % 2 == 0, xname, i * 100 + j, j % 2 == 1)
            out_type = list(TYPES.values())[(i + j) % 3]
            out = product(x, xs, codes, scales, zs, group, out_type)
            check_product(x, each, codes, scales, zs, group, out)


@pytest.mark.parametrize("xname", ["bf16", "f16", "i8", "e4m3"])
@pytest.mark.parametrize("T,N,K", [(1, 4096, 4096), (16, 2048, 1088), (40, 1024, 4096), (300, 512, 1024), (777, 384, 640), (2050, 136, 192),
                                   (300, 5000, 328), (1000, 2500, 1100)])
def test_product_large(xname, T, N, K):
    x, xs, each, codes, scales, zs = operands(T, N, K, 128, T % 2 == 1, xname, T, T == 300)
    out = product(x, xs, codes, scales, zs, 128, torch.float32)
    check_product(x, each, codes, scales, zs, 128, out)


@pytest.mark.parametrize("xname", ["bf16", "f16", "i8", "e4m3"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T,N,K", [(300, 5000, 328), (193, 9500, 161), (384, 4800, 329), (12, 6200, 4160), (9, 128, 4096)])
def test_product_of_every_kernel(xname, group, T, N, K):
    """Shapes that the largest blocks take (whole and ragged columns, addresses for copies or not), and the smallest."""
    x, xs, each, codes, scales, zs = operands(T, N, K, group, K % 2 == 0, xname, T, T == 300)
    out = product(x, xs, codes, scales, zs, group, torch.bfloat16)
    check_product(x, each, codes, scales, zs, group, out)


@pytest.mark.parametrize("xname", ["bf16", "f16", "i8", "e4m3"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", [12, 30, 50, 100])
def test_product_of_several_tiles_per_block(xname, group, T):
    """More tiles than a GPU has SMs, with odd and even numbers of groups and of blocks of columns."""
    for K in (97, 161, 200, 328):
        x, xs, each, codes, scales, zs = operands(T, 20001, K, group, K % 2 == 0, xname, T + K, K > 180)
        out = product(x, xs, codes, scales, zs, group, torch.float16 if xname == "f16" else torch.float32)
        check_product(x, each, codes, scales, zs, group, out)


@pytest.mark.parametrize("xname", ["bf16", "f16", "i8", "e4m3"])
@pytest.mark.parametrize("T", [1, 5, 20, 70, 200])
def test_product_of_rows_apart(xname, T):
    """Rows of x at strides that are and are not multiples of 16 bytes; what lies between out's rows stays."""
    for K, xpad, pad in ((128, 16, 0), (129, 0, 3), (1000, 1, 1), (512, 4, 5)):
        x, xs, each, codes, scales, zs = operands(T, 50, K, 64, True, xname, K + T)
        out = product(_apart(x, xpad), xs, codes, scales, zs, 64, torch.bfloat16, pad)
        check_product(x, each, codes, scales, zs, 64, out)


@pytest.mark.parametrize("xname", ["bf16", "f16", "i8", "e4m3"])
@pytest.mark.parametrize("T", [2, 17, 33, 70, 129])
def test_product_of_rows_at_odd_addresses(xname, T):
    """Rows of an odd number of columns, from less than a word to several blocks of columns; NaN (int8: -100)
    between them and behind the last one."""
    for K, pad in ((1, 0), (3, 0), (5, 2), (63, 0), (64, 1), (65, 0), (129, 6), (191, 4), (701, 0), (1280, 3)):
        x, xs, each, codes, scales, zs = operands(T, 130, K, 32, True, xname, K + T)
        if xname in ("i8", "e4m3"):
            buf = torch.full((T * (K + pad) + 40,), -100 if xname == "i8" else 127, dtype=torch.int8, device="cuda").view(x.dtype)
        else:
            buf = torch.full((T * (K + pad) + 40,), float("nan"), dtype=x.dtype, device="cuda")
        rows = buf.view(torch.int8 if x.element_size() == 1 else torch.int16).as_strided((T, K), (K + pad, 1))
        rows.copy_(x.view(rows.dtype))
        out = product(rows.view(x.dtype), xs, codes, scales, zs, 32, torch.float32)
        check_product(x, each, codes, scales, zs, 32, out)


def _apart(x, pad):
    """x with its rows `pad` elements further apart, NaN (int8: 77) between them."""
    if not pad:
        return x
    if x.dtype == torch.float8_e4m3fn:
        return strided(x.view(torch.int8), pad).view(torch.float8_e4m3fn)       # 77 is finite
    return strided(x, pad)


@pytest.mark.parametrize("T", [1, 3, 30, 150])
def test_product_of_whole_numbers_is_exact(T):
    """int8 rows, scales of one: every sum is a whole number below 2^24."""
    for N, K, group in ((40, 1024, 32), (100, 1000, 128), (33, 500, 64)):
        x, _, _, codes, _, zs = operands(T, N, K, group, True, "i8", K)
        x.fill_(127)
        x[:, ::3] = -128
        G = -(-K // group)
        one, xs = torch.ones((G, N), device="cuda"), torch.ones((T, 1), device="cuda")
        out = product(x, xs, codes, one, zs, group, torch.float32)
        assert torch.equal(out.double(), x.double() @ weights64(codes, one, zs, group).t())


@pytest.mark.parametrize("T", [1, 9, 40, 130])
def test_rows_do_not_mix(T):
    """NaN and infinity in one row of x stay in its row of out; a NaN scale stays in its column."""
    x, _, each, codes, scales, zs = operands(T, 70, 384, 128, False, "bf16", 9)
    x[0, 5] = float("nan")
    if T > 2:
        x[T - 1, 383] = float("inf")
    scales = scales.clone()
    scales[1, 13] = float("nan")
    out = product(x, None, codes, scales, zs, 128, torch.float32)
    assert out[0].isnan().all() and out[:, 13].isnan().all()
    keep = [t for t in range(1, T - 1)]
    cols = [n for n in range(70) if n != 13]
    if keep:
        assert torch.isfinite(out[keep][:, cols]).all()
    if T > 2:
        # infinity times code - zero: infinite, or NaN where that is 0
        zero = codes[:, 383] == 8
        zero[13] = True
        assert out[T - 1][zero].isnan().all() and out[T - 1][~zero].isinf().all()


def test_product_of_no_rows():
    d = X.make_w4_desc(40, 100, 32)
    packed, scales, _ = X.alloc_w4(d)
    X.xnor_w4_matmul(torch.empty((0, 100), device="cuda", dtype=torch.bfloat16), None, packed, scales, None, d,
                     torch.empty((0, 40), device="cuda"))


def test_one_row_for_all():
    x, _, each, codes, scales, zs = operands(1, 100, 256, 64, True, "f16", 4)
    for T in (5, 50):
        out = product(x.expand(T, 256), None, codes, scales, zs, 64, torch.float16)
        assert (out == out[0]).all()
        check_product(x, each, codes, scales, zs, 64, out[:1])


@pytest.mark.parametrize("T", [1, 12, 60, 300])
def test_same_bits_every_time(T):
    x, xs, _, codes, scales, zs = operands(T, 500, 2048, 128, True, "i8", 5, True)
    first = product(x, xs, codes, scales, zs, 128, torch.float32)
    for _ in range(4):
        assert torch.equal(first, product(x, xs, codes, scales, zs, 128, torch.float32))


@pytest.mark.parametrize("T", [2, 40])
def test_rows_beyond_32_bits(T):
    """Rows of x and of out that lie 2^31 elements behind the first ones."""
    x, _, each, codes, scales, zs = operands(T, 64, 64, 64, False, "bf16", 6)
    far = ((1 << 31) + 64) // (T - 1) + 16 & ~15
    bigx = torch.zeros(far * (T - 1) + 64, dtype=torch.bfloat16, device="cuda")
    bigo = torch.zeros(far * (T - 1) + 64, dtype=torch.bfloat16, device="cuda")
    fx, fo = bigx.as_strided((T, 64), (far, 1)), bigo.as_strided((T, 64), (far, 1))
    fx.copy_(x)
    d = X.make_w4_desc(64, 64, 64)
    X.xnor_w4_matmul(fx, None, pack_codes(codes.cpu().numpy()).cuda(), scales, zs, d, fo)
    check_product(x, each, codes, scales, zs, 64, fo)
    assert int((bigo != 0).sum()) == int((fo != 0).sum())
