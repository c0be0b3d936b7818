"""Backward pass of norms and rotations of heads: gradients that overflow on their way out, and no norm, through the C entry."""
import ctypes

import pytest
import torch

import paper_1603_05279_b200 as X
from paper_1603_05279_b200 import binding as B
from kv4_util import TYPES, heads_backward64, weight_error
from rows_util import Guards, U, gen, half_step, least, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,D", [(9, 128), (17, 128), (3, 64), (17, 64), (5, 256), (33, 256), (9, 80)])
@pytest.mark.parametrize("over", ["gradients that arrive", "values", "neither"])
def test_a_gradient_too_large_for_its_type_leaves_the_weights_alone(H, D, over):
    """The first head's gradient overflows F16 where it is stored; the weight's gradient, in fp32, does not."""
    T = 40
    g = gen(1)
    x, dy = randn((T, H, D), g, torch.float16), randn((T, H, D), g, torch.float16)
    x[:, 0] *= 2.0 ** -12
    dy[:, 0] *= 2.0 ** 6
    pos, rope = torch.arange(T, dtype=torch.int32, device="cuda"), X.make_rope(T, 64)
    want, _, w64, size = heads_backward64(dy, x, None, 1e-12, rope, pos, False)
    assert (want[:, 0].abs() > 65520).double().mean() > 0.5 and (want[:, 1:].abs() < 60000).all() and w64.isfinite().all()
    dx = dy if over == "gradients that arrive" else x if over == "values" else torch.empty_like(x)
    dw, _, work = X.alloc_qk_backward(T, H, 0, D)
    X.xnor_qk_norm_rope_backward(dy, None, x, None, None, None, 1e-12, pos, rope, False, dx, None, dw, None, work)
    X.xnor_check_device()
    assert dx[:, 0].isinf().any() and dx[:, 1:].isfinite().all()
    assert ((dw.double() - w64).abs() <= weight_error(T, H) * size).all()


@pytest.mark.parametrize("D", [64, 128, 256, 80])
@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("in_place", [False, True])
def test_without_norm_neither_values_nor_weights_are_read(D, t, in_place):
    """q and k are null, their strides and the weights anything: the gradients are the turned ones, the weights' zeros."""
    T, Hq, Hk, g, guards = 30, 5, 3, gen(9), Guards()
    dq_out, dk_out = randn((T, Hq, D), g, TYPES[t]), randn((T, Hk, D), g, TYPES[t])
    wants = [heads_backward64(d, None, None, None, X.make_rope(T, 64), torch.arange(T, device="cuda"), False)[:2] for d in (dq_out, dk_out)]
    dq, dk = (dq_out, dk_out) if in_place else (guards.rows(T, Hq * D, TYPES[t]), guards.rows(T, Hk * D, TYPES[t]))
    dqw, dkw = (guards.flat(D, torch.float32) for _ in "qk")
    pos, rope = torch.arange(T, dtype=torch.int32, device="cuda"), X.make_rope(T, 64)
    d = B.xnor_heads_desc(rows=T, dim=D, q_heads=Hq, k_heads=Hk, type={"bf16": B.XNOR_BF16, "f32": B.XNOR_F32}[t], weight_type=99, norm=0,
                          eps=-1.0, rot=64, pairs=0, positions=T, q_stride=-7, k_stride=3, v_stride=0, q_out_stride=Hq * D,
                          k_out_stride=Hk * D, dq_stride=Hq * D, dk_stride=Hk * D)
    p = lambda x: ctypes.c_void_p(x.data_ptr())
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    null, odd = ctypes.c_void_p(0), ctypes.c_void_p(rope.data_ptr() + 4)
    assert X.load().xnor_qk_norm_rope_backward(p(dq_out), p(dk_out), null, null, odd, odd, p(pos), p(rope), ctypes.byref(d), p(dq), p(dk), p(dqw),
                                               p(dkw), null, stream) == B.XNOR_OK
    X.xnor_check_device()
    guards.check()
    h = half_step(TYPES[t])
    for got, (want, size) in zip((dq, dk), wants):
        # two products and their sum: 2 U
        assert ((got.view(want.shape).double() - want).abs() <= h * want.abs() + (1 + h) * 2 * U * size + least(TYPES[t])).all()
    assert (dqw == 0).all() and (dkw == 0).all()
