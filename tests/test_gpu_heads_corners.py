"""Backward pass of norms and rotations of heads: gradients that overflow on their way out."""
import pytest
import torch

import paper_1603_05279_b200 as X
from kv4_util import TYPES, heads_backward64, weight_error
from rows_util import gen, randn

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
