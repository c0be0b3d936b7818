"""Quantisation of weights so small that their scale itself loses bits: codes stay within 0 .. 15."""
import pytest
import torch

import paper_1603_05279_b200 as X
from rows_util import unpack_codes
from test_gpu_w4 import quantize64, quantized

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -149                   # the least number of fp32


def units(counts, device="cuda"):
    """Whole numbers of units as fp32, by their bits."""
    c = torch.as_tensor(counts, dtype=torch.int32, device=device)
    return (c.abs() | torch.where(c < 0, torch.tensor(-2 ** 31, dtype=torch.int32, device=device), 0)).view(torch.float32)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_codes_of_the_smallest_weights(group, zeros):
    """Largest magnitudes of 0 to 300 units, of either sign, alone and among others: the scale is the nearest whole number
    of units to a seventh (or to a 15th of the span), so that quotients reach 10 and zero points would reach 22."""
    for sign in (1, -1):
        N, K = 301, 2 * group
        c = torch.zeros((N, K), dtype=torch.int32, device="cuda")
        top = torch.arange(N, dtype=torch.int32, device="cuda")
        c[:, 0] = sign * top
        c[:, 5] = -sign * (top // 3)
        c[:, 17] = sign * (top * 3 // 4)
        c[:, group + 3] = sign * top                  # alone in its group
        w = units(c)
        codes, scales, zs = quantize64(w, group, zeros)
        d, packed, s, z = quantized(w, group, zeros)
        assert torch.equal(s, scales) and (z is None or torch.equal(z, zs))
        got = torch.from_numpy(unpack_codes(packed, N, K)).cuda()
        bad = (got != codes).any(1)
        assert not bad.any(), (sign, torch.nonzero(bad).view(-1)[:20].tolist())
