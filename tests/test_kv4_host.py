"""What the library works out on the host for the attention over a cache in 4 bits (no GPU needed)."""
import ctypes

import pytest

import paper_1603_05279_b200 as X
from paper_1603_05279_b200 import binding as B
from test_binding import run_child


@pytest.mark.parametrize("seqs", [0, -1, -(1 << 31), (1 << 20) + 1])
def test_numbers_of_sequences_that_no_call_takes_have_no_scratch(seqs):
    for rows in (0, 1, 100, 100000):
        for heads in (1, 8):
            d, r = B.xnor_kv4_desc(8, 32, heads, 64, seqs, 4), B.xnor_kv4_rows(rows, 8, B.XNOR_BF16, 0, 0.1, 512, 512)
            assert X.load().xnor_kv4_work_bytes(ctypes.byref(d), ctypes.byref(r)) == 0
            d.seqs = 1
            assert X.load().xnor_kv4_work_bytes(ctypes.byref(d), ctypes.byref(r)) > 0


def test_a_table_of_no_sequences_is_refused():
    run_child("""
d = X.make_kv4_desc(8, 32, 1, 64)
f = lambda *s, t=torch.int32: fake(*s, dtype=t)
for rows in (1, 100, 3000):
    q = f(rows, 1, 64, t=torch.bfloat16)
    raises(X.XnorError, lambda: X.xnor_kv4_attention(q, f(8, 1, 2, 16 * 72, t=torch.uint8), f(1), f(0), f(0, 4), d, 0.1, 0, f(rows, 1, 64, t=torch.bfloat16),
                                                     None, f(1 << 24, t=torch.uint8), stream=0))
""")
