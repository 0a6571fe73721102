"""heads_k = 0: nothing that belongs to keys is looked at, whatever it holds.  No device needed."""
import ctypes

from test_base4_cpu import FAR, lib, rope_args  # noqa: F401
from test_block_cpu import EALIGN, EINVAL


def test_nothing_of_the_keys_is_looked_at(lib):
    from paper_2605_24058_b200 import lordba
    h = lordba.Heads
    wrong = [dict(w_k=6 * FAR + 1), dict(w_k=3 * FAR), dict(w_q=0, w_k=6 * FAR, w_dtype=9), dict(w_q=0, w_k=6 * FAR, flags=lordba.ROPE_NO_NORM), dict(k=h(0, 0, 0), k_out=h(0, 0, 0)),
             dict(k=h(3 * FAR, -1, -1), k_out=h(FAR, 1, 1))]
    for kw in wrong:
        a = rope_args(heads_k=0, **kw)
        assert lib.lordba_norm_rope(ctypes.byref(a), 8, lordba.BF16, None) not in (EINVAL, EALIGN, 2), kw
        g = lordba.NormRopeGrad(f=a, dq=h(9 * FAR, 256, 64), dk=h(9 * FAR + 1, 1, 1), dw_q=0, dw_k=0)
        assert lib.lordba_norm_rope_backward(ctypes.byref(g), 8, lordba.BF16, None, 0, None) not in (EINVAL, EALIGN, 2), kw
    # those of the queries are
    assert lib.lordba_norm_rope(ctypes.byref(rope_args(heads_k=0, w_q=5 * FAR + 1)), 8, lordba.BF16, None) == EALIGN
