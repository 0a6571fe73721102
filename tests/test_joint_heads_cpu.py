"""Queries and keys as slices of a joint projection's output that hold their entries in turns, head by head: outputs may lie there
(in place, or gradients in a joint buffer), as long as no two vectors share an entry.  Checks on the host, no device needed."""
import ctypes

import pytest

from test_base4_cpu import FAR, lib, rope_args  # noqa: F401
from test_block_cpu import EINVAL


def calls(lib, T, heads_q, heads_k, d, ins, outs):
    """Statuses of the forward call, and of the backward call with `outs` as gradients of q and k."""
    from paper_2605_24058_b200 import lordba
    h = lambda v: lordba.Heads(*v)
    rest = dict(heads_q=heads_q, heads_k=heads_k, d=d, rotary=d // 2 * 2, w_q=50 * FAR, w_k=51 * FAR, positions=52 * FAR, inv_freq=53 * FAR)
    a = rope_args(q=h(ins[0]), k=h(ins[1]), q_out=h(outs[0]), k_out=h(outs[1]), **rest)
    forward = lib.lordba_norm_rope(ctypes.byref(a), T, lordba.BF16, None)
    f = rope_args(q=h(ins[0]), k=h(ins[1]), q_out=h((60 * FAR, heads_q * d, d)), k_out=h((62 * FAR, heads_k * d, d)), **rest)
    g = lordba.NormRopeGrad(f=f, dq=h(outs[0]), dk=h(outs[1]), dw_q=0, dw_k=0)
    return forward, lib.lordba_norm_rope_backward(ctypes.byref(g), T, lordba.BF16, None, 0, None)


@pytest.mark.parametrize("T", [1, 2, 9])
@pytest.mark.parametrize("heads", [1, 4])
@pytest.mark.parametrize("d", [64, 7])
def test_entries_in_turns(lib, T, heads, d):
    """(token, head, 3, entry): q, k and v of a head side by side."""
    e = 2
    at = lambda i, base=FAR: (base + i * d * e, heads * 3 * d, 3 * d)
    elsewhere = lambda i: at(i, 20 * FAR)
    for ins, outs in [((at(0), at(1)), (at(0), at(1))), ((at(0), at(1)), (elsewhere(0), elsewhere(1))), ((at(2), at(0)), (at(2), at(0)))]:
        assert EINVAL not in calls(lib, T, heads, heads, d, ins, outs)
    shifted = lambda i, n, base=FAR: (base + (i * d + n) * e, heads * 3 * d, 3 * d)
    # over one another by an entry, over the other side, one buffer for both
    for outs in [(shifted(0, 1), at(1)), (at(0), shifted(1, -1)), (at(1), at(0)), (elsewhere(0), elsewhere(0)), (elsewhere(0), shifted(0, d - 1, 20 * FAR))]:
        assert calls(lib, T, heads, heads, d, (at(0), at(1)), outs) == (EINVAL, EINVAL), (T, heads, outs)


@pytest.mark.parametrize("T", [1, 5])
def test_fewer_keys_in_turns(lib, T):
    """Four queries, a key and a value in turns cannot be written as one distance between heads; two keys behind pairs can."""
    d, e = 32, 2
    q, k = (FAR, 4 * 2 * d, 2 * d), (FAR + d * e, 4 * 2 * d, 4 * d)           # q x q k ..., in rows of eight vectors
    assert EINVAL not in calls(lib, T, 4, 2, d, (q, k), (q, k))
    assert calls(lib, T, 4, 2, d, (q, k), (q, (FAR + 2 * d * e, 8 * d, 4 * d))) == (EINVAL, EINVAL)
