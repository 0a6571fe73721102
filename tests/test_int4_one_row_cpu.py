"""A single row of a 4-bit product has no pitch: no copy of it is asked for because of its width.  No device needed."""
import ctypes

import pytest

from test_base4_cpu import FAR, INT4, lib  # noqa: F401
from test_block_cpu import make


@pytest.mark.parametrize("ld", [201, 200, 203, 1 << 50])
def test_no_workspace(lib, ld):
    from paper_2605_24058_b200 import lordba
    forward, backward = lib.lordba_int4_linear_workspace_bytes, lib.lordba_int4_linear_backward_workspace_bytes
    p = lambda **kw: ctypes.byref(make(lordba.Int4Proj, INT4, **dict(dict(d_in=199, d_out=201, ld_in=ld, ld_out=201, ld_zero=4), **kw)))
    assert forward(p(), 1) == 0 and backward(p(ld_in=max(ld, 201)), 1) == 0
    # off the 16-byte boundaries, and more rows than one of such a pitch, are copied as before
    assert forward(p(input=FAR + 2), 1) > 0 and backward(p(input=FAR + 2), 1) > 0
    assert (forward(p(), 2) > 0) == (ld % 8 != 0)
