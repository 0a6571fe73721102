"""What the workspace queries of the operators next to the adapters answer for: the call with these very pointers and
pitches, as the header says.  Without a device (the pointers are fake but well formed) unaligned operands are copied."""
import ctypes

import pytest

from paper_2605_24058_b200 import lordba


@pytest.fixture(scope="module")
def lib():
    from paper_2605_24058_b200 import build
    build.build_library()
    return lordba.load()


def piece(rows, bytes_a_row):
    """Bytes of an aligned copy: rows on 16-byte boundaries, the whole a multiple of 256."""
    return (rows * ((bytes_a_row + 15) // 16 * 16) + 255) // 256 * 256


def test_int8_linear(lib):
    T, d_in, d_out = 300, 1001, 777
    base = dict(s_x=0x200000, s_w=0x400000, y=0x500000, d_in=d_in, d_out=d_out, ldx=1008, ldw=1008, ldy=d_out)
    need = lambda **kw: lib.lordba_int8_linear_workspace_bytes(ctypes.byref(lordba.Int8Proj(**{**base, **kw})), T)
    assert need() == 0 and need(x=0x100000, w=0x300000) == 0                  # NULL counts as aligned
    a, b = need(x=0x100001, w=0x300000), need(x=0x100000, w=0x300008)
    both, pitch = need(x=0x100001, w=0x300008), need(x=0x100000, w=0x300000, ldw=1001)
    if a:                # a device may have a kernel that takes such operands as they are
        assert (a, b, both, pitch) == (piece(T, d_in), piece(d_out, d_in), piece(T, d_in) + piece(d_out, d_in), piece(d_out, d_in))
    # a workspace that was sized for other pointers is refused before anything is launched
    if a:
        p = lordba.Int8Proj(**{**base, "x": 0x100001, "w": 0x300000})
        before = lordba.launch_count()
        assert lib.lordba_int8_linear(ctypes.byref(p), T, lordba.F32, 0x700000, need(x=0x100000, w=0x300000), None) == 1
        assert lordba.launch_count() == before


def test_gated(lib):
    T, d_in, n = 300, 130, 257
    base = dict(h=0x800000, d_in=d_in, d_hidden=n, ldx=136, ldw=136, ldh=n)
    need = lambda **kw: lib.lordba_gated_workspace_bytes(ctypes.byref(lordba.Gated(**{**base, **kw})), T)
    assert need() == 0 and need(x=0x100000, w_gate=0x200000, w_up=0x300000) == 0
    odd = need(x=0x100000, w_gate=0x200000, w_up=0x300002)
    assert odd in (0, piece(n, 2 * d_in))


def test_gated_backward(lib):
    T, d_in, n = 300, 130, 257
    base = dict(dh=0x100000, gate=0x200000, up=0x300000, x=0x400000, w_gate=0x500000, w_up=0x600000, dgate=0x700000, dup=0x800000, d_in=d_in,
                d_hidden=n, ld_dh=n, ld_pre=n, ldx=136, ldw=136, ld_dpre=n, ld_dx=136, ld_dw=136)
    need = lambda T=T, **kw: lib.lordba_gated_backward_workspace_bytes(ctypes.byref(lordba.GatedGrad(**{**base, **kw})), T)
    assert need() == 0                                                    # nothing is made but dgate and dup
    parts = dict(dx=0x900000), dict(dw_gate=0xA00000, dw_up=0xB00000)
    one, other = (need(**p) for p in parts)
    assert need(**parts[0], **parts[1]) == max(one, other)                    # they run one after the other
    assert need(**parts[0], ld_dpre=264) == 0 and need(**parts[1], ld_dpre=264) == 0
    # up to 64 tokens the rest of dgate and dup lies there too
    few = 2 * piece(8, 2 * n)
    assert need(T=8, **parts[0], ld_dpre=264) >= few and need(T=8, **parts[1], ld_dpre=264) >= few
    assert need(T=0, **parts[0]) == 0
