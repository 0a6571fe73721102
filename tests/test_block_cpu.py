"""Host-side checks of the operators next to the adapters: bad arguments are found before any launch, so
none of these needs a device (the pointers are fake but well formed)."""
import ctypes

import pytest

EINVAL, EUNSUP, EALIGN = 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    from paper_2605_24058_b200 import build, lordba
    build.build_library()
    return lordba.load()


def make(cls, base, **kw):
    values = dict(base)
    values.update(kw)
    return cls(**values)


INT8 = dict(x=0x100000, s_x=0x200000, w=0x300000, s_w=0x400000, y=0x500000, d_in=64, d_out=32, ldx=64, ldw=64, ldy=32)
GATED = dict(x=0x100000, w_gate=0x200000, w_up=0x300000, h=0x400000, d_in=64, d_hidden=32, ldx=64, ldw=64, ldh=32)
GRAD = dict(dh=0x100000, gate=0x200000, up=0x300000, x=0x400000, w_gate=0x500000, w_up=0x600000, dgate=0x700000, dup=0x800000, dx=0x900000,
            dw_gate=0xA00000, dw_up=0xB00000, d_in=64, d_hidden=32, ld_dh=32, ld_pre=32, ldx=64, ldw=64, ld_dpre=32, ld_dx=64, ld_dw=64)


def test_int8_linear_arguments(lib):
    from paper_2605_24058_b200 import lordba
    before = lordba.launch_count()
    call = lambda T=4, dt=lordba.BF16, **kw: lib.lordba_int8_linear(ctypes.byref(make(lordba.Int8Proj, INT8, **kw)), T, dt, None, 0, None)
    assert lib.lordba_int8_linear(None, 4, lordba.BF16, None, 0, None) == EINVAL
    assert call(T=0) == 0 and call(T=0, x=0, y=0) == 0
    assert call(T=-1) == EINVAL and call(d_in=0) == EINVAL and call(T=1 << 31) == EINVAL
    assert call(ldx=63) == EINVAL and call(ldw=63) == EINVAL and call(ldy=31) == EINVAL
    assert call(dt=7) == EUNSUP
    long = lordba.INT8_MAX_DIN + 1
    assert call(d_in=long, ldx=long, ldw=long) == EUNSUP
    for name in ("x", "s_x", "w", "s_w", "y"):
        assert call(**{name: 0}) == EINVAL
    assert call(s_x=0x200002) == EALIGN and call(y=0x500001) == EALIGN and call(dt=lordba.F32, y=0x500002) == EALIGN
    assert call(y=0x100010) == EINVAL and call(y=0x300000) == EINVAL and call(y=0x200000) == EINVAL      # y over x, w, s_x
    # operands off 16-byte boundaries need a workspace
    odd = make(lordba.Int8Proj, INT8, x=0x100001)
    need = lib.lordba_int8_linear_workspace_bytes(ctypes.byref(odd), 4)
    assert lib.lordba_int8_linear_workspace_bytes(ctypes.byref(make(lordba.Int8Proj, INT8)), 4) == 0
    if need:
        assert call(x=0x100001) == EINVAL
        assert lib.lordba_int8_linear(ctypes.byref(odd), 4, lordba.BF16, 0x700010, need, None) == EALIGN
    assert lib.lordba_int8_quantize_rows(0x100000, 64, 0x200000, 64, 0x300000, 0, 64, lordba.BF16, None) == 0
    q = lambda x=0x100000, ldx=64, q=0x200000, ldq=64, s=0x300000, T=4, d=64, dt=lordba.BF16: lib.lordba_int8_quantize_rows(x, ldx, q, ldq, s, T, d, dt, None)
    assert q(dt=9) == EUNSUP and q(d=0) == EINVAL and q(T=-1) == EINVAL and q(ldx=60) == EINVAL and q(ldq=60) == EINVAL
    assert q(x=0) == EINVAL and q(q=0) == EINVAL and q(s=0) == EINVAL and q(x=0x100001) == EALIGN and q(s=0x300002) == EALIGN
    assert q(q=0x100040) == EINVAL
    assert lordba.launch_count() == before


def test_gated_arguments(lib):
    from paper_2605_24058_b200 import lordba
    before = lordba.launch_count()
    call = lambda T=4, dt=lordba.BF16, **kw: lib.lordba_gated_forward(ctypes.byref(make(lordba.Gated, GATED, **kw)), T, dt, None, 0, None)
    assert lib.lordba_gated_forward(None, 4, lordba.BF16, None, 0, None) == EINVAL
    assert call(T=0) == 0 and call(T=0, x=0) == 0
    assert call(dt=lordba.F32) == EUNSUP and call(act=2) == EUNSUP and call(flags=2) == EINVAL
    assert call(T=-1) == EINVAL and call(d_in=0) == EINVAL and call(d_hidden=0) == EINVAL
    assert call(ldx=63) == EINVAL and call(ldw=63) == EINVAL and call(ldh=31) == EINVAL
    for name in ("x", "w_gate", "w_up", "h"):
        assert call(**{name: 0}) == EINVAL
    assert call(x=0x100001) == EALIGN and call(h=0x400001) == EALIGN
    assert call(gate=0x700000, ld_pre=32) == EINVAL                          # gate without up
    assert call(gate=0x700000, up=0x800000, ld_pre=31) == EINVAL
    assert call(gate_add=0x700000, ld_add=32) == EINVAL
    assert call(gate=0x700000, up=0x700000, ld_pre=32) == EINVAL                # one buffer for both
    assert call(gate=0x400000, up=0x800000, ld_pre=32) == EINVAL                # gate over h
    assert call(gate_add=0x700000, up_add=0x800000, ld_add=32, gate=0x800000, up=0x700000, ld_pre=32) == EINVAL     # crossed
    assert call(h=0x100000) == EINVAL and call(h=0x200000) == EINVAL
    assert call(s_x=0x700000) == EINVAL                                      # scales without the flag
    assert call(flags=lordba.GATED_INT8) == EINVAL                           # the flag without scales
    long = lordba.INT8_MAX_DIN + 1
    assert call(flags=lordba.GATED_INT8, s_x=0x700000, s_gate=0x800000, s_up=0x900000, d_in=long, ldx=long, ldw=long) == EUNSUP
    assert lordba.launch_count() == before


def test_gated_backward_arguments(lib):
    from paper_2605_24058_b200 import lordba
    before = lordba.launch_count()
    call = lambda T=4, dt=lordba.BF16, **kw: lib.lordba_gated_backward(ctypes.byref(make(lordba.GatedGrad, GRAD, **kw)), T, dt, None, 0, None)
    assert lib.lordba_gated_backward(None, 4, lordba.BF16, None, 0, None) == EINVAL
    assert call(dt=lordba.F32) == EUNSUP and call(act=-1) == EUNSUP and call(flags=1) == EINVAL
    assert call(T=-1) == EINVAL and call(d_in=0) == EINVAL
    for name in ("ld_dh", "ld_pre", "ldx", "ldw", "ld_dpre", "ld_dx", "ld_dw"):
        assert call(**{name: 31}) == EINVAL
    for name in ("dh", "gate", "up", "x", "w_gate", "w_up", "dgate", "dup", "dw_gate", "dw_up"):
        assert call(**{name: 0}) == EINVAL
    for name in ("dh", "dgate", "dx", "dw_up"):
        assert call(**{name: GRAD[name] + 1}) == EALIGN
    assert call(dgate=GRAD["dh"]) == EINVAL and call(dx=GRAD["w_gate"]) == EINVAL and call(dw_gate=GRAD["dw_up"]) == EINVAL
    assert call(T=0, dx=0, dw_gate=0, dw_up=0) == 0
    assert lordba.launch_count() == before


def test_dropout_arguments(lib):
    from paper_2605_24058_b200 import lordba
    before = lordba.launch_count()

    def call(x=0x100000, ldx=64, r=None, ldr=64, out=0x200000, ldo=64, T=4, d=64, p=0.1, dt=lordba.BF16):
        return lib.lordba_dropout(x, ldx, r, ldr, out, ldo, T, d, p, 1, 2, dt, None)

    assert call(dt=3) == EUNSUP
    assert call(p=-0.1) == EINVAL and call(p=1.1) == EINVAL and call(p=float("nan")) == EINVAL
    assert call(T=-1) == EINVAL and call(d=0) == EINVAL and call(T=1 << 32) == EINVAL
    assert call(ldx=60) == EINVAL and call(ldo=60) == EINVAL and call(r=0x300000, ldr=60) == EINVAL
    assert call(x=0) == EINVAL and call(out=0) == EINVAL and call(x=0x100001) == EALIGN and call(r=0x300001) == EALIGN
    assert call(out=0x100010) == EINVAL and call(r=0x200010) == EINVAL
    assert call(T=0) == 0 and call(T=0, x=0, out=0) == 0
    assert lordba.launch_count() == before
