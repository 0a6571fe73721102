"""Host-side checks of the operators around a 4-bit base: bad arguments are found before any launch, so none of these
needs a device (the pointers are fake but well formed)."""
import ctypes

import pytest

from test_block_cpu import EALIGN, EINVAL, EUNSUP, make

FAR = 1 << 20


@pytest.fixture(scope="module")
def lib():
    from paper_2605_24058_b200 import build, lordba
    build.build_library()
    return lordba.load()


# 200 columns: two blocks of the carrier, four groups of 64
INT4 = dict(input=1 * FAR, out=2 * FAR, q=3 * FAR, scale=4 * FAR, zero=5 * FAR, d_in=200, d_out=32, ld_in=200, ld_out=200, ldq=128,
            ld_scale=4, ld_zero=4, group=64)


@pytest.mark.parametrize("backward", [False, True])
def test_int4_product_arguments(lib, backward):
    from paper_2605_24058_b200 import lordba
    before = lordba.launch_count()
    f = lib.lordba_int4_linear_backward if backward else lib.lordba_int4_linear
    query = lib.lordba_int4_linear_backward_workspace_bytes if backward else lib.lordba_int4_linear_workspace_bytes
    call = lambda T=4, dt=lordba.BF16, **kw: f(ctypes.byref(make(lordba.Int4Proj, INT4, **kw)), T, dt, None, 0, None)
    assert f(None, 4, lordba.BF16, None, 0, None) == EINVAL and query(None, 4) == 0
    assert call(T=0) == 0 and call(T=0, input=0, out=0, q=0) == 0
    assert call(T=-1) == EINVAL and call(T=1 << 31) == EINVAL and call(d_in=0) == EINVAL and call(d_out=0) == EINVAL and call(flags=1) == EINVAL
    assert call(dt=lordba.F32) == EUNSUP and call(dt=9) == EUNSUP
    for group in (0, 16, 48, 96, -32):
        assert call(group=group) == EINVAL
    assert call(ldq=64) == EINVAL and call(ld_scale=3) == EINVAL and call(ld_zero=3) == EINVAL
    assert call(ld_in=31 if backward else 199) == EINVAL and call(ld_out=199 if backward else 31) == EINVAL
    for name in ("input", "out", "q", "scale"):
        assert call(**{name: 0}) == EINVAL
    assert call(q=3 * FAR + 8) == EALIGN and call(ldq=136) == EALIGN
    for name in ("input", "out", "scale"):
        assert call(**{name: INT4[name] + 1}) == EALIGN
    for name in ("input", "q", "scale", "zero"):
        assert call(out=INT4[name]) == EINVAL                       # the result over what is read
    need = query(ctypes.byref(make(lordba.Int4Proj, INT4)), 300)
    if need:
        assert f(ctypes.byref(make(lordba.Int4Proj, INT4)), 300, lordba.BF16, 8 * FAR, need - 1, None) == EINVAL
        assert f(ctypes.byref(make(lordba.Int4Proj, INT4)), 300, lordba.BF16, 8 * FAR + 16, need, None) == EALIGN
    assert query(ctypes.byref(make(lordba.Int4Proj, INT4, group=33)), 4) == 0 and query(ctypes.byref(make(lordba.Int4Proj, INT4)), 0) == 0
    assert lordba.launch_count() == before


def test_int4_carrier_arguments(lib):
    from paper_2605_24058_b200 import lordba
    before = lordba.launch_count()
    assert [lordba.int4_row_bytes(d) for d in (1, 128, 129, 4096)] == [64, 64, 128, 2048] and lordba.int4_row_bytes(0) == -1
    pack = lambda v=FAR, ldv=200, q=2 * FAR, ldq=128, n=32, d=200: lib.lordba_int4_pack(v, ldv, q, ldq, n, d, None)
    assert pack(n=0) == 0 and pack(v=0) == EINVAL and pack(q=0) == EINVAL and pack(ldv=199) == EINVAL and pack(ldq=64) == EINVAL
    assert pack(d=0) == EINVAL and pack(n=-1) == EINVAL and pack(q=2 * FAR + 4) == EALIGN and pack(ldq=132) == EALIGN and pack(q=FAR + 16) == EINVAL

    def quantize(w=FAR, ldw=200, wt=lordba.F32, q=2 * FAR, ldq=128, scale=3 * FAR, lds=4, zero=4 * FAR, ldz=4, n=32, d=200, group=64, dt=lordba.F16):
        return lib.lordba_int4_quantize(w, ldw, wt, q, ldq, scale, lds, zero, ldz, n, d, group, dt, None)

    assert quantize(n=0) == 0 and quantize(wt=7) == EUNSUP and quantize(dt=lordba.F32) == EUNSUP
    assert quantize(group=24) == EINVAL and quantize(ldw=199) == EINVAL and quantize(ldq=100) == EINVAL and quantize(lds=3) == EINVAL and quantize(ldz=3) == EINVAL
    assert quantize(w=0) == EINVAL and quantize(q=0) == EINVAL and quantize(scale=0) == EINVAL and quantize(n=-1) == EINVAL
    assert quantize(w=FAR + 2) == EALIGN and quantize(q=2 * FAR + 8) == EALIGN and quantize(scale=3 * FAR + 1) == EALIGN
    assert quantize(q=FAR + 16) == EINVAL and quantize(scale=FAR) == EINVAL and quantize(zero=3 * FAR) == EINVAL and quantize(zero=2 * FAR) == EINVAL
    back = lambda dt=lordba.BF16, **kw: lib.lordba_int4_dequantize(ctypes.byref(make(lordba.Int4Proj, INT4, **kw)), dt, None)
    assert lib.lordba_int4_dequantize(None, lordba.BF16, None) == EINVAL and back(dt=lordba.F32) == EUNSUP
    assert back(out=0) == EINVAL and back(q=0) == EINVAL and back(ld_out=199) == EINVAL and back(group=8) == EINVAL and back(out=2 * FAR + 1) == EALIGN
    assert back(out=3 * FAR) == EINVAL
    assert lordba.launch_count() == before


def rope_args(**kw):
    from paper_2605_24058_b200 import lordba
    h = lambda p, token=64 * 4, head=64: lordba.Heads(p, token, head)
    values = dict(q=h(FAR), k=h(2 * FAR), q_out=h(3 * FAR), k_out=h(4 * FAR), w_q=5 * FAR, w_k=6 * FAR, positions=7 * FAR, inv_freq=8 * FAR,
                  heads_q=4, heads_k=4, d=64, rotary=64, w_dtype=lordba.F32, flags=0, eps=1e-6)
    values.update(kw)
    return lordba.NormRope(**values)


def test_norm_rope_arguments(lib):
    from paper_2605_24058_b200 import lordba
    before = lordba.launch_count()
    h = lordba.Heads
    call = lambda T=8, dt=lordba.BF16, **kw: lib.lordba_norm_rope(ctypes.byref(rope_args(**kw)), T, dt, None)
    assert lib.lordba_norm_rope(None, 8, lordba.BF16, None) == EINVAL
    assert call(T=0) == 0 and call(T=0, positions=0) == 0
    assert call(T=-1) == EINVAL and call(dt=5) == EUNSUP and call(w_dtype=5) == EUNSUP and call(flags=4) == EINVAL
    assert call(d=0) == EINVAL and call(d=lordba.ROPE_MAX_D + 1) == EUNSUP and call(heads_q=0) == EINVAL and call(heads_k=-1) == EINVAL
    assert call(rotary=63) == EINVAL and call(rotary=66) == EINVAL and call(rotary=-2) == EINVAL
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(eps=eps) == EINVAL
    assert call(flags=lordba.ROPE_NO_NORM) == EINVAL                          # weights without a norm
    none = h(0, 0, 0)
    assert call(k=none) == EINVAL and call(k_out=none) == EINVAL               # keys in, none out
    assert call(q=none) == EINVAL and call(q_out=none) == EINVAL and call(positions=0) == EINVAL and call(inv_freq=0) == EINVAL
    assert call(q=h(FAR + 1, 256, 64)) == EALIGN and call(positions=7 * FAR + 4) == EALIGN and call(inv_freq=8 * FAR + 2) == EALIGN
    assert call(w_q=5 * FAR + 2) == EALIGN and call(dt=lordba.F32, k_out=h(4 * FAR + 2, 256, 64)) == EALIGN
    assert call(q=h(FAR, -256, 64)) == EINVAL and call(q_out=h(3 * FAR, 128, 64)) == EINVAL and call(q_out=h(3 * FAR, 256, 32)) == EINVAL    # vectors that share entries
    assert call(q_out=h(2 * FAR, 256, 64)) == EINVAL and call(q_out=h(4 * FAR, 256, 64)) == EINVAL         # over the keys, over k_out
    assert call(q_out=h(FAR + 128, 256, 64)) == EINVAL                         # q, moved by a head
    assert call(q_out=h(5 * FAR, 256, 64)) == EINVAL and call(k_out=h(7 * FAR, 256, 64)) == EINVAL
    assert lordba.launch_count() == before


def test_norm_rope_backward_arguments(lib):
    from paper_2605_24058_b200 import lordba
    before = lordba.launch_count()
    h = lordba.Heads
    none = h(0, 0, 0)

    def args(f=None, **kw):
        values = dict(f=rope_args(**(f or {})), dq=h(9 * FAR, 256, 64), dk=h(10 * FAR, 256, 64), dw_q=11 * FAR, dw_k=12 * FAR)
        values.update(kw)
        return lordba.NormRopeGrad(**values)

    def call(T=8, dt=lordba.BF16, f=None, ws=None, nbytes=0, **kw):
        return lib.lordba_norm_rope_backward(ctypes.byref(args(f, **kw)), T, dt, ws, nbytes, None)

    assert lib.lordba_norm_rope_backward(None, 8, lordba.BF16, None, 0, None) == EINVAL
    need = lib.lordba_norm_rope_backward_workspace_bytes(ctypes.byref(args()), 8)
    assert need > 0 and lib.lordba_norm_rope_backward_workspace_bytes(ctypes.byref(args(dw_q=0, dw_k=0)), 8) == 0
    assert call() == EINVAL and call(ws=20 * FAR, nbytes=need - 1) == EINVAL and call(ws=20 * FAR + 16, nbytes=need) == EALIGN
    assert call(dq=none) == EINVAL and call(dk=none) == EINVAL and call(f=dict(k=none)) == EINVAL and call(f=dict(heads_k=0)) == EINVAL
    assert call(f=dict(flags=lordba.ROPE_NO_NORM, w_q=0, w_k=0)) == EINVAL      # dw without a norm
    assert call(dw_q=11 * FAR + 2) == EALIGN and call(dw_q=12 * FAR) == EINVAL and call(dw_k=FAR) == EINVAL and call(dw_k=10 * FAR) == EINVAL
    assert call(dq=h(2 * FAR, 256, 64)) == EINVAL and call(dq=h(4 * FAR, 256, 64)) == EINVAL and call(dq=h(10 * FAR, 256, 64)) == EINVAL
    assert call(T=0, dw_q=0, dw_k=0) == 0 and call(T=-1) == EINVAL and call(dt=4) == EUNSUP
    assert lordba.launch_count() == before


DISTILL = dict(logits=1 * FAR, ids=2 * FAR, teacher=3 * FAR, weight=4 * FAR, loss=5 * FAR, lse=6 * FAR, dlogits=7 * FAR, vocab=100, top=8,
               ld_logits=100, ld_ids=8, ld_teacher=8, ld_dlogits=100, temperature=2.0, teacher_dtype=1, flags=1)


@pytest.mark.parametrize("backward", [False, True])
def test_distill_arguments(lib, backward):
    from paper_2605_24058_b200 import lordba
    before = lordba.launch_count()
    f = lib.lordba_distill_backward if backward else lib.lordba_distill_loss
    call = lambda T=4, dt=lordba.BF16, ws=None, nbytes=0, **kw: f(ctypes.byref(make(lordba.Distill, DISTILL, **kw)), T, dt, ws, nbytes, None)
    assert f(None, 4, lordba.BF16, None, 0, None) == EINVAL
    need = lib.lordba_distill_workspace_bytes(ctypes.byref(make(lordba.Distill, DISTILL)), 3000)
    assert need > 0 and lib.lordba_distill_workspace_bytes(None, 4) == 0 and lib.lordba_distill_workspace_bytes(ctypes.byref(make(lordba.Distill, DISTILL)), 4) == 0
    assert call(T=3000) == EINVAL and call(T=3000, ws=20 * FAR, nbytes=need - 1) == EINVAL and call(T=3000, ws=20 * FAR + 8, nbytes=need) == EALIGN
    assert call(T=0) == 0 and call(T=0, logits=0) == 0
    assert call(T=-1) == EINVAL and call(vocab=0) == EINVAL and call(flags=2) == EINVAL and call(dt=8) == EUNSUP and call(teacher_dtype=8) == EUNSUP
    assert call(top=0) == EINVAL and call(top=lordba.DISTILL_MAX_TOP + 1, ld_ids=300, ld_teacher=300) == EUNSUP
    for name in ("ld_logits", "ld_ids", "ld_teacher", "ld_dlogits"):
        assert call(**{name: 7}) == EINVAL
    for tau in (0.0, -1.0, float("nan"), float("inf"), 1e-39):
        assert call(temperature=tau) == EINVAL
    for name in ("logits", "ids", "teacher", "lse") + (("dlogits",) if backward else ("loss",)):
        assert call(**{name: 0}) == EINVAL
    for name in ("logits", "teacher", "dlogits", "lse", "weight"):
        assert call(**{name: DISTILL[name] + 1}) == EALIGN
    assert call(ids=2 * FAR + 4) == EALIGN and call(teacher_dtype=0, teacher=3 * FAR + 2) == EALIGN
    assert call(dlogits=1 * FAR, ld_dlogits=104) == EINVAL                      # the logits' place in another pitch
    for name in ("ids", "teacher", "weight", "lse"):
        assert call(dlogits=DISTILL[name]) == EINVAL
    if not backward:
        assert call(loss=6 * FAR) == EINVAL and call(loss=4 * FAR) == EINVAL and call(lse=1 * FAR) == EINVAL
    assert lordba.launch_count() == before
