"""Distances between rows or heads that no memory has: refused on the host, whatever the products of sizes would come to in 64 bits.
None of these needs a device (the pointers are fake but well formed)."""
import ctypes

import pytest

from test_base4_cpu import DISTILL, FAR, INT4, lib, rope_args  # noqa: F401
from test_block_cpu import EINVAL, make


# tokens and a distance, the products of the last pairs being 2^64 and nothing in 64 bits
@pytest.mark.parametrize("T,token", [(2, 1 << 62), (3000, 1 << 52), ((1 << 31) - 1000, 1 << 40), ((1 << 24) + 1, 1 << 40), ((1 << 30) + 1, 1 << 34)])
def test_tokens_of_heads(lib, T, token):
    from paper_2605_24058_b200 import lordba
    before = lordba.launch_count()
    # all of them apart, so that nothing else is wrong
    places = {name: lordba.Heads((i + 1) << 42, 256, 64) for i, name in enumerate(("q", "k", "q_out", "k_out", "dq", "dk"))}
    rest = dict(w_q=0, w_k=0, positions=8 << 42, inv_freq=9 << 42)
    for name in places:
        a = dict(places, **{name: lordba.Heads(places[name].p, token, 64)})
        f = rope_args(**rest, **{n: a[n] for n in ("q", "k", "q_out", "k_out")})
        if name not in ("dq", "dk"):
            assert lib.lordba_norm_rope(ctypes.byref(f), T, lordba.BF16, None) == EINVAL, name
        g = lordba.NormRopeGrad(f=f, dq=a["dq"], dk=a["dk"], dw_q=0, dw_k=0)
        assert lib.lordba_norm_rope_backward(ctypes.byref(g), T, lordba.BF16, None, 0, None) == EINVAL, name
    assert lordba.launch_count() == before


@pytest.mark.parametrize("heads,head", [(4, 1 << 62), (4, 1 << 55), ((1 << 20), 1 << 40)])
def test_heads_far_apart(lib, heads, head):
    from paper_2605_24058_b200 import lordba
    before = lordba.launch_count()
    for name in ("q", "q_out"):
        a = rope_args(heads_q=heads, heads_k=0, **{name: lordba.Heads(64 * FAR, 1 << 26, head)})
        assert lib.lordba_norm_rope(ctypes.byref(a), 1, lordba.BF16, None) == EINVAL, name
    assert lordba.launch_count() == before


@pytest.mark.parametrize("ld", [1 << 52, (1 << 61) + 64, 1 << 62])
def test_pitches(lib, ld):
    from paper_2605_24058_b200 import lordba
    before = lordba.launch_count()
    for T in (3000,) if ld < 1 << 56 else (1, 3000):
        for name in ("ld_in", "ld_out") + (("ldq", "ld_scale", "ld_zero") if T > 1 else ()):
            p = make(lordba.Int4Proj, INT4, **dict(dict(d_out=3000, ld_in=3000, ld_out=3000), **{name: ld}))
            for f in (lib.lordba_int4_linear, lib.lordba_int4_linear_backward):
                assert f(ctypes.byref(p), T, lordba.BF16, 8 * FAR, 1 << 40, None) == EINVAL, name
        for name in ("ld_logits", "ld_ids", "ld_teacher", "ld_dlogits"):
            d = make(lordba.Distill, DISTILL, **{name: ld})
            for f in (lib.lordba_distill_loss, lib.lordba_distill_backward):
                assert f(ctypes.byref(d), T, lordba.F32, 20 * FAR, 1 << 40, None) == EINVAL, name
    assert lib.lordba_int4_pack(FAR, ld, 2 * FAR, 128, 3000, 200, None) == EINVAL and lib.lordba_int4_pack(FAR, 200, 2 * FAR, ld, 3000, 200, None) == EINVAL
    names = ("ldw", "ldq", "lds", "ldz")
    for name in names:
        ldw, ldq, lds, ldz = (ld if n == name else small for n, small in zip(names, (200, 128, 4, 4)))
        assert lib.lordba_int4_quantize(FAR, ldw, lordba.F32, 2 * FAR, ldq, 3 * FAR, lds, 4 * FAR, ldz, 3000, 200, 64, lordba.F16, None) == EINVAL, name
    assert lib.lordba_int4_dequantize(ctypes.byref(make(lordba.Int4Proj, INT4, ld_out=ld)), lordba.BF16, None) == EINVAL
    # the operators next to the adapters
    assert lib.lordba_dropout(FAR, ld, None, 0, 2 * FAR, 64, 3000, 64, 0.5, 1, 0, lordba.F32, None) == EINVAL
    assert lib.lordba_int8_quantize_rows(FAR, 64, 2 * FAR, ld, 3 * FAR, 3000, 64, lordba.F32, None) == EINVAL
    assert lordba.launch_count() == before


def test_a_pitch_whose_bytes_come_to_nothing(lib):
    """Single rows that meet, of a pitch of 2^64 bytes: no remainder is taken by it."""
    from paper_2605_24058_b200 import lordba
    both = make(lordba.Distill, DISTILL, ld_logits=1 << 62, ld_dlogits=1 << 62, dlogits=1 * FAR + 16)
    assert lib.lordba_distill_loss(ctypes.byref(both), 1, lordba.F32, None, 0, None) == EINVAL
