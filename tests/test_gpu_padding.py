"""What lies between the rows of y belongs to the caller: the tcgen05 adapter kernel, whose copy engine writes 16 bytes at
a time, on widths that are no multiple of 8 in padded rows.  Results against the oracle (bounds of gpu_util.py), the
columns behind each row bit for bit as they were, NaN patterns among them."""
import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba, workloads
from gpu_util import DeviceProj, assert_close, oracle_forward, torch_to_f64

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _auto_afterwards():
    yield
    lordba.set_variant(lordba.VARIANT_AUTO)


def in_padded_rows(d, p, ldy, seed):
    """The projection with y inside a buffer of random bits; (buffer, the bits behind the rows)."""
    rng = np.random.default_rng(seed)
    bits = torch.from_numpy(rng.integers(-32768, 32768, (p.T + 1, ldy), dtype=np.int16)).cuda()
    buf = bits.view(d.y.dtype)
    buf[:p.T, :p.d_out] = d.y
    d.y = buf[:p.T, :p.d_out]
    return bits


def behind(bits, p):
    return bits[:p.T, p.d_out:].clone(), bits[p.T:].clone()


# one tile and several, one CTA a tile and clusters; a last chunk that is all tail (65, 71), that holds whole pieces too, and
# that is one element short of whole; rows that end in their own piece (1001 in 1008) and with whole pieces behind
SIZES = [(512, 250, 256), (512, 65, 72), (256, 71, 72), (1024, 1001, 1008), (512, 1007, 1024), (320, 257, 288), (2048, 2050, 2056)]


@pytest.mark.parametrize("d_in,d_out,ldy", SIZES)
@pytest.mark.parametrize("T", [1, 130, 2400])
@pytest.mark.parametrize("dtype,r", [("bf16", 16), ("f16", 32), ("f16-exact", 64)])
def test_the_tcgen05_kernel_leaves_what_is_behind_the_rows(oracle, d_in, d_out, ldy, T, dtype, r):
    p = workloads.make_projection(d_in, d_out, r, T, dtype[:4].rstrip("-"), seed=d_out + T, scales_f16=dtype == "f16-exact")
    if dtype == "f16-exact":
        p.meta["scales_f16"] = True
    d = DeviceProj(p)
    bits = in_padded_rows(d, p, ldy, d_out)
    before = behind(bits, p)
    lordba.set_variant(lordba.VARIANT_TC)
    code = lordba.BF16 if p.dtype == "bf16" else lordba.F16
    assert lordba.query_variant([d.proj()], T, code) == [lordba.VARIANT_TC]
    lordba.adapter_forward_batched([d.proj()], T, code)          # takes the pitch also where there is one row
    assert lordba.device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(behind(bits, p), before))
    assert_close(torch_to_f64(d.y), oracle_forward(oracle, p), p.dtype, "padded rows")


def test_the_kernel_that_auto_takes_leaves_what_is_behind_the_rows(oracle):
    p = workloads.make_projection(512, 1001, 16, 300, "bf16", seed=7)
    d = DeviceProj(p)
    bits = in_padded_rows(d, p, 1008, 8)
    before = behind(bits, p)
    lordba.set_variant(lordba.VARIANT_AUTO)
    assert lordba.query_variant([d.proj()], 300, lordba.BF16) == [lordba.VARIANT_TC]
    d.forward()
    assert lordba.device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(behind(bits, p), before))
    assert_close(torch_to_f64(d.y), oracle_forward(oracle, p), "bf16", "padded rows, auto")


@pytest.mark.parametrize("T", [150, 2400])
def test_two_envelopes_in_a_batch_leave_what_is_behind_the_rows(oracle, T):
    projs, wants, kept = [], [], []
    for i, (d_out, ell, ldy) in enumerate([(252, 2, 256), (1001, 1, 1008), (130, 1, 136)]):
        p = workloads.make_projection(512, d_out, 16, T, "bf16", seed=50 + i)
        d = DeviceProj(p)
        rng = np.random.default_rng(i)
        s = [np.stack([v] + [v * np.exp(rng.normal(0, 0.3, v.shape)).astype(np.float32) for _ in range(ell - 1)]) for v in (p.s_in, p.s_r, p.s_out)]
        t = [torch.from_numpy(v if ell > 1 else v[0]).cuda() for v in s]
        bits = in_padded_rows(d, p, ldy, i)
        kept.append((d, t, bits, behind(bits, p)))
        projs.append(lordba.make_proj(d.x, d.packed_A, d.packed_B, t[0], t[1], t[2], d.y, p.r))
        wants.append(oracle.adapter_forward_ell(p.x_f64(), p.A_sign, p.B_sign, *(v.astype(np.float64) for v in s), p.y_f64()))
    lordba.set_variant(lordba.VARIANT_TC)
    assert set(lordba.query_variant(projs, T, lordba.BF16)) == {lordba.VARIANT_TC}
    lordba.adapter_forward_batched(projs, T, lordba.BF16)
    assert lordba.device_status() == 0
    for (d, _, bits, before), want in zip(kept, wants):
        assert all(torch.equal(a, b) for a, b in zip(behind(bits, d.p), before))
        assert_close(torch_to_f64(d.y), want, "bf16", "batch, d_out %d" % d.p.d_out)


def test_neighbours_in_one_buffer(oracle):
    """Two outputs whose rows lie side by side, seven elements of somebody else's between them, one call after the other."""
    T = 300
    bits = torch.from_numpy(np.random.default_rng(1).integers(-32768, 32768, (T, 1008 + 136), dtype=np.int16)).cuda()
    lordba.set_variant(lordba.VARIANT_TC)
    between = bits[:, 1001:1008].clone(), bits[:, 1138:].clone()
    for d_out, first in ((130, 1008), (1001, 0)):
        p = workloads.make_projection(512, d_out, 16, T, "bf16", seed=d_out)
        d = DeviceProj(p)
        place = bits.view(torch.bfloat16)[:, first:first + d_out]
        place.copy_(d.y)
        d.y = place
        d.forward()
        if first:
            neighbour = place.clone()
        assert_close(torch_to_f64(d.y), oracle_forward(oracle, p), "bf16", "columns %d ..." % first)
    assert lordba.device_status() == 0
    assert torch.equal(bits.view(torch.bfloat16)[:, 1008:1138], neighbour)
    assert torch.equal(bits[:, 1001:1008], between[0]) and torch.equal(bits[:, 1138:], between[1])
