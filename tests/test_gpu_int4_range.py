"""4-bit products near the end of float16's range, and what stands in the carrier behind the last column: it is not looked at, so
a weight that it would make, beyond what float16 holds, spoils nothing.  Bounds as in test_gpu_int4."""
import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import clean, close, f64
from test_gpu_int4 import carrier_bytes, product_bound

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d_in,group", [(200, 128), (200, 32), (129, 64), (135, 256), (1001, 64), (65, 32)])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("T", [1, 20, 33, 64, 200, 300])
def test_columns_behind_the_last_make_no_weights(T, d_in, group, zeros):
    rng = np.random.default_rng(d_in + T)
    d_out, g = 150, -(-d_in // group)
    middle = 12 if zeros else 8
    u = rng.integers(middle - 2, middle + 3, (d_out, d_in)).astype(np.uint8)                 # weights up to 18000
    scale = torch.from_numpy(rng.uniform(8500, 9000, (d_out, g)).astype(np.float32)).half().cuda()
    zero = torch.full((d_out, g), middle, dtype=torch.uint8, device="cuda") if zeros else None
    q = lordba.int4_pack(torch.from_numpy(u).cuda())                                        # zeros behind: -68000 and less
    x = torch.from_numpy((rng.standard_normal((T, d_in)) * 2.0 ** -8).astype(np.float32)).half().cuda()
    w = np.repeat(f64(scale), group, axis=1)[:, :d_in] * (u - float(middle))
    y = lordba.int4_linear(x, q, scale, zero, group)
    close(y, f64(x) @ w.T, product_bound(f64(x), w.T, "f16"), "f16", "y")
    blocks = q.shape[1] * 2
    rest = torch.from_numpy(carrier_bytes(np.pad(np.zeros((1, d_in), np.uint8), ((0, 0), (0, blocks - d_in)), constant_values=15))).cuda()
    assert torch.equal(lordba.int4_linear(x, q | rest, scale, zero, group), y)
    dy = torch.from_numpy((rng.standard_normal((T, d_out)) * 2.0 ** -8).astype(np.float32)).half().cuda()
    dx = lordba.int4_linear_backward(dy, q, scale, d_in, zero, group)
    close(dx, f64(dy) @ w, product_bound(f64(dy), w, "f16"), "f16", "dx")
    clean()
