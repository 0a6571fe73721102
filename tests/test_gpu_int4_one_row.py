"""One token of any width through a 4-bit product and back is one launch, and right.  Bounds as in test_gpu_int4."""
import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import clean, close, f64
from test_gpu_int4 import Weights, product_bound

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d_in,d_out", [(1, 1), (7, 9), (129, 131), (1001, 1533), (4090, 333), (200, 201)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("far", [0, 1 << 22])
def test_one_row(d_in, d_out, dtype, far):
    rng = np.random.default_rng(d_in)
    w = Weights(rng, d_out, d_in, 32, True, dtype)
    for back in (False, True):
        n = d_out if back else d_in
        row = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).to(w.scale.dtype).cuda()
        x = row.as_strided((1, n), (n + far, 1))                  # a pitch that no row uses
        before = lordba.launch_count()
        y = lordba.int4_linear_backward(x, w.q, w.scale, d_in, **w.args()) if back else lordba.int4_linear(x, w.q, w.scale, **w.args())
        assert lordba.launch_count() == before + 1
        v = w.v if back else w.v.T
        close(y, f64(x) @ v, product_bound(f64(x), v, dtype), dtype, "dx" if back else "y")
    clean()
