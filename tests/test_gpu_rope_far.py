"""The rotation at positions of any size: angles taken off in whole turns by exact arithmetic here.  Tolerances as in test_gpu_rope (a sine is
good to 2^-21 wherever the position is)."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2605_24058_b200 import lordba
from test_gpu_block import TYPES, f64
from test_gpu_rope import check

pytestmark = pytest.mark.gpu

PI = Fraction(31415926535897932384626433832795028841971693993751058209749445923078164062862092, 10 ** 79)
POSITIONS = [0, 1, -1, 12345, -131072, (1 << 31) + 5, (1 << 32) - 1, 1 << 32, (1 << 32) + 1, -(1 << 32), -(1 << 32) - 1, 1 << 40, -(1 << 40) - 77, (1 << 45) + 3, (1 << 53) + 1,
             -(1 << 53) - 1, (1 << 62) + 987654321, (1 << 63) - 1, -(1 << 63)]


def angles(inv_freq):
    """Of every position and frequency, within a turn, in float64."""
    out = np.empty((len(POSITIONS), len(inv_freq)))
    for i, p in enumerate(POSITIONS):
        for j, f in enumerate(inv_freq):
            turns = p * Fraction(float(f)) / (2 * PI)
            out[i, j] = float((turns - round(turns)) * 2 * PI)
    return out


@pytest.mark.parametrize("d,R,interleaved,pad", [(64, 64, False, 0), (128, 128, True, 0), (128, 128, False, 5), (80, 40, False, 0), (33, 32, True, 3)])
@pytest.mark.parametrize("base", [1.0, 15.9])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_any_position(d, R, interleaved, pad, base, dtype):
    rng = np.random.default_rng(d)
    inv = (base * 10000.0 ** (-np.arange(0, R, 2) / R)).astype(np.float32)
    T, H = len(POSITIONS), 3
    buf = torch.from_numpy(rng.standard_normal((T, H * d + pad)).astype(np.float32)).to(TYPES[dtype]).cuda()
    q = buf[:, :H * d].unflatten(1, (H, d))
    v, a = f64(q), angles(inv)[:, None]
    c, s = np.cos(a), np.sin(a)
    first, second = (np.arange(0, R, 2), np.arange(1, R, 2)) if interleaved else (np.arange(R // 2), np.arange(R // 2, R))
    pos, freq = torch.tensor(POSITIONS, device="cuda"), torch.from_numpy(inv).cuda()
    E = (d + 64) * 2.0 ** -23
    for sign, got in ((1, lordba.norm_rope(q, None, pos, freq, norm=False, interleaved=interleaved)[0]),
                      (-1, lordba.norm_rope_backward(q, None, q, None, pos, freq, norm=False, interleaved=interleaved)[0])):
        want, size = v.copy(), np.abs(v)
        want[..., first], want[..., second] = v[..., first] * c - sign * v[..., second] * s, v[..., second] * c + sign * v[..., first] * s
        size[..., first] = size[..., second] = np.abs(v[..., first]) + np.abs(v[..., second])
        check(got, want, E * size, dtype, "turned by %d" % sign)
