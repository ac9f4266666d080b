"""Clipping of gradients near the largest fp32 values: the factor by which they are multiplied is below fp32's normal numbers, or below all of them, though the clipped values are not.

Tolerances as for other values (test_gpu_grad_clip.py): the product is rounded once, and once more only where the value itself is below the normal numbers (2^-149)."""
import numpy as np
import pytest

from test_gpu_grad_clip import F16, F32, HALF, SINGLE, check

pytestmark = pytest.mark.gpu

FAR = [  # values, how many of each, inv_scale, max_norm
    ((3e38,), 1, 1.0, 1e-7),                            # factor 3e-46
    ((3e38, -1e38, 1e30, 0.0, 1e-30), 1, 1.0, 1e-3),    # 3e-42
    ((1e38, -2e37), 500000, 2.0 ** -16, 1.0),           # 1e-41
    ((3.4e38, 3e38), 3, 2.0 ** -20, 2.0 ** -100),       # 1e-69
    ((3e38, 2.0 ** 100), 70, 2.0 ** -16, 2.0 ** -149),  # 2e-85, what comes out is below the normal numbers or zero
    ((1e38, 1.0), 9, 2.0 ** -126, 1.0),                 # unscaled alone, by the least normal number
    ((1e38, 1.0), 9, 1e-42, float("inf")),              # and by less
    ((1e30,), 100, 2.0 ** -60, 0.0),
]


@pytest.mark.parametrize("values,each,inv_scale,max_norm", FAR)
def test_factors_below_the_normal_numbers(hgnn, dev, values, each, inv_scale, max_norm):
    print(f"clip of {values} x {each}, inv_scale {inv_scale}, max_norm {max_norm}", flush=True)
    inv_scale, max_norm = float(F32(inv_scale)), float(F32(max_norm))  # what the call takes
    a = [np.repeat(np.array(values, F32), each), np.array([65504, 1, 0], F16)]
    check(hgnn, dev, a, None, inv_scale, max_norm)
    check(hgnn, dev, a, [SINGLE, SINGLE], inv_scale, max_norm)
    check(hgnn, dev, a, [HALF, HALF], inv_scale, max_norm)
    m = np.tile(np.array(values, F32), (11, 1))
    check(hgnn, dev, [m], [SINGLE], inv_scale, max_norm, pitches=[len(values) + 3], offsets=[1])
