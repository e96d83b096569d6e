"""Long rows: sums of squares of up to 2^28 values, against the 64-bit checker and exact values."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import binding
    return binding


# A row of one value: every addition of a lane's sum is rounded the same way for as long as the sum stays between two powers of two, so
# nothing averages out.  The sum of squares: eight products of a unit in two chains of four and their sum, 5 roundings; a lane's units,
# 2 whatever their number; 5 steps over lanes, 32 warps, the mean's two: 44 in all, halved by the root.  The root's two units (four
# roundings), eps, two products: 29; h itself is exact.
NORM = (44 / 2 + 4 + 1 + 2) * U


@pytest.mark.parametrize("value", [1.39, 1.0, 0.0123, 7.77, 1.0009765625])
@pytest.mark.parametrize("k", [1 << 23, (1 << 25) + 4099])
def test_norm_of_long_constant_rows(gl, k, value):
    ap = gl.AccessPattern
    x = torch.full((2, k), value, device="cuda")
    x[1] = -x[1]
    v = x[0, 0].double().item()
    want = v / np.sqrt(v * v + float(np.float32(1e-6)))
    out = gl.gl_compute_norm_rms(ap(x, 1), None, 1e-6).tensor
    for row, sign in ((0, 1.0), (1, -1.0)):
        assert ((out[row].double() * sign - want).abs() <= NORM * want).all(), (out[row, 0].item() * sign / want - 1) / U
    q = gl.gl_f8_dequantize(gl.gl_compute_norm_rms_f8(ap(x, 1), None, 1e-6)).tensor
    assert torch.equal(q, gl.gl_f8_dequantize(gl.gl_f8_quantize(ap(out, 1))).tensor)
