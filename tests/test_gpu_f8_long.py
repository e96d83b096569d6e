"""Long rows: sums of squares and products of up to 2^28 values, against exact values."""
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
@pytest.mark.parametrize("k", [1 << 23, (1 << 25) + 4099, 1 << 28])
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


# ---- products of more values than one accumulator adds up ----

STRETCH = 65536


def _lost(k):
    """What sums of k products may be off by, relative to the sum of their magnitudes.  An instruction adds 32 products to an
    accumulator: each is cut to 2^-25 of the largest term and the sum to fp32, 32 * 2^-25 + 2^-23 = 9 * 2^-23 of the magnitudes so
    far, for at most 65536 values; these stretches and the ranks of a cluster are added with rounding to nearest."""
    return min(k, STRETCH) * 9 * 2.0 ** -28 + (k / STRETCH + 8) * U


def _rows(base, rows):
    """`base` [K] times 2^0, 2^1, 2^2, 2^-1, ..: every row's codes are those of the first."""
    factor = torch.tensor([2.0 ** (i % 5 - 1) for i in range(rows)], device="cuda")
    return base.to(BF)[None] * factor.to(BF)[:, None], factor.double()


# few rows in every width, several tiles of rows of A, tiles; K of one stretch, just beyond one, of many
@pytest.mark.parametrize("m,o", [(1, 40), (20, 130), (50, 64), (100, 200), (200, 300), (1500, 2000)])
@pytest.mark.parametrize("k", [STRETCH, STRETCH + 128, 3 * STRETCH + 17, (1 << 20) - 77, 1 << 22])
def test_small_products_behind_a_large_one(gl, m, o, k):
    """The first block brings the sum to 2^24.6; each product behind it is less than an accumulator of that size keeps."""
    if m * k > 1 << 31:
        m, o = 600, 4200                          # (tiles too, in less memory)
    ap = gl.AccessPattern
    a, b = torch.full((k,), 0.46875, device="cuda"), torch.ones(k, device="cuda")
    a[:128], b[:128] = 448.0, 448.0
    want = 448.0 * 448.0 * 128 + 0.46875 * (k - 128)
    (xa, fa), (xb, fb) = _rows(a, m), _rows(b, o)
    qb = gl.gl_f8_quantize(ap(xb, 1))
    del xb
    ref = want * fa[:, None] * fb[None]
    for flags, unit in ((0, 0.0), (gl.GL_OUT_BF16 | gl.GL_EPILOGUE_RELU, 2.0 ** -8)):
        out = gl.gl_dense_f8(ap(xa, 1), qb, flags=flags).tensor.double()
        assert ((out - ref).abs() <= (_lost(k) + unit * (1 + _lost(k))) * ref).all(), ((out - ref) / ref).abs().max().item()
    assert gl.gl_poll_device_status() == 0


@pytest.mark.parametrize("m,o", [(1, 300), (17, 129), (64, 40), (130, 200), (700, 3600)])
@pytest.mark.parametrize("k", [STRETCH + 1, 2 * STRETCH, 5 * STRETCH + 4000, (1 << 19) + 31, (1 << 20) + 515])
def test_long_whole_numbers_are_exact(gl, m, o, k):
    """Every sum of magnitudes is below 2^24, so nothing is cut or rounded: a stretch that is missing, or added twice, shows."""
    if m > 600 and k > 1 << 19:
        return                                    # (the reference alone takes seconds)
    ap = gl.AccessPattern
    g = torch.Generator("cuda").manual_seed(m + k)
    a, b = (torch.randint(-3, 4, (n, k), generator=g, dtype=torch.int8, device="cuda").to(BF) for n in (m, o))
    qa, qb = gl.gl_f8_quantize(ap(a, 1)), gl.gl_f8_quantize(ap(b, 1))
    want = torch.zeros((m, o), dtype=torch.float64, device="cuda")
    for at in range(0, k, 1 << 15):
        want += (a[:, at:at + (1 << 15)].float() @ b[:, at:at + (1 << 15)].float().t()).double()
    out = gl.gl_cartesian_dot_f8(qa, qb).tensor
    assert torch.equal(out.double(), want)
    relu = gl.gl_cartesian_dot_f8(qa, qb, flags=gl.GL_OUT_BF16 | gl.GL_EPILOGUE_RELU).tensor
    assert torch.equal(relu, want.clamp_min(0).to(BF)) and gl.gl_poll_device_status() == 0


@pytest.mark.parametrize("m,o", [(1, 1), (70, 2)])
def test_the_longest_products(gl, m, o):
    """2^28 values of an item, 4096 stretches; 2^24 of seventy."""
    k = 1 << (28 if m == 1 else 24)
    test_small_products_behind_a_large_one(gl, m, o, k)


def test_long_products_repeat(gl):
    ap = gl.AccessPattern
    for m, o in ((3, 500), (90, 500), (1500, 1500)):
        k = 200000
        a, b = (torch.randn((n, k), generator=torch.Generator("cuda").manual_seed(n), device="cuda") for n in (m, o))
        qa, qb = gl.gl_f8_quantize(ap(a, 1)), gl.gl_f8_quantize(ap(b, 1))
        once = gl.gl_cartesian_dot_f8(qa, qb).tensor
        assert all(torch.equal(gl.gl_cartesian_dot_f8(qa, qb).tensor, once) for _ in range(3))
        want = gl.gl_f8_dequantize(qa).tensor.double() @ gl.gl_f8_dequantize(qb).tensor.double().t()
        mag = gl.gl_f8_dequantize(qa).tensor.double().abs() @ gl.gl_f8_dequantize(qb).tensor.double().abs().t()
        assert ((once.double() - want).abs() <= _lost(k) * mag).all()
