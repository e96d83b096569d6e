"""GPU parity of the 4-bit operands: quantisation bit for bit, products against 64 bits."""
import numpy as np
import pytest
import torch

from oracle import mx4
from paper_2105_09377_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import binding
    return binding


def _to_bf16(x):
    """Rounded to eight significant bits, ties to even (float64 in and out)."""
    m, e = np.frexp(x)
    return np.ldexp(np.round(m * 256.0), e - 8)


def _within(got, ref, tol, bf16):
    """|result before the last rounding - ref| <= tol, as far as the rounded result can show it: rounding is monotonic."""
    lo, hi = ref - tol, ref + tol
    return (got >= (_to_bf16(lo) if bf16 else lo)) & (got <= (_to_bf16(hi) if bf16 else hi))


def _unpack(m, rows, k):
    """(codes, exponents) of an Mx4 in the checker's form, read by the documented storage order."""
    nb, kt = -(-k // 32), -(-k // 128)
    d = m.data.cpu().numpy().reshape(rows, nb * 16)
    codes = np.stack([d & 15, d >> 4], -1).reshape(rows, nb, 32)
    s = m.scale.cpu().numpy().reshape(-(-rows // 128), kt, 32, 4, 4)      # row tile, K tile, r % 32, r / 32, block
    s = s.transpose(0, 3, 2, 1, 4).reshape(-1, kt * 4)[:rows, :nb]
    return codes, s


def _wide(shape, seed, dtype):
    """Values over many binades, zeros, exact ties and blocks of nothing."""
    x = synth.normal(seed, 1, shape) * np.exp2(np.round(synth.uniform(seed, 2, shape[:1] + (1,), -20.0, 20.0)))
    x = np.where(synth.uniform(seed, 3, shape, 0.0, 1.0) < 0.2, np.round(x * 4) / 4, x)
    x[:, 64:96] = 0.0
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()
    return t.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,k", [(1, 1), (1, 31), (2, 32), (3, 33), (5, 128), (130, 100), (257, 1111), (33, 1024), (64, 136),
                                    (1, 4097), (2500, 2000)])
def test_quantize_bit_for_bit(gl, rows, k, dtype):
    x = _wide((rows, k), rows * 7 + k, dtype)
    out = gl.mx4_empty((rows, k), 1, "cuda")
    out.data.fill_(0xEE)
    gl.gl_mx4_quantize(gl.AccessPattern(x, 1), out)
    codes, exps = mx4.quantize(x.float().cpu().numpy())
    got_codes, got_exps = _unpack(out, rows, k)
    assert np.array_equal(got_exps, exps) and np.array_equal(got_codes, codes)
    for back in (torch.float32, torch.bfloat16):
        y = gl.gl_mx4_dequantize(out, gl.AccessPattern(torch.full((rows, k), 7.0, dtype=back, device="cuda"), 1)).tensor
        assert np.array_equal(y.double().cpu().numpy(), mx4.values(codes, exps, k))


def test_quantize_extremes(gl):
    x = torch.zeros(6, 96)
    x[0, 5], x[1, 40], x[2, 70] = float("nan"), float("inf"), float("-inf")
    x[3, :3] = torch.tensor([3.3e38, -1e38, 1e-38])
    x[4, :3] = torch.tensor([1e-45, -2e-39, 1.2e-38])
    x[5, 33] = -0.0
    m = gl.gl_mx4_quantize(gl.AccessPattern(x.cuda(), 1))
    codes, exps = mx4.quantize(x.numpy())
    got_codes, got_exps = _unpack(m, 6, 96)
    assert np.array_equal(got_exps, exps)
    assert np.array_equal(got_codes[exps != 255], codes[exps != 255])
    y = gl.gl_mx4_dequantize(m).tensor.cpu().double().numpy()
    np.testing.assert_array_equal(y, mx4.values(codes, exps, 96))


def test_quantize_items_of_several_dims(gl):
    x = synth.normal(3, 1, (4, 5, 3, 7)).astype(np.float32)
    m = gl.gl_mx4_quantize(gl.AccessPattern(torch.from_numpy(x).cuda(), 2))
    assert m.shape == ((4, 5), (3, 7))
    codes, exps = _unpack(m, 20, 21)
    want = mx4.quantize(x.reshape(20, 21))
    assert np.array_equal(codes, want[0]) and np.array_equal(exps, want[1])


PRODUCTS = [(1, 32, 1), (1, 4096, 1000), (2, 64, 9), (7, 1, 5), (16, 3136, 1000), (33, 96, 130), (128, 256, 128), (129, 257, 127),
            (17, 8192, 264), (301, 1111, 777), (256, 512, 384), (64, 130, 2049), (300, 640, 512), (513, 2048, 260),
            (2049, 320, 4200), (2300, 700, 2311), (100, 5000, 650), (9, 20000, 70),
            (1, 1000, 9000), (3, 33000, 40), (4, 2049, 129)]


@pytest.mark.parametrize("form", ["product", "dense"])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("m,k,o", PRODUCTS)
def test_products(gl, m, k, o, bf16, form):
    relu = (m + o) % 2 == 1
    x = torch.from_numpy(synth.normal(11, 1, (m, k)).astype(np.float32)).cuda().to(torch.bfloat16)
    w = torch.from_numpy(synth.normal(12, 2, (o, k)).astype(np.float32)).cuda().to(torch.bfloat16)
    flags = (gl.GL_EPILOGUE_RELU if relu else 0) | (gl.GL_OUT_BF16 if bf16 else 0)
    xa, wq = gl.AccessPattern(x, 1), gl.gl_mx4_quantize(gl.AccessPattern(w, 1))
    guard = torch.full((m * o + 256,), 3.0, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    out = gl.AccessPattern(guard[128:128 + m * o].view(m, o), 2)
    if form == "dense":
        gl.gl_dense_mx4(xa, wq, out, flags)
    else:
        gl.gl_cartesian_dot_mx4(gl.gl_mx4_quantize(xa), wq, out, flags)
    a, b = mx4.rounded(x.double().cpu().numpy()), mx4.rounded(w.double().cpu().numpy())
    ref = a @ b.T
    # Products of two-bit significands are exact; K/32 partial sums of at most sum |a b| are each rounded (or cut) to
    # 24 bits; a bf16 result is rounded once more.
    tol = (k / 32 + 2) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)
    if relu:
        ref = np.maximum(ref, 0.0)     # (moves no two values further apart)
    got = out.tensor.double().cpu().numpy()
    assert _within(got, ref, tol, bf16).all(), float((np.abs(got - ref) - tol).max())
    assert (guard[:128] == 3.0).all() and (guard[128 + m * o:] == 3.0).all()
    assert gl.gl_poll_device_status() == 0


@pytest.mark.parametrize("m", [1, 8, 40, 200])
def test_scales_of_many_binades_and_rows_repeat(gl, m):
    """Every row and column with scales of its own; the result of a row does not depend on its neighbours."""
    k, o = 640, 300
    x = synth.normal(21, 1, (m, k)) * np.exp2(np.round(synth.uniform(21, 2, (m, k // 32), -8, 8))).repeat(32, 1)
    w = synth.normal(22, 1, (o, k)) * np.exp2(np.round(synth.uniform(22, 2, (o, k // 32), -8, 8))).repeat(32, 1)
    x, w = (torch.from_numpy(t.astype(np.float32)).cuda() for t in (x, w))
    wq = gl.gl_mx4_quantize(gl.AccessPattern(w, 1))
    got = gl.gl_dense_mx4(gl.AccessPattern(x, 1), wq).tensor
    a, b = mx4.rounded(x.double().cpu().numpy()), mx4.rounded(w.double().cpu().numpy())
    assert (np.abs(got.double().cpu().numpy() - a @ b.T) <= (k / 32 + 2) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)).all()
    assert torch.equal(got, gl.gl_dense_mx4(gl.AccessPattern(x, 1), wq).tensor)


@pytest.mark.parametrize("m", [3, 140])
def test_nan_stays_in_its_row(gl, m):
    x = torch.from_numpy(synth.normal(31, 1, (m, 300)).astype(np.float32)).cuda()
    w = torch.from_numpy(synth.normal(32, 1, (260, 300)).astype(np.float32)).cuda()
    x[1, 70] = float("inf")
    w[258, 299] = float("nan")
    out = gl.gl_dense_mx4(gl.AccessPattern(x, 1), gl.gl_mx4_quantize(gl.AccessPattern(w, 1)), flags=gl.GL_EPILOGUE_RELU).tensor.cpu()
    nan = torch.isnan(out)
    assert nan[1].all() and nan[:, 258].all()
    nan[1], nan[:, 258] = False, False
    assert not nan.any()


def test_items_of_several_dims_on_another_stream(gl):
    x = torch.from_numpy(synth.normal(41, 1, (2, 3, 5, 8)).astype(np.float32)).cuda().bfloat16()
    w = torch.from_numpy(synth.normal(42, 1, (4, 6, 5, 8)).astype(np.float32)).cuda().bfloat16()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    wq = gl.gl_mx4_quantize(gl.AccessPattern(w, 2), stream=side)
    with torch.cuda.stream(side):
        out = gl.gl_dense_mx4(gl.AccessPattern(x, 2), wq)
    side.synchronize()
    assert out.shape == ((2, 3, 4, 6), ())
    a, b = mx4.rounded(x.double().cpu().numpy().reshape(6, 40)), mx4.rounded(w.double().cpu().numpy().reshape(24, 40))
    assert (np.abs(out.tensor.double().cpu().numpy().reshape(6, 24) - a @ b.T) <= 4 * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)).all()


def test_prepared_calls_in_a_graph(gl):
    x = torch.zeros(5, 256, dtype=torch.bfloat16, device="cuda")
    w = torch.from_numpy(synth.normal(52, 1, (64, 256)).astype(np.float32)).cuda()
    wq = gl.gl_mx4_quantize(gl.AccessPattern(w, 1))
    out = gl.AccessPattern(torch.zeros(5, 64, device="cuda"), 2)
    call = gl.prepare_dense_mx4(gl.AccessPattern(x, 1), wq, out)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    x.copy_(torch.from_numpy(synth.normal(51, 1, (5, 256)).astype(np.float32)))
    graph.replay()
    want = gl.gl_dense_mx4(gl.AccessPattern(x, 1), wq).tensor
    assert torch.equal(out.tensor, want) and want.abs().sum() > 0
