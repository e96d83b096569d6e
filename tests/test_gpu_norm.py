"""The root-mean-square norm with its residual, against the 64-bit checker."""
import numpy as np
import pytest
import torch

from oracle import f8
from paper_2105_09377_b200 import synth

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
EPS = {BF: 2.0 ** -8, F32: 2.0 ** -24}


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import binding
    return binding


def _device(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(dtype)


def _np(t):
    return t.double().cpu().numpy()


def _inputs(rows, k, dtype, res, wtype):
    x = _device(synth.normal(21, rows * 7 + k, (rows, k)) * np.exp(synth.normal(22, rows, (rows, 1))), dtype)
    r = None if res is None else _device(synth.normal(23, rows * 7 + k, (rows, k), 2.0), res)
    w = None if wtype is None else _device(1 + synth.normal(24, k, (k,), 0.2), wtype)
    return x, r, w


def _check(gl, rows, k, dtype, res, wtype, out_type, eps=1e-5):
    x, r, w = _inputs(rows, k, dtype, res, wtype)
    ap = gl.AccessPattern
    total = None if res is None else ap(torch.full((rows, k), 3.0, dtype=res, device="cuda"), 1)
    out = gl.f8_empty((rows, k), 1, "cuda") if out_type == "f8" else ap(torch.empty((rows, k), dtype=out_type, device="cuda"), 1)
    opt = lambda t, n: None if t is None else ap(t, n)
    gl.gl_compute_norm_rms(ap(x, 1), opt(w, 0), eps, opt(r, 1), total, out)
    h, y = f8.norm_rms(_np(x), None if r is None else _np(r), None if w is None else _np(w), eps)
    if res is not None:
        # h is one fp32 sum: exact to 2^-24 of itself, then half a unit of its type
        assert (np.abs(_np(total.tensor) - h) <= (EPS[res] + 2.0 ** -24) * np.abs(h) * (1 + 2.0 ** -8)).all()
    # sum of squares: up to 32 products in a lane, 5 steps over lanes, 32 warps: 69 roundings, half of it after the root; the
    # mean, eps, the reciprocal root (two units, four roundings) and three products: 12 more at most; h itself 1
    tol = (69 / 2 + 12 + 1) * 2.0 ** -24 * np.abs(y)
    if out_type == "f8":
        plain = gl.gl_compute_norm_rms(ap(x, 1), opt(w, 0), eps, opt(r, 1), None, ap(torch.empty((rows, k), device="cuda"), 1))
        both = gl.gl_f8_quantize(plain)        # the same values rounded by the operator that the format belongs to
        nb, pitch = -(-k // 128), -(-k // 16) * 16
        at = torch.from_numpy(f8.scale_at(rows, nb)).cuda()
        assert torch.equal(out.data[: rows * pitch], both.data[: rows * pitch]) and torch.equal(out.scale[at], both.scale[at])
        out = plain
        out_type = F32
    err = np.abs(_np(out.tensor) - y)
    assert (err <= tol + EPS[out_type] * (np.abs(y) + tol)).all(), (err / np.maximum(np.abs(y), 1e-30)).max()


@pytest.mark.parametrize("out_type", [BF, F32, "f8"])
@pytest.mark.parametrize("rows,k", [(1, 1), (3, 7), (1, 8), (2, 128), (9, 200), (5, 255), (70, 256), (1, 264), (300, 1111), (260, 1024),
                                    (1, 2048), (3, 2056), (400, 4096), (2, 8191), (1, 8192), (170, 8192), (160, 9000)])
def test_sizes(gl, rows, k, out_type):
    _check(gl, rows, k, BF, BF, BF, out_type)
    _check(gl, rows, k, F32, None, F32, out_type)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("res", [None, BF, F32])
@pytest.mark.parametrize("wtype", [None, BF, F32])
@pytest.mark.parametrize("out_type", [BF, F32, "f8"])
def test_types(gl, dtype, res, wtype, out_type):
    _check(gl, 5, 1000, dtype, res, wtype, out_type)
    _check(gl, 5, 333, dtype, res, wtype, out_type, eps=0.0)


@pytest.mark.parametrize("rows,k", [(2, 16400), (200, 16384), (3, 33001), (2, 40000), (1, 1 << 20)])
def test_long_rows(gl, rows, k):
    """Rows of more units than a block keeps in registers (and the last that it does keep).  A lane adds up to 2^20 / 8192 units of
    eight: 136 roundings instead of 32 in the derivation above, which its 1 / sqrt halves: 52 more."""
    x, r, w = _inputs(rows, k, BF, F32, F32)
    ap = gl.AccessPattern
    total = ap(torch.empty((rows, k), device="cuda"), 1)
    out = gl.gl_compute_norm_rms(ap(x, 1), ap(w, 0), 1e-5, ap(r, 1), total, ap(torch.empty((rows, k), device="cuda"), 1))
    h, y = f8.norm_rms(_np(x), _np(r), _np(w), 1e-5)
    assert (np.abs(_np(total.tensor) - h) <= 2.0 ** -24 * np.abs(h)).all()
    assert (np.abs(_np(out.tensor) - y) <= 102 * 2.0 ** -24 * np.abs(y)).all()
    q = gl.gl_compute_norm_rms_f8(ap(x, 1), ap(w, 0), 1e-5, ap(r, 1))
    assert torch.equal(gl.gl_f8_dequantize(q).tensor, gl.gl_f8_dequantize(gl.gl_f8_quantize(out)).tensor)


@pytest.mark.parametrize("rows,k", [(70, 128), (40000, 24), (76003, 128), (3, 1000), (200, 1111), (2, 8192), (300, 4096), (2, 33001), (1, 40000)])
def test_in_place(gl, rows, k):
    """The sum takes the residual's place, or x's; the result takes x's."""
    ap = gl.AccessPattern
    for dtype in (BF, F32):
        x, r, w = _inputs(rows, k, dtype, dtype, BF)
        want_sum, want = ap(torch.empty_like(r), 1), ap(torch.empty_like(x), 1)
        gl.gl_compute_norm_rms(ap(x, 1), ap(w, 0), 1e-5, ap(r, 1), want_sum, want)
        x1, r1 = x.clone(), r.clone()
        gl.gl_compute_norm_rms(ap(x1, 1), ap(w, 0), 1e-5, ap(r1, 1), ap(r1, 1), ap(x1, 1))
        assert torch.equal(r1, want_sum.tensor) and torch.equal(x1, want.tensor)
        x2, r2 = x.clone(), r.clone()
        gl.gl_compute_norm_rms(ap(x2, 1), ap(w, 0), 1e-5, ap(r2, 1), ap(x2, 1), ap(r2, 1))
        assert torch.equal(x2, want_sum.tensor) and torch.equal(r2, want.tensor)


def test_values_at_the_ends(gl):
    """Rows of zeros, of tiny and large values; a NaN or an Inf stays in its row."""
    ap = gl.AccessPattern
    x = torch.randn(6, 500, device="cuda")
    x[0] = 0
    x[1] *= 1e-20
    x[2] *= 1e15
    x[3, 499] = float("nan")
    x[4, 0] = float("inf")
    out = gl.gl_compute_norm_rms(ap(x, 1), None, 1e-6).tensor
    assert (out[0] == 0).all() and torch.isnan(out[3]).all()
    assert torch.isnan(out[4, 0]) and (out[4, 1:] == 0).all()
    _, y = f8.norm_rms(_np(x[[0, 1, 2, 5]]), None, None, 1e-6)
    assert (np.abs(_np(out[[0, 1, 2, 5]]) - y) <= 64 * 2.0 ** -24 * np.abs(y)).all()
    q = gl.gl_f8_dequantize(gl.gl_compute_norm_rms_f8(ap(x, 1), None, 1e-6)).tensor
    assert (q[0] == 0).all() and torch.isnan(q[3]).all() and torch.isnan(q[4, :128]).all() and (q[4, 128:] == 0).all()
    assert torch.isnan(gl.gl_compute_norm_rms(ap(x[:1], 1), None, 0.0).tensor).all()         # 0 / 0


@pytest.mark.parametrize("out_type", [BF, F32, "f8"])
@pytest.mark.parametrize("rows,k", [(1, 16), (5, 24), (31, 8), (1000, 120), (4097, 64), (80001, 128), (999, 40), (300001, 8), (90000, 72),
                                    (310003, 32)])
def test_short_rows(gl, rows, k, out_type):
    """Several rows side by side in a warp: heads, in every number of lanes, one or four groups a warp."""
    _check(gl, rows, k, BF, None, BF, out_type)
    _check(gl, rows, k, F32, BF, None, out_type)
    _check(gl, rows, k, BF, F32, F32, out_type)


@pytest.mark.parametrize("rows,k,wtype", [(1100, 8192, BF), (4300, 2048, F32), (2100, 4096, None), (300, 32768, BF)])
def test_rows_held_as_they_came(gl, rows, k, wtype):
    """bf16 rows without a residual into F8, eight units a warp: the same codes as of the fp32 result; rows of 128 units and one more."""
    _check(gl, rows, k, BF, None, wtype, "f8")
    _check(gl, 40, k + 256, BF, None, wtype, "f8")


def test_items_of_several_dimensions_and_guard_bands(gl):
    ap = gl.AccessPattern
    shape = (3, 5, 7, 11)
    x, r = torch.randn(shape, device="cuda").to(BF), torch.randn(shape, device="cuda")
    w = torch.randn(7, 11, device="cuda")
    n = 3 * 5 * 77
    stores = [torch.full((n + 512,), 7.0, dtype=t, device="cuda") for t in (F32, BF)]
    total, out = (ap(s[256:256 + n].view(shape), 2) for s in stores)
    gl.gl_compute_norm_rms(ap(x, 2), ap(w, 0), 1e-5, ap(r, 2), total, out)
    h, y = f8.norm_rms(_np(x).reshape(15, 77), _np(r).reshape(15, 77), _np(w).reshape(77), 1e-5)
    assert (np.abs(_np(out.tensor).reshape(15, 77) - y) <= (2.0 ** -8 + 2.0 ** -17) * np.abs(y)).all()
    for s in stores:
        assert (s[:256] == 7).all() and (s[256 + n:] == 7).all()


def test_rows_do_not_depend_on_the_batch(gl):
    """A row's result is the same bits whatever else the call holds, as long as the same kernel takes it; and on every repetition."""
    ap = gl.AccessPattern
    x = torch.randn(700, 2048, device="cuda").to(BF)
    a, b = (gl.gl_compute_norm_rms(ap(x, 1)).tensor for _ in range(2))
    assert torch.equal(a, b) and torch.equal(gl.gl_compute_norm_rms(ap(x[100:600], 1)).tensor, a[100:600])


def test_graph_and_stream(gl):
    ap = gl.AccessPattern
    x, r, w = _inputs(20, 1024, BF, BF, BF)
    total, q = ap(torch.empty_like(r), 1), gl.f8_empty((20, 1024), 1, "cuda")
    call = gl.prepare_compute_norm_rms(ap(x, 1), ap(w, 0), q, 1e-5, ap(r, 1), total)
    call()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3):
        x.copy_(torch.randn(20, 1024, generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        mine = gl.gl_compute_norm_rms_f8(ap(x, 1), ap(w, 0), 1e-5, ap(r, 1), stream=side)
        torch.cuda.synchronize()
        assert torch.equal(gl.gl_f8_dequantize(q).tensor, gl.gl_f8_dequantize(mine).tensor)


def test_beyond_two_to_the_31_values(gl):
    ap = gl.AccessPattern
    rows, k = 270000, 8192
    x = torch.ones((rows, k), dtype=BF, device="cuda")
    x[-2:] = torch.randn((2, k), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    want = gl.gl_compute_norm_rms(ap(x[-2:].clone(), 1), None, 0.0, ap(x[-2:].clone(), 1), None, ap(torch.empty((2, k), dtype=BF, device="cuda"), 1)).tensor
    ends = x[-2:] + x[-2:]
    gl.gl_compute_norm_rms(ap(x, 1), None, 0.0, ap(x, 1), ap(x, 1), q := gl.f8_empty((rows, k), 1, "cuda"))
    assert (x[:-2] == 2).all() and torch.equal(x[-2:], ends)
    back = gl.gl_f8_dequantize(q, ap(x, 1)).tensor
    assert (back[:-2] == 1).all() and ((back[-2:].double() - want.double()).abs() <= (2.0 ** -4 + 2.0 ** -7) * want.double().abs() + 2.0 ** -9).all()   # (want is bf16)
