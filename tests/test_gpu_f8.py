"""Operands held in 8 bits: rounding (bit for bit), reading back, products, against the 64-bit checker."""
import numpy as np
import pytest
import torch

from oracle import f8
from paper_2105_09377_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import binding
    return binding


def _device(x, dtype):
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()
    return t.to(dtype)


def _specials():
    """Rows of one block each: ends of the range, ties, zeros, infinities and NaN."""
    rows = []
    for top in (448.0, 449.0, 2.0 ** 120, 3.0e38, 2.0 ** -126, 2.0 ** -133, 2.0 ** -149, 1.75, np.nextafter(np.float32(1.75), np.float32(2)), 255.9):
        r = np.linspace(-1, 1, 128) * top
        r[0] = top
        rows.append(r)
    rows.append(np.zeros(128))
    rows.append(-np.zeros(128))
    ties = np.repeat(np.concatenate([f8.GRID[:126] + np.diff(f8.GRID) / 2, [448.0, 0.0]]), 1)
    rows.append(ties)
    rows.append(-ties)
    for bad in (np.inf, -np.inf, np.nan):
        r = np.ones(128)
        r[77] = bad
        rows.append(r)
    return np.asarray(rows, dtype=np.float32)


def _codes(q, rows, k):
    pitch = -(-k // 16) * 16
    nb = -(-k // 128)
    codes = q.data[: rows * pitch].cpu().numpy().reshape(rows, pitch)
    full = np.zeros((rows, nb * 128), dtype=np.uint8)
    full[:, : min(pitch, nb * 128)] = codes[:, : nb * 128]
    exps = q.scale.cpu().numpy()[f8.scale_at(rows, nb)]
    return full.reshape(rows, nb, 128), exps


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,k", [(1, 1), (1, 7), (3, 16), (5, 17), (2, 127), (2, 128), (129, 129), (7, 255), (3, 256), (4, 264),
                                    (260, 300), (33, 1111), (1, 8192), (300, 640), (130, 2056)])
def test_quantize_bit_for_bit(gl, rows, k, dtype):
    x = _device(synth.normal(3, rows * 10007 + k, (rows, k)) * np.exp(synth.normal(4, k, (rows, 1))), dtype)
    q = gl.f8_empty((rows, k), 1, "cuda")
    q.data.fill_(0xAB)
    gl.gl_f8_quantize(gl.AccessPattern(x, 1), q)
    want, we = f8.quantize(x.double().cpu().numpy())
    got, ge = _codes(q, rows, k)
    assert np.array_equal(ge, we) and np.array_equal(got, want)
    back = gl.gl_f8_dequantize(q).tensor
    ref = f8.values(want, we, k)
    assert np.array_equal(back.double().cpu().numpy(), ref)
    half = gl.gl_f8_dequantize(q, gl.AccessPattern(torch.empty((rows, k), dtype=torch.bfloat16, device="cuda"), 1)).tensor
    assert np.array_equal(half.double().cpu().numpy(), ref)


@pytest.mark.parametrize("rows,k", [(1, 8), (200, 24), (31, 40), (130, 64), (600, 72), (65, 120)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_short_rows(gl, rows, k, dtype):
    test_quantize_bit_for_bit(gl, rows, k, dtype)


def test_quantize_many_rows(gl):
    """Several units a warp: more rows than one pass over the SMs, a ragged end."""
    for rows, k, dtype in ((90001, 128, torch.bfloat16), (80003, 72, torch.float32), (300007, 8, torch.bfloat16), (2000, 120, torch.float32),
                           (20001, 264, torch.bfloat16), (9001, 263, torch.float32), (40003, 129, torch.bfloat16)):
        g = torch.Generator("cuda").manual_seed(rows)
        x = torch.randn((rows, k), generator=g, device="cuda").to(dtype)
        back = gl.gl_f8_dequantize(gl.gl_f8_quantize(gl.AccessPattern(x, 1)), gl.AccessPattern(torch.empty_like(x), 1)).tensor
        pick = np.r_[0:40, rows // 2:rows // 2 + 40, rows - 40:rows]
        assert np.array_equal(back[pick].double().cpu().numpy(), f8.rounded(x[pick].double().cpu().numpy()))
        assert ((back.double() - x.double()).abs() <= 2.0 ** -4 * x.double().abs() + 2.0 ** -10 * 2.0 ** -6).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_ends_of_the_range(gl, dtype):
    x = _device(_specials(), dtype)
    q = gl.gl_f8_quantize(gl.AccessPattern(x, 1))
    want, we = f8.quantize(x.double().cpu().numpy())
    got, ge = _codes(q, *x.shape)
    assert np.array_equal(ge, we) and np.array_equal(got, want)
    with np.errstate(over="ignore"):
        ref = f8.values(want, we).astype(np.float32)            # (2^128 is Inf)
    assert np.array_equal(gl.gl_f8_dequantize(q).tensor.cpu().numpy(), ref, equal_nan=True)
    # bf16 rounds what lies below 2^-124 * 2^-9
    half = gl.gl_f8_dequantize(q, gl.AccessPattern(torch.empty(x.shape, dtype=torch.bfloat16, device="cuda"), 1)).tensor
    assert torch.equal(half.cpu().nan_to_num(7), torch.from_numpy(ref).to(torch.bfloat16).nan_to_num(7))


def test_nothing_is_written_outside(gl):
    rows, k = 37, 1111
    s = gl._f8_meta((rows, k), 1)
    import ctypes
    nd, ns = gl.LIB.gl_f8_data_bytes(ctypes.byref(s)), gl.LIB.gl_f8_scale_bytes(ctypes.byref(s))
    data, scale = (torch.full((n + 512,), 0x5A, dtype=torch.uint8, device="cuda") for n in (nd, ns))
    q = gl.F8(data[256:256 + nd], scale[256:256 + ns], (rows, k), 1)
    x = _device(synth.normal(1, 2, (rows, k)), torch.float32)
    gl.gl_f8_quantize(gl.AccessPattern(x, 1), q)
    back = torch.full((rows * k + 256,), 7.0, device="cuda")
    gl.gl_f8_dequantize(q, gl.AccessPattern(back[128:128 + rows * k].view(rows, k), 1))
    for t, n, fill in ((data, nd, 0x5A), (scale, ns, 0x5A)):
        assert (t[:256] == fill).all() and (t[256 + n:] == fill).all()
    assert (back[:128] == 7).all() and (back[128 + rows * k:] == 7).all()
    assert np.array_equal(back[128:128 + rows * k].view(rows, k).double().cpu().numpy(), f8.rounded(x.double().cpu().numpy()))


# ---- products ----

def _close(got, a, b, relu, bf16):
    """Every one of the K exact products and the running sum loses at most an fp32 unit of sum |a||b| when it is aligned or
    added: K 2^-23 of it; then half a unit of bf16."""
    ref, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    if relu:
        ref = np.maximum(ref, 0.0)
    tol = a.shape[1] * 2.0 ** -23 * mag
    if bf16:
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
    err = np.abs(got.double().cpu().numpy().reshape(ref.shape) - ref)
    assert (err <= tol).all(), (err - tol).max()


SHAPES = [(1, 1, 1), (1, 17, 9), (1, 8192, 300), (2, 1111, 777), (4, 512, 129), (5, 640, 130), (16, 130, 40), (17, 896, 200),
          (33, 4096, 64), (64, 1000, 1000), (65, 96, 31), (128, 1184, 513), (129, 512, 128), (130, 33, 257), (301, 1111, 777),
          (256, 1024, 256), (511, 1600, 384), (700, 640, 1500), (1024, 2048, 2048)]


@pytest.mark.parametrize("m,k,o", SHAPES)
@pytest.mark.parametrize("relu,bf16", [(False, False), (True, True)])
def test_product_and_dense(gl, m, k, o, relu, bf16):
    x = _device(synth.normal(7, m * 31 + k, (m, k)) * np.exp(synth.normal(8, k, (1, k))), torch.bfloat16)
    w = _device(synth.normal(9, o * 31 + k, (o, k), k ** -0.5), torch.bfloat16)
    flags = (gl.GL_EPILOGUE_RELU if relu else 0) | (gl.GL_OUT_BF16 if bf16 else 0)
    a, b = f8.rounded(x.double().cpu().numpy()), f8.rounded(w.double().cpu().numpy())
    qw = gl.gl_f8_quantize(gl.AccessPattern(w, 1))
    _close(gl.gl_cartesian_dot_f8(gl.gl_f8_quantize(gl.AccessPattern(x, 1)), qw, flags=flags).tensor, a, b, relu, bf16)
    _close(gl.gl_dense_f8(gl.AccessPattern(x, 1), qw, flags=flags).tensor, a, b, relu, bf16)
    _close(gl.gl_dense_f8(gl.AccessPattern(x.float(), 1), qw, flags=flags).tensor, a, b, relu, bf16)
    assert gl.gl_poll_device_status() == 0


@pytest.mark.parametrize("m,k,o", SHAPES)
def test_whole_numbers_are_exact(gl, m, k, o):
    """Small whole numbers with block scales of every size between 2^-4 and 2^4: every sum is a whole number of 2^-8 below 2^24 of
    them, so nothing is rounded."""
    def side(seed, rows):
        x = synth.uniform_int(seed, rows * 7 + k, (rows, k), -3, 3).astype(np.float64)
        shift = synth.uniform_int(seed + 1, rows * 5 + k, (rows, -(-k // 128)), -4, 1)
        return x * np.repeat(np.exp2(shift.astype(np.float64)), 128, 1)[:, :k]
    a, b = side(11, m), side(13, o)
    assert np.array_equal(f8.rounded(a), a) and (np.abs(a) @ np.abs(b).T).max() * 256 < 2 ** 24
    qa, qb = (gl.gl_f8_quantize(gl.AccessPattern(_device(v, torch.float32), 1)) for v in (a, b))
    assert np.array_equal(gl.gl_cartesian_dot_f8(qa, qb).tensor.double().cpu().numpy(), a @ b.T)
    assert np.array_equal(gl.gl_dense_f8(gl.AccessPattern(_device(a, torch.bfloat16), 1), qb).tensor.double().cpu().numpy(), a @ b.T)


# K cut over clusters with more than 64 and more than 128 rows, a second block per SM, pairs of SMs with rows that start anywhere,
# several rounds of pairs, bands of tile rows of two heights
@pytest.mark.parametrize("m,k,o", [(70, 2100, 200), (300, 2100, 200), (129, 2048, 99), (200, 8300, 8200), (70, 100, 19000),
                                   (2000, 300, 2001), (4096, 300, 4099), (5000, 200, 1500), (900, 700, 3000)])
@pytest.mark.parametrize("bf16", [False, True])
def test_every_way_of_cutting_a_product(gl, m, k, o, bf16):
    g = torch.Generator("cuda").manual_seed(m + k + o)
    a = torch.randint(-3, 4, (m, k), generator=g, device="cuda").float()
    b = torch.randint(-3, 4, (o, k), generator=g, device="cuda").float()
    out = gl.gl_dense_f8(gl.AccessPattern(a, 1), gl.gl_f8_quantize(gl.AccessPattern(b, 1)), flags=gl.GL_OUT_BF16 if bf16 else 0).tensor
    want = a.double() @ b.double().t()              # whole numbers below 2^24: every sum is exact
    assert torch.equal(out, want.to(out.dtype)) and gl.gl_poll_device_status() == 0


def test_what_lies_behind_rows_and_blocks_does_not_matter(gl):
    """Scale bytes of rows and blocks that do not exist are never written; as NaN they must not reach a result."""
    for m, k, o in ((1, 130, 5), (40, 700, 200), (130, 900, 131), (600, 300, 700)):
        ops = []
        for rows in (m, o):
            q = gl.f8_empty((rows, k), 1, "cuda")
            q.data.fill_(0x7F)
            q.scale.fill_(0xFF)
            x = torch.randint(-3, 4, (rows, k), generator=torch.Generator("cuda").manual_seed(rows), device="cuda").float()
            ops.append((x, gl.gl_f8_quantize(gl.AccessPattern(x, 1), q)))
        (a, qa), (b, qb) = ops
        want = (a.double() @ b.double().t()).float()
        assert torch.equal(gl.gl_cartesian_dot_f8(qa, qb).tensor, want)
        assert torch.equal(gl.gl_dense_f8(gl.AccessPattern(a, 1), qb).tensor, want)


@pytest.mark.parametrize("m", [1, 20, 200])
def test_scales_far_from_one(gl, m):
    """Factors of every size whose products stay inside fp32: the scales of both sides meet before anything is rounded."""
    k, o = 640, 150
    a = synth.uniform_int(41, m, (m, k), -3, 3).astype(np.float64)
    b = synth.uniform_int(42, o, (o, k), -3, 3).astype(np.float64)
    for ea, eb in ((-100, 90), (100, -110), (60, 50), (-60, -50), (-118, 118)):
        fa, fb = 2.0 ** ea, 2.0 ** eb
        qb = gl.gl_f8_quantize(gl.AccessPattern(_device(b * fb, torch.float32), 1))
        out = gl.gl_dense_f8(gl.AccessPattern(_device(a * fa, torch.float32), 1), qb).tensor
        assert np.array_equal(out.double().cpu().numpy(), (a @ b.T) * fa * fb), (ea, eb)


def test_beyond_two_to_the_31_values(gl):
    """Offsets of operands and of results in 64 bits."""
    rows, k = 270000, 8192
    x = torch.empty((rows, k), dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn((3, k), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    x[:-3].fill_(1.0)
    q = gl.gl_f8_quantize(gl.AccessPattern(x, 1))
    back = gl.gl_f8_dequantize(q, gl.AccessPattern(x, 1)).tensor           # (x has been read)
    last = torch.randn((3, k), generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    assert np.array_equal(back[-3:].double().cpu().numpy(), f8.rounded(last.double().cpu().numpy())) and (back[:-3] == 1).all()
    w = torch.randint(-3, 4, (8200, k), generator=torch.Generator("cuda").manual_seed(2), device="cuda").float()
    qw = gl.gl_f8_quantize(gl.AccessPattern(w, 1))
    del x, back
    out = gl.gl_cartesian_dot_f8(q, qw, flags=gl.GL_OUT_BF16).tensor
    assert torch.equal(out[:-3].amin(0), w.sum(1).to(torch.bfloat16)) and torch.equal(out[:-3].amax(0), w.sum(1).to(torch.bfloat16))
    a = f8.rounded(last.double().cpu().numpy())
    _close(out[-3:], a, w.double().cpu().numpy(), False, True)


def test_item_shapes_and_guard_bands(gl):
    """((B, T),(c, d)) x ((h, e),(c, d)) -> ((B, T, h, e),()); rows without 16-byte multiples, guarded."""
    for m, o, bf16 in (((2, 3), (3, 5), True), ((2, 70), (3, 43), False), ((3, 67), (5, 31), True)):
        x = _device(synth.normal(2, m[1], m + (6, 40)), torch.bfloat16)
        w = _device(synth.normal(3, o[1], o + (6, 40)), torch.bfloat16)
        n = m[0] * m[1] * o[0] * o[1]
        dtype = torch.bfloat16 if bf16 else torch.float32
        store = torch.full((n + 1024,), 7.0, dtype=dtype, device="cuda")
        out = gl.AccessPattern(store[512:512 + n].view(m + o), 4)
        gl.gl_dense_f8(gl.AccessPattern(x, 2), gl.gl_f8_quantize(gl.AccessPattern(w, 2)), out, gl.GL_OUT_BF16 if bf16 else 0)
        a, b = (f8.rounded(t.double().cpu().numpy().reshape(-1, 240)) for t in (x, w))
        _close(out.tensor, a, b, False, bf16)
        assert (store[:512] == 7).all() and (store[512 + n:] == 7).all()


@pytest.mark.parametrize("m", [1, 40, 300])
def test_nan_blocks_reach_their_row_only(gl, m):
    """A block that holds an Inf is NaN; rows and columns without one are what they were, relu lets NaN through."""
    k, o = 700, 200
    x, w = synth.bf16_round(synth.normal(2, m, (m, k))), synth.bf16_round(synth.normal(3, m, (o, k)))
    clean = f8.rounded(x) @ f8.rounded(w).T
    tol = k * 2.0 ** -23 * (np.abs(f8.rounded(x)) @ np.abs(f8.rounded(w)).T)
    x[m // 2, 650], w[11, 3] = np.inf, np.nan
    out = gl.gl_dense_f8(gl.AccessPattern(_device(x, torch.bfloat16), 1), gl.gl_f8_quantize(gl.AccessPattern(_device(w, torch.bfloat16), 1)),
                         flags=gl.GL_EPILOGUE_RELU).tensor.double().cpu().numpy()
    bad = np.zeros((m, o), dtype=bool)
    bad[m // 2], bad[:, 11] = True, True
    assert np.isnan(out[bad]).all()
    assert (np.abs(out - np.maximum(clean, 0)) <= tol)[~bad].all()


def test_graph_streams_and_two_workspaces(gl):
    """Captured once, replayed on changed inputs; at the same time eager calls on another stream."""
    x = torch.randn(48, 1024, device="cuda").to(torch.bfloat16)
    w = gl.gl_f8_quantize(gl.AccessPattern(torch.randn(512, 1024, device="cuda"), 1))
    out = gl.AccessPattern(torch.empty(48, 512, device="cuda"), 2)
    call = gl.prepare_dense_f8(gl.AccessPattern(x, 1), w, out)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    side = torch.cuda.Stream()
    for seed in range(3):
        x.copy_(torch.randn(48, 1024, generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        other = gl.gl_dense_f8(gl.AccessPattern(x, 1), w, stream=side)
        torch.cuda.synchronize()
        want = gl.gl_dense_f8(gl.AccessPattern(x, 1), w)
        assert torch.equal(out.tensor, want.tensor) and torch.equal(other.tensor, want.tensor)
