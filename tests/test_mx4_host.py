"""Host-only checks of the 4-bit operators: the checker's rounding rules, storage sizes, refused arguments."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import mx4


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import build
    build.build()
    from paper_2105_09377_b200 import binding
    return binding


def test_checker_rounds_to_the_nearest_with_ties_to_even():
    block = np.zeros((1, 32))
    block[0, :17] = [6.0, 0.25, 0.26, 0.75, 0.74, 1.25, 1.26, 1.75, 1.74, 2.5, 2.51, 3.5, 3.49, 5.0, 5.01, 7.9, -0.25]
    codes, exps = mx4.quantize(block)      # largest 7.9: scale 1
    assert exps[0, 0] == 127
    want = [6, 0, .5, 1, .5, 1, 1.5, 2, 1.5, 2, 3, 4, 3, 4, 6, 6, 0]
    assert np.array_equal(mx4.values(codes, exps)[0, :17], want) and codes[0, 0, 16] == 8   # minus zero keeps its sign
    # scales: a power of two below 8 times the largest; floor at 2^-127; NaN and Inf take the block with them
    for top, e in [(8.0, 128), (7.999999, 127), (4.0, 127), (3.999, 126), (2.0 ** -126, 0), (2.0 ** -140, 0), (3.3e38, 252), (0.0, 0)]:
        x = np.zeros((1, 40))
        x[0, 3] = -top
        assert mx4.quantize(x)[1].tolist() == [[e, 0]], top
    x = np.ones((1, 64))
    x[0, 40] = np.inf
    assert mx4.quantize(x)[1].tolist() == [[125, 255]]
    x[0, 40] = np.nan
    assert np.isnan(mx4.rounded(x)[0, 32:]).all() and not np.isnan(mx4.rounded(x)[0, :32]).any()


def test_checker_attention_against_torch():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(3, 4, 64)), rng.normal(size=(10, 2, 64)), rng.normal(size=(10, 2, 64))
    out, _ = mx4.attend(q, k, v, 2, 0.125, 7)
    mask = torch.ones(3, 10, dtype=torch.bool).tril(7)
    ref = torch.nn.functional.scaled_dot_product_attention(
        torch.tensor(q).transpose(0, 1), torch.tensor(k).transpose(0, 1).repeat_interleave(2, 0),
        torch.tensor(v).transpose(0, 1).repeat_interleave(2, 0), attn_mask=mask, scale=0.125).transpose(0, 1).numpy()
    np.testing.assert_allclose(out, ref, rtol=1e-12, atol=1e-14)
    assert not mx4.attend(q, k, v, 2, 0.125, -2)[0][0].any()     # row 0 sees nothing


@pytest.mark.parametrize("shape,na,data,scale", [
    ((5, 32), 1, 5 * 16, 512), ((1, 1), 1, 16, 512), ((129, 33), 1, 129 * 32, 1024), ((3, 4, 2, 100), 2, 12 * 112, 1024),
    ((7, 9), 2, 63 * 16, 512), ((200, 129), 1, 200 * 80, 2 * 2 * 512)])
def test_storage_sizes(gl, shape, na, data, scale):
    s = gl._mx4_meta(shape, na)
    assert gl.LIB.gl_mx4_data_bytes(ctypes.byref(s)) == data
    assert gl.LIB.gl_mx4_scale_bytes(ctypes.byref(s)) == scale


def test_struct_layouts(gl):
    assert ctypes.sizeof(gl.GlMx4) == 2 * 8 + 2 * 4 + 8 * 8
    assert ctypes.sizeof(gl.GlCache4) == 2 * 8 + 4 * 4 and ctypes.sizeof(gl.GlPages) == 2 * 8 + 2 * 4


FAKE = 1 << 20   # an aligned address that no refused call touches


def _ap(gl, shape, na, dtype=None, data=FAKE):
    return gl._meta(shape, na, gl.GL_BF16 if dtype is None else dtype, data)


def _mx(gl, shape, na, data=FAKE, scale=FAKE):
    s = gl._mx4_meta(shape, na)
    s.data, s.scale = data, scale
    return s


def test_refusals_of_quantisation(gl):
    r = ctypes.byref
    f = gl.LIB.gl_mx4_quantize
    ok_in, ok_out = _ap(gl, (4, 64), 1), _mx(gl, (4, 64), 1)
    assert f(None, r(ok_out), None) == 1 and f(r(ok_in), None, None) == 1
    assert f(r(ok_in), r(_mx(gl, (4, 64), 1, data=0)), None) == 1
    assert f(r(ok_in), r(_mx(gl, (4, 64), 1, scale=FAKE + 8)), None) == 6
    assert f(r(_ap(gl, (4, 64), 1, data=FAKE + 2)), r(ok_out), None) == 6
    assert f(r(_ap(gl, (4, 64), 1, dtype=7)), r(ok_out), None) == 2
    assert f(r(ok_in), r(_mx(gl, (4, 63), 1)), None) == 4 and f(r(ok_in), r(_mx(gl, (4, 64), 2)), None) == 4
    assert f(r(ok_in), r(_mx(gl, (4, 0), 1)), None) == 4
    big = (1 << 20, 1 << 16)
    assert f(r(_ap(gl, big, 1)), r(_mx(gl, big, 1)), None) == 7
    g = gl.LIB.gl_mx4_dequantize
    assert g(None, r(ok_in), None) == 1 and g(r(ok_out), r(_ap(gl, (64, 4), 1)), None) == 4
    assert g(r(_mx(gl, big, 1)), r(_ap(gl, big, 1)), None) == 7


def test_refusals_of_the_products(gl):
    r = ctypes.byref
    f = gl.LIB.gl_cartesian_dot_mx4
    a, b = _mx(gl, (4, 64), 1), _mx(gl, (6, 64), 1)
    out = _ap(gl, (4, 6), 2, gl.GL_F32)
    assert f(None, r(b), r(out), 0, None) == 1 and f(r(a), None, r(out), 0, None) == 1 and f(r(a), r(b), None, 0, None) == 1
    assert f(r(a), r(_mx(gl, (6, 32), 1)), r(out), 0, None) == 4                      # items differ
    assert f(r(a), r(_mx(gl, (6, 8, 8), 1)), r(out), 0, None) == 4                    # the same length, another shape
    assert f(r(a), r(b), r(_ap(gl, (6, 4), 2, gl.GL_F32)), 0, None) == 4
    assert f(r(a), r(b), r(_ap(gl, (4, 6), 2)), 0, None) == 2 and f(r(a), r(b), r(out), gl.GL_OUT_BF16, None) == 2
    assert f(r(a), r(b), r(out), gl.GL_OUT_NCHW, None) == 7
    assert f(r(a), r(b), r(_ap(gl, (4, 6), 2, gl.GL_F32, FAKE + 4)), 0, None) == 6
    d = gl.LIB.gl_dense_mx4
    x = _ap(gl, (4, 64), 1)
    need = gl.LIB.gl_dense_mx4_workspace(r(x), r(b))
    assert need >= 4 * 32 + 512
    assert d(r(x), r(b), r(out), 0, None, 0, None) == 8 and d(r(x), r(b), r(out), 0, FAKE, need - 1, None) == 8
    assert d(r(x), r(b), r(out), 0, FAKE + 16, need, None) == 8
    assert d(r(_ap(gl, (4, 32), 1)), r(b), r(out), 0, FAKE, need, None) == 4


def _cache(gl, pages=4, heads=2, page=32, d=64, data=FAKE):
    s = gl.GlCache4()
    s.data, s.pages, s.kv_heads, s.page_tokens, s.head_dim = data, pages, heads, page, d
    return s


def _at(gl, batch=3, width=2, table=FAKE, lengths=FAKE):
    s = gl.GlPages()
    s.page_table, s.lengths, s.batch, s.table_width = table, lengths, batch, width
    return s


def test_refusals_of_the_cache(gl):
    r = ctypes.byref
    assert gl.LIB.gl_cache4_bytes(r(_cache(gl))) == 4 * 2 * 2 * 17 * 64
    assert gl.LIB.gl_cache4_bytes(r(_cache(gl, page=24))) == 0 and gl.LIB.gl_cache4_bytes(r(_cache(gl, d=96))) == 0
    f = gl.LIB.gl_cache4_append
    k = _ap(gl, (3, 5, 2, 64), 3)

    def call(cache=None, kk=k, vv=k, pitch=0, at=None):
        return f(r(cache or _cache(gl)), r(kk), r(vv), pitch, r(at or _at(gl)), None)

    assert call(cache=_cache(gl, page=24)) == 7 and call(cache=_cache(gl, d=96)) == 7 and call(cache=_cache(gl, pages=0)) == 4
    assert call(cache=_cache(gl, data=0)) == 1 and call(cache=_cache(gl, data=FAKE + 4)) == 6
    assert call(at=_at(gl, table=0)) == 1 and call(at=_at(gl, lengths=0)) == 1 and call(at=_at(gl, lengths=FAKE + 2)) == 6
    assert call(at=_at(gl, batch=0)) == 4 and call(at=_at(gl, width=0)) == 4 and call(at=_at(gl, batch=2)) == 4
    assert call(at=_at(gl, width=1 << 30)) == 7                                           # more than 2^31 tokens
    assert call(kk=_ap(gl, (3, 5, 2, 64), 3, gl.GL_F32)) == 2 and call(kk=_ap(gl, (3, 5, 2, 64), 2)) == 3
    assert call(kk=_ap(gl, (3, 5, 1, 64), 3)) == 4 and call(vv=_ap(gl, (3, 4, 2, 64), 3)) == 4
    assert call(pitch=127) == 4 and call(pitch=132) == 6
    assert gl.LIB.gl_cache4_read(r(_cache(gl)), r(_at(gl)), r(k), r(_ap(gl, (3, 5, 2, 128), 3)), None) == 4


def test_refusals_of_the_attention(gl):
    r = ctypes.byref
    q, out = _ap(gl, (3, 5, 6, 64), 3), _ap(gl, (3, 5, 6, 64), 3, gl.GL_F32)

    def call(qq=q, oo=out, pitch=0, cache=None, at=None, scale=0.125, flags=0, ws=FAKE, n=1 << 40):
        return gl.LIB.gl_attend_cache4(r(qq), pitch, r(cache or _cache(gl)), r(at or _at(gl)), scale, r(oo), flags, ws, n, None)

    assert gl.LIB.gl_attend_cache4_workspace(r(q), r(_cache(gl))) > 0
    assert gl.LIB.gl_attend_cache4_workspace(r(_ap(gl, (3, 5, 5, 64), 3)), r(_cache(gl))) == 0
    assert call(qq=_ap(gl, (3, 5, 5, 64), 3), oo=_ap(gl, (3, 5, 5, 64), 3, gl.GL_F32)) == 4      # heads are no multiple
    assert call(qq=_ap(gl, (3, 5, 6, 64), 3, gl.GL_F32)) == 2 and call(oo=q) == 2 and call(flags=gl.GL_OUT_BF16) == 2
    assert call(oo=_ap(gl, (3, 5, 6, 64), 2, gl.GL_F32)) == 4 and call(oo=_ap(gl, (3, 5, 6, 64), 3, gl.GL_F32, FAKE + 4)) == 6
    for s in (0.0, -1.0, float("inf"), float("nan")):
        assert call(scale=s) == 4
    assert call(flags=gl.GL_EPILOGUE_RELU) == 7 and call(pitch=8) == 4
    assert call(ws=None) == 8 and call(n=16) == 8 and call(ws=FAKE + 64) == 8
    assert call(at=_at(gl, batch=4)) == 4


def test_binding_refuses_what_it_cannot_describe(gl):
    with pytest.raises(ValueError):
        gl._tokens_struct(torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16).transpose(1, 2))
    with pytest.raises(ValueError):
        gl._tokens_struct(torch.zeros(2, 6, 4, 64, dtype=torch.bfloat16)[:, ::2][:, :2])
    fused = torch.zeros(2, 3, 12, 64, dtype=torch.bfloat16)
    assert gl._tokens_struct(fused[:, :, 4:8])[1] == 12 * 64
    with pytest.raises(ValueError):
        gl._pages_struct(torch.zeros(2, 3, dtype=torch.int64), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        gl._mx4_struct(gl.Mx4(torch.zeros(16, dtype=torch.uint8), torch.zeros(511, dtype=torch.uint8), (1, 32), 1))
