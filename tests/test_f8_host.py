"""Host-only checks of the 8-bit operators, the norm and the rotation: the checker itself, sizes, refusals, the rotary plan, what
the binding hands on."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import f8

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import build
    build.build()
    from paper_2105_09377_b200 import binding
    return binding


# ---- the checker ----

def test_grid_is_e4m3():
    ours = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(f8.GRID, ours) and f8.GRID[-1] == 448.0


def test_rounding_of_the_checker():
    x = np.array([[1.0, 448.0, 0.0, -16.9, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10]])
    codes, exps = f8.quantize(x)
    assert exps[0, 0] == 127
    assert f8.values(codes, exps, 8).tolist() == [[1.0, 448.0, 0.0, -16.0, 16.0, 20.0, 0.0, 2.0 ** -8]]
    assert f8.quantize([[449.0]])[1][0, 0] == 128 and f8.quantize([[0.0]])[1][0, 0] == 0
    assert f8.quantize([[1.75]])[1][0, 0] == 127 - 8 and f8.quantize([[1.7500001]])[1][0, 0] == 127 - 7
    assert f8.quantize([[1.0, np.inf]])[1][0, 0] == 255 and np.isnan(f8.rounded([[1.0, np.nan]])).all()
    r = np.random.default_rng(1).standard_normal((9, 1000)) * 10
    assert (np.abs(f8.rounded(r) - r) <= 2.0 ** -4 * np.abs(r) + 2.0 ** -10 * 2.0).all()


def test_norm_and_rotation_of_the_checker():
    h, y = f8.norm_rms([[3.0, 4.0]], [[0.0, 0.0]], [1.0, 2.0], 0.0)
    assert h.tolist() == [[3.0, 4.0]] and np.allclose(y, [[3 / math.sqrt(12.5), 8 / math.sqrt(12.5)]])
    x = np.arange(1.0, 7.0).reshape(1, 1, 1, 6)
    quarter = [2 ** 62, 2 ** 63]
    assert np.allclose(f8.rotate(x, np.ones((1, 1, 1), int), quarter, [0, 0], False), [[[[-3, -2, 1, -4, 5, 6]]]])
    assert np.allclose(f8.rotate(x, np.ones((1, 1, 1), int), quarter, [0, 0], True), [[[[-2, 1, -3, -4, 5, 6]]]])
    assert f8.turns(-1, 2 ** 62) == -0.25 and f8.turns(3, 2 ** 62) == -0.25 and f8.turns(4, 2 ** 62) == 0


# ---- sizes and refusals ----

@pytest.mark.parametrize("rows,k", [(1, 1), (3, 16), (3, 17), (128, 512), (129, 513), (777, 1111)])
def test_bytes(gl, rows, k):
    s = gl._f8_meta((rows, k), 1)
    assert gl.LIB.gl_f8_data_bytes(ctypes.byref(s)) == rows * (-(-k // 16) * 16)
    assert gl.LIB.gl_f8_scale_bytes(ctypes.byref(s)) == -(-rows // 128) * -(-k // 512) * 512
    assert f8.scale_at(rows, -(-k // 128)).max() < -(-rows // 128) * -(-k // 512) * 512


def test_operands_beyond_the_limits_have_no_size(gl):
    for shape in ((2 ** 31, 4), (4, 2 ** 28 + 1), (2 ** 30, 300), (2 ** 35, 2 ** 35, 2 ** 35), (3, 0)):
        s = gl._f8_meta(shape, 1)
        assert gl.LIB.gl_f8_data_bytes(ctypes.byref(s)) == 0 and gl.LIB.gl_f8_scale_bytes(ctypes.byref(s)) == 0
    with pytest.raises(gl.GlError):
        gl.f8_empty((3, 0), 1, "cpu")


def _ap(gl, shape, access, dtype, data=0x1000):
    return gl._meta(shape, access, dtype, data)


def _f8(gl, shape, access, data=0x1000, scale=0x1000):
    s = gl._f8_meta(shape, access)
    s.data, s.scale = data, scale
    return s


def test_refusals_of_rounding(gl):
    """Checked before anything is launched (there is no GPU here to launch on)."""
    r = ctypes.byref
    ok = _ap(gl, (4, 64), 1, gl.GL_BF16)
    q = lambda a, m: gl.LIB.gl_f8_quantize(r(a), r(m), None)
    d = lambda m, a: gl.LIB.gl_f8_dequantize(r(m), r(a), None)
    assert q(_ap(gl, (4, 64), 1, gl.GL_BF16, 0), _f8(gl, (4, 64), 1)) == 1
    assert q(ok, _f8(gl, (4, 64), 1, data=0)) == 1 and q(ok, _f8(gl, (4, 64), 1, scale=0)) == 1
    assert q(ok, _f8(gl, (4, 64), 1, scale=0x1008)) == 6 and q(_ap(gl, (4, 64), 1, gl.GL_BF16, 0x1004), _f8(gl, (4, 64), 1)) == 6
    assert q(ok, _f8(gl, (4, 65), 1)) == 4 and q(ok, _f8(gl, (4, 64), 2)) == 4 and q(ok, _f8(gl, (2, 2, 64), 2)) == 4
    assert q(_ap(gl, (4, 64), 1, 7), _f8(gl, (4, 64), 1)) == 2
    assert q(_ap(gl, (2 ** 30, 300), 1, gl.GL_BF16), _f8(gl, (2 ** 30, 300), 1)) == 7
    assert d(_f8(gl, (4, 64), 1), _ap(gl, (4, 63), 1, gl.GL_F32)) == 4 and d(_f8(gl, (4, 64), 1, data=0), ok) == 1
    assert gl.LIB.gl_f8_quantize(None, r(_f8(gl, (4, 64), 1)), None) == 1 and gl.LIB.gl_f8_quantize(r(ok), None, None) == 1


def test_refusals_of_products(gl):
    r = ctypes.byref
    a, b, out = _f8(gl, (4, 64), 1), _f8(gl, (6, 64), 1), _ap(gl, (4, 6), 2, gl.GL_F32)
    dot = lambda a, b, o, f=0: gl.LIB.gl_cartesian_dot_f8(r(a), r(b), r(o), f, None)
    assert dot(a, _f8(gl, (6, 65), 1), out) == 4 and dot(a, _f8(gl, (6, 8, 8), 1), out) == 4
    assert dot(a, b, _ap(gl, (4, 7), 2, gl.GL_F32)) == 4 and dot(a, b, _ap(gl, (4, 6), 1, gl.GL_F32)) == 4
    assert dot(a, b, _ap(gl, (4, 6), 2, gl.GL_BF16)) == 2 and dot(a, b, out, gl.GL_OUT_BF16) == 2
    assert dot(a, b, out, gl.GL_OUT_NCHW) == 7 and dot(a, b, out, 0x400) == 7
    assert dot(a, b, _ap(gl, (4, 6), 2, gl.GL_F32, 0x1004)) == 6 and dot(_f8(gl, (4, 64), 1, data=0), b, out) == 1
    x = _ap(gl, (4, 64), 1, gl.GL_F32)
    dense = lambda ws, n, x=x, o=out: gl.LIB.gl_dense_f8(r(x), r(b), r(o), 0, ws, n, None)
    need = gl.LIB.gl_dense_f8_workspace(r(x), r(b))
    assert need == 1024 + 512
    assert dense(None, 0) == 8 and dense(0x4000, need - 1) == 8 and dense(0x4200, need) == 8
    assert dense(0x4000, need, _ap(gl, (4, 65), 1, gl.GL_F32)) == 4
    assert dense(0x4000, need, _ap(gl, (2 ** 30, 1, 64), 2, gl.GL_F32), _ap(gl, (2 ** 30, 1, 6), 3, gl.GL_F32)) in (7, 8)


def test_refusals_of_the_norm(gl):
    r = ctypes.byref
    x, out, w = _ap(gl, (4, 64), 1, gl.GL_BF16), _ap(gl, (4, 64), 1, gl.GL_F32), _ap(gl, (64,), 0, gl.GL_F32)
    res, p = _ap(gl, (4, 64), 1, gl.GL_F32), lambda a: None if a is None else r(a)

    def norm(x=x, res=None, w=w, eps=1e-5, total=None, out=out):
        return gl.LIB.gl_compute_norm_rms(p(x), p(res), p(w), eps, p(total), p(out), None)

    assert norm(x=None) == 1 and norm(out=None) == 1 and norm(total=res) == 1                    # a sum of what?
    assert norm(x=_ap(gl, (4, 64), 2, gl.GL_BF16)) == 4                                          # nothing to take the mean of
    assert norm(res=_ap(gl, (4, 65), 1, gl.GL_F32)) == 4 and norm(res=_ap(gl, (4, 64), 2, gl.GL_F32)) == 4
    assert norm(res=res, total=_ap(gl, (4, 64), 1, gl.GL_BF16)) == 2                             # the residual's type
    assert norm(res=res, total=_ap(gl, (4, 63), 1, gl.GL_F32)) == 4
    assert norm(w=_ap(gl, (63,), 0, gl.GL_F32)) == 4 and norm(w=_ap(gl, (64,), 1, gl.GL_F32)) == 4
    assert norm(w=_ap(gl, (64,), 0, gl.GL_F32, 0x1008)) == 6
    for eps in (-1e-9, math.nan, math.inf):
        assert norm(eps=eps) == 4
    assert norm(out=_ap(gl, (4, 63), 1, gl.GL_F32)) == 4 and norm(out=_ap(gl, (4, 64), 1, 5)) == 2
    assert norm(x=_ap(gl, (4, 64), 1, gl.GL_BF16, 0x1002)) == 6
    assert norm(res=res, total=_ap(gl, (4, 64), 1, gl.GL_F32, 0x7000), out=_ap(gl, (4, 64), 1, gl.GL_F32, 0x7000)) == 7
    assert norm(x=_ap(gl, (2 ** 31, 64), 1, gl.GL_BF16), out=_ap(gl, (2 ** 31, 64), 1, gl.GL_F32)) == 7
    eight = lambda m: gl.LIB.gl_compute_norm_rms_f8(r(x), None, r(w), 1e-5, None, r(m), None)
    assert eight(_f8(gl, (4, 65), 1)) == 4 and eight(_f8(gl, (4, 64), 1, scale=0)) == 1 and eight(_f8(gl, (4, 64), 1, data=0x1001)) == 6


def test_refusals_of_the_rotation(gl):
    r = ctypes.byref
    plan = gl.rotary_plan(16, sections=(10, 6))
    x = _ap(gl, (2, 3, 4, 40), 3, gl.GL_BF16)

    def rotate(x=x, pitch=0, plan=plan, pos=0x1000, out=None, out_pitch=0, flags=0):
        out = _ap(gl, (2, 3, 4, 40), 3, gl.GL_BF16, 0x9000) if out is None else out
        return gl.LIB.gl_compute_rotate(r(x), pitch, r(plan), pos, r(out), out_pitch, flags, None)

    assert rotate(pos=None) == 1 and rotate(pos=0x1002) == 6 and rotate(flags=1) == 7
    assert rotate(x=_ap(gl, (2, 3, 4, 40), 2, gl.GL_BF16)) == 3 and rotate(x=_ap(gl, (6, 4, 40), 2, gl.GL_BF16)) == 3
    assert rotate(out=_ap(gl, (2, 3, 4, 41), 3, gl.GL_BF16)) == 4 and rotate(out=_ap(gl, (2, 3, 4, 40), 3, gl.GL_F32)) == 2
    assert rotate(pitch=159) == 4 and rotate(out_pitch=159) == 4 and rotate(pitch=-160) == 4
    assert rotate(out=_ap(gl, (2, 3, 4, 40), 3, gl.GL_BF16), pitch=160, out_pitch=168) == 4      # in place: one view
    assert rotate(plan=gl.rotary_plan(21)) == 4                                                  # 42 values of a head of 40
    for field, value in (("pairs", 0), ("pairs", 129), ("axes", 0), ("axes", 17), ("adjacent", 2)):
        bad = gl.rotary_plan(16, sections=(10, 6))
        setattr(bad, field, value)
        assert rotate(plan=bad) == 4, field
    bad = gl.rotary_plan(16, sections=(10, 6))
    bad.axis[7] = 2
    assert rotate(plan=bad) == 4
    big = lambda d: _ap(gl, d, 3, gl.GL_BF16, 0x9000)
    assert rotate(x=big((2 ** 20, 2 ** 12, 4, 40)), out=big((2 ** 20, 2 ** 12, 4, 40))) == 7
    assert rotate(x=big((1, 1, 2 ** 20, 40)), out=big((1, 1, 2 ** 20, 40))) == 7


# ---- the rotary plan ----

def test_steps_of_the_plan(gl):
    """2^64 base^(-i/n) / (2 pi), to what a long double carries: 2^-62 of the value and half a unit."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
    for pairs, base in ((1, 10000.0), (64, 10000.0), (128, 500000.0), (33, 1.0)):
        plan = gl.rotary_plan(pairs, base)
        for i in range(pairs):
            want = Decimal(base) ** (Decimal(-i) / Decimal(pairs)) / (2 * pi) * 2 ** 64
            assert abs(Decimal(plan.step[i]) - want) <= Decimal(0.5) + want / 2 ** 60, i
        assert not any(plan.axis[:128]) and plan.pairs == pairs and plan.axes == 1
    plan = gl.rotary_plan(3, freq=[-math.pi / 2, 2 * math.pi * 5, 7.0])
    assert abs(plan.step[0] - 3 * 2 ** 62) < 2 ** 12 and min(plan.step[1], 2 ** 64 - plan.step[1]) < 2 ** 16
    assert abs(plan.step[2] / 2 ** 64 - (7.0 / (2 * math.pi) - 1)) < 1e-15


def test_sections_of_the_plan(gl):
    assert list(gl.rotary_plan(6, sections=(3, 1, 2)).axis[:6]) == [0, 0, 0, 1, 2, 2]
    assert list(gl.rotary_plan(5, sections=(0, 5, 0)).axis[:5]) == [1] * 5
    assert list(gl.rotary_plan(5, sections=(2, 0, 3)).axis[:5]) == [0, 0, 2, 2, 2]
    for args in (dict(pairs=0), dict(pairs=129), dict(pairs=8, sections=(4, 5)), dict(pairs=8, sections=(9, -1)), dict(pairs=8, base=0.5),
                 dict(pairs=8, base=math.nan), dict(pairs=2, sections=(1, 1, 0)), dict(pairs=2, freq=[1.0, math.inf])):
        with pytest.raises(gl.GlError):
            gl.rotary_plan(**args)
    with pytest.raises(ValueError):
        gl.rotary_plan(3, freq=[1.0])
    assert gl.LIB.gl_rotary_plan(4, 10000.0, None, None, 2, 0, ctypes.byref(gl.GlRotary())) == 1
    assert gl.LIB.gl_rotary_plan(4, 10000.0, None, None, 1, 0, None) == 1
    assert ctypes.sizeof(gl.GlRotary) == 16 + 128 * 8 + 128


# ---- the binding ----

def _made(shape, dtype):
    return torch.zeros(shape, dtype=dtype)


def _calls(gl):
    """Every call as a function of tensors that live on the host."""
    ap = gl.AccessPattern
    m = lambda rows, k: gl.f8_empty((rows, k), 1, "cpu")
    x, y, out = ap(_made((4, 64), BF), 1), ap(_made((4, 64), BF), 1), ap(_made((4, 6), F32), 2)
    w = ap(_made((64,), F32), 0)
    plan = gl.rotary_plan(16)
    t, pos = ap(_made((2, 3, 4, 64), BF), 3), _made((2, 3), torch.int32)
    ws = _made(1 << 16, torch.uint8)
    return {
        "quantize": lambda: gl.gl_f8_quantize(x, m(4, 64)), "dequantize": lambda: gl.gl_f8_dequantize(m(4, 64), x),
        "product": lambda: gl.gl_cartesian_dot_f8(m(4, 64), m(6, 64), out), "dense": lambda: gl.gl_dense_f8(x, m(6, 64), out),
        "norm": lambda: gl.gl_compute_norm_rms(x, w, 1e-5, y, y, x), "norm_f8": lambda: gl.gl_compute_norm_rms_f8(x, w, 1e-5, y, y, m(4, 64)),
        "rotate": lambda: gl.gl_compute_rotate(t, plan, pos, t),
        "prepare_quantize": lambda: gl.prepare_f8_quantize(x, m(4, 64)), "prepare_dequantize": lambda: gl.prepare_f8_dequantize(m(4, 64), x),
        "prepare_product": lambda: gl.prepare_cartesian_dot_f8(m(4, 64), m(6, 64), out),
        "prepare_dense": lambda: gl.prepare_dense_f8(x, m(6, 64), out, workspace=ws),
        "prepare_norm": lambda: gl.prepare_compute_norm_rms(x, w, m(4, 64), 1e-5, y, y),
        "prepare_rotate": lambda: gl.prepare_compute_rotate(t, plan, pos, t),
    }


@pytest.mark.parametrize("name", ["quantize", "dequantize", "product", "dense", "norm", "norm_f8", "rotate", "prepare_quantize",
                                  "prepare_dequantize", "prepare_product", "prepare_dense", "prepare_norm", "prepare_rotate"])
def test_host_tensors_are_refused(gl, name):
    with pytest.raises(ValueError, match="GPU"):
        _calls(gl)[name]()


def test_the_gpu_of_the_tensors_is_the_current_one(gl, monkeypatch):
    """Another one's streams would run the kernels on addresses that are not theirs; a prepared call asks again."""
    class T:                                       # (what the check looks at; this machine has no GPU)
        is_cuda = True

        def __init__(self, device):
            self.device = torch.device(device)
    now = [0]
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda gpu: 3 + gpu, raising=False)
    assert gl._on_this_gpu(T("cuda:0"), None, T("cuda:0")) == 0
    for devices in (("cuda:1", "cuda:1"), ("cuda:0", "cuda:1")):
        with pytest.raises(ValueError):
            gl._on_this_gpu(*(T(d) for d in devices))
    ran = []
    call = gl.Prepared(lambda raw: ran.append(raw.value) or 0, (), (), gpu=1)
    with pytest.raises(ValueError):
        call()
    now[0] = 1
    call()
    call(9)
    assert ran == [4, 9] and gl._on_this_gpu(T("cuda:1")) == 1


def test_prepared_calls_hand_on_the_same_values(gl, monkeypatch):
    """Converted once instead of on every call: refusals come back as from the call itself, whatever the type of an argument."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda gpu: 0, raising=False)
    r = ctypes.byref
    x, w, out, q = _ap(gl, (4, 64), 1, gl.GL_BF16), _f8(gl, (6, 64), 1), _ap(gl, (4, 6), 2, gl.GL_F32), _f8(gl, (4, 64), 1)
    plan, t = gl.rotary_plan(16), _ap(gl, (2, 3, 4, 40), 3, gl.GL_BF16)
    cases = [(gl.LIB.gl_compute_norm_rms, (r(x), None, None, -1.0, None, r(x)), 4), (gl.LIB.gl_compute_norm_rms, (None, None, None, 1.0, None, r(x)), 1),
             (gl.LIB.gl_dense_f8, (r(x), r(w), r(out), 0x400, 0x4000, 1 << 20), 7), (gl.LIB.gl_dense_f8, (r(x), r(w), r(out), 0, 0x4000, 8), 8),
             (gl.LIB.gl_cartesian_dot_f8, (r(q), r(w), r(out), gl.GL_OUT_BF16), 2),
             (gl.LIB.gl_compute_rotate, (r(t), 159, r(plan), 0x1000, r(t), 0, 0), 4), (gl.LIB.gl_f8_quantize, (r(x), r(w)), 4)]
    for fn, args, code in cases:
        with pytest.raises(gl.GlError) as e:
            gl.Prepared(fn, args, (), gpu=0)()
        assert e.value.code == code and fn.__name__ in str(e.value)
        assert fn(*args, None) == code


def test_tensors_that_the_binding_refuses(gl, monkeypatch):
    monkeypatch.setattr(gl, "_on_this_gpu", lambda *t: 0)
    ap, plan = gl.AccessPattern, gl.rotary_plan(16, sections=(10, 6))
    t = ap(_made((2, 3, 4, 64), BF), 3)
    for pos in (_made((2, 2, 3), torch.int64), _made((2, 3), torch.int32), _made((1, 2, 3), torch.int32), _made((2, 2, 6), torch.int32)[..., ::2]):
        with pytest.raises(ValueError, match="positions"):
            gl._rotate_args(t, plan, pos, t, 0)
    one = ap(_made((1, 1, 4, 64), BF).expand(2, 3, 4, 64), 3)
    with pytest.raises(ValueError, match="overlap"):
        gl._rotate_args(t, plan, _made((2, 2, 3), torch.int32), one, 0)
    q = gl.f8_empty((4, 64), 1, "cpu")
    for bad in (gl.F8(q.data[:-1], q.scale, (4, 64), 1), gl.F8(q.data, q.scale[::2], (4, 64), 1), gl.F8(q.data.view(torch.int8), q.scale, (4, 64), 1)):
        with pytest.raises(ValueError, match="contiguous bytes"):
            gl._f8_struct(bad)


class _Stream:
    cuda_stream = 7


def test_storage_is_taken_on_the_stream_of_the_call(gl, monkeypatch):
    import contextlib
    ap = gl.AccessPattern
    rows, w = ap(_made((4, 64), BF), 1), gl.f8_empty((6, 64), 1, "cpu")
    a, t, plan, pos = gl.f8_empty((4, 64), 1, "cpu"), ap(_made((2, 3, 4, 64), BF), 3), gl.rotary_plan(16), _made((2, 3), torch.int32)
    calls = [lambda s: gl.gl_f8_quantize(rows, stream=s), lambda s: gl.gl_f8_dequantize(a, stream=s),
             lambda s: gl.gl_cartesian_dot_f8(a, w, stream=s), lambda s: gl.gl_dense_f8(rows, w, stream=s),
             lambda s: gl.gl_compute_norm_rms(rows, stream=s), lambda s: gl.gl_compute_norm_rms_f8(rows, stream=s),
             lambda s: gl.gl_compute_rotate(t, plan, pos, stream=s)]
    now, taken, launched = [], [], []

    @contextlib.contextmanager
    def stream(s):
        now.append(s.cuda_stream)
        yield
        now.pop()

    class Lib:
        def __getattr__(self, name):
            f = getattr(real, name)
            if name.endswith(("_workspace", "_bytes")):
                return f
            call = lambda *args: launched.append(args[-1]) or 0
            call.__name__ = name
            return call

    real, empty = gl.LIB, torch.empty
    monkeypatch.setattr(gl, "LIB", Lib())
    monkeypatch.setattr(gl, "_on_this_gpu", lambda *t: 0)
    monkeypatch.setattr(gl, "_stream", lambda s: 3 if s is None else s if isinstance(s, int) else s.cuda_stream)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda raw: _Stream() if raw == 7 else None)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: taken.append(now[-1] if now else 3) or empty(*a, **k))
    for given, raw in ((None, 3), (_Stream(), 7), (7, 7)):
        for i, call in enumerate(calls):
            del taken[:], launched[:]
            call(given)
            assert launched == [raw] and taken and set(taken) == {raw}, (i, given, taken)
