"""Calls on 8-bit operands, the norm and the rotation that are refused or hold on to nothing of their caller's, checked on the host."""
import ctypes
import random
import sys
from decimal import Decimal, getcontext
from fractions import Fraction

import pytest
import torch

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import build
    build.build()
    from paper_2105_09377_b200 import binding
    return binding


def _tokens(gl, shape=(2, 3, 4, 64)):
    return gl.AccessPattern(torch.zeros(shape, dtype=BF), 3)


# ---- positions ----

def test_positions_are_counted_with_every_number_of_axes(gl, monkeypatch):
    """A single number is not [axes, batch, tokens]: the kernel would read behind it."""
    monkeypatch.setattr(gl, "_on_this_gpu", lambda *t: 0)
    t = _tokens(gl)
    for sections in ((16,), (10, 6), (4, 4, 8)):
        plan = gl.rotary_plan(16, sections=sections)
        n = len(sections)
        for shape in ((), (1,), (n,), (n, 6), (n, 2, 3, 1), (n + 1, 2, 3), (n, 3, 2), (3,)):
            with pytest.raises(ValueError, match="positions"):
                gl._rotate_args(t, plan, torch.zeros(shape, dtype=torch.int32), t, 0)
        gl._rotate_args(t, plan, torch.zeros((n, 2, 3), dtype=torch.int32), t, 0)
    gl._rotate_args(t, gl.rotary_plan(16), torch.zeros((2, 3), dtype=torch.int32), t, 0)


def test_a_prepared_rotation_keeps_its_own_plan(gl, monkeypatch):
    """The positions were counted for the plan as it was: axes that its caller adds later would be read behind them."""
    monkeypatch.setattr(gl, "_on_this_gpu", lambda *t: 0)
    plan, t = gl.rotary_plan(16), _tokens(gl)
    args = gl._rotate_args(t, plan, torch.zeros((1, 2, 3), dtype=torch.int32), t, 0)
    step = plan.step[3]
    plan.axes, plan.axis[3], plan.step[3] = 2, 1, 5
    held = args[2]._obj
    assert (held.axes, held.axis[3], held.step[3], held.pairs) == (1, 0, step, 16)


# ---- prepared calls that threads share ----

def test_a_prepared_call_keeps_to_its_own_stream(gl, monkeypatch):
    """Another call of the same object, on another stream, between any two lines of this one (as a thread that takes over there
    makes it): each goes to the stream that it was given."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda gpu: 3, raising=False)
    ran = []
    call = gl.Prepared(lambda raw: ran.append(raw.value) or 0, (), (), gpu=0)
    between = [0]

    def other(frame, event, arg):
        if event in ("line", "return") and frame.f_code.co_filename == gl.__file__:
            sys.settrace(None)
            call(1000 + between[0])
            between[0] += 1
            sys.settrace(other)
        return other

    for given, raw in ((7, 7), (None, 3), (8, 8)):
        del ran[:]
        between[0] = 0
        sys.settrace(other)
        try:
            call(given)
        finally:
            sys.settrace(None)
        assert between[0] >= 5 and sorted(ran) == [raw] + [1000 + i for i in range(between[0])], (given, ran)


# ---- places that operands and results share ----

UNSUPPORTED = 7


def _norm(gl, x, out, residual=None, total=None, weight=None):
    """Status of a norm of (4, 64): operands as (type, address), an F8 result as a pair of addresses."""
    r = ctypes.byref
    at = lambda a, shape=(4, 64): None if a is None else r(gl._meta(shape, len(shape) - 1, a[0], a[1]))
    args = (at(x), at(residual), at(weight, (64,)), 1e-5, at(total))
    if out[0] in (gl.GL_F32, gl.GL_BF16):
        return gl.LIB.gl_compute_norm_rms(*args, at(out), None)
    q = gl._f8_meta((4, 64), 1)
    q.data, q.scale = out
    return gl.LIB.gl_compute_norm_rms_f8(*args, r(q), None)


def test_a_norm_in_place_of_another_type_is_refused(gl):
    """Rows lie at other distances in the two views, so a block would write over rows that another has not read."""
    b, f, a = gl.GL_BF16, gl.GL_F32, 0x100000
    away, far = (f, 0x800000), (f, 0x900000)
    for x, out, more in (((b, a), (f, a), {}), ((f, a), (b, a), {}),                          # the result in x's place
                         (away, (b, a), dict(residual=(f, a))), (away, (f, a), dict(residual=(b, a))),
                         ((b, a), away, dict(residual=far, total=(f, a))),                    # the sum in x's place
                         ((f, a), away, dict(residual=(b, 0x900000), total=(b, a)))):
        assert _norm(gl, x, out, **more) == UNSUPPORTED, (x, out, more)


def test_a_norm_beside_itself_is_refused(gl):
    """A row further on, or half of one: neither the same place nor another."""
    f, a, size, far = gl.GL_F32, 0x100000, 4 * 64 * 4, (gl.GL_F32, 0x900000)
    for d in (16, 256, size - 16, -16, -256, 16 - size):
        assert _norm(gl, (f, a), (f, a + d)) == UNSUPPORTED, d
        assert _norm(gl, far, (f, a + d), residual=(f, a)) == UNSUPPORTED, d
        assert _norm(gl, far, (f, 0x800000), residual=(f, a), total=(f, a + d)) == UNSUPPORTED, d
        assert _norm(gl, (f, a), (f, 0x800000), residual=far, total=(f, a + d)) == UNSUPPORTED, d
        assert _norm(gl, (f, 0x700000), (f, a + d), residual=far, total=(f, a)) == UNSUPPORTED, d
    weight = (f, a + 128)                                                                     # 256 bytes
    for out in (a, a + 368, a - size + 144):
        assert _norm(gl, far, (f, out), weight=weight) == UNSUPPORTED
        assert _norm(gl, far, (f, 0x800000), residual=(f, out), total=(f, out), weight=weight) == UNSUPPORTED


def test_a_norm_into_f8_over_its_operands_is_refused(gl):
    """(4, 64): 256 bytes of codes, 512 of scales."""
    f, b, a, far = gl.GL_F32, gl.GL_BF16, 0x100000, (gl.GL_F32, 0x900000)
    for codes, scales in ((a, 0x800000), (0x800000, a), (a + 512 - 16, 0x800000), (0x800000, a - 512 + 16)):
        assert _norm(gl, (b, a), (codes, scales)) == UNSUPPORTED
        assert _norm(gl, far, (codes, scales), residual=(b, a)) == UNSUPPORTED
        assert _norm(gl, far, (codes, scales), residual=(b, 0xA00000), total=(b, a)) == UNSUPPORTED
    assert _norm(gl, far, (a, 0x800000), weight=(f, a)) == UNSUPPORTED and _norm(gl, far, (0x800000, a), weight=(f, a)) == UNSUPPORTED
    assert _norm(gl, far, (a, a + 240)) == UNSUPPORTED and _norm(gl, far, (a + 496, a)) == UNSUPPORTED


def _rotate(gl, n, width, x, px, out, po):
    """Status of a rotation of n tokens of `width` bf16 values, the operand's from element x on, the result's from `out` on."""
    r, base = ctypes.byref, 0x10000000
    at = lambda where: r(gl._meta((1, n, 1, width), 3, gl.GL_BF16, base + 2 * where))
    return gl.LIB.gl_compute_rotate(at(x), px, r(gl.rotary_plan(4)), 0x1000, at(out), po, 0, None)


def test_a_rotation_beside_itself_is_refused(gl):
    """Views of one projection that share values without being one view: blocks would read what others have turned."""
    heads = 64
    for d in (8, heads, 2 * heads, 5 * heads, 8 * heads - 8, 10 * heads + 8, 12 * heads, 9 * 12 * heads, -heads, -12 * heads, 4 * heads - 12 * heads - 8):
        # eight heads of twelve, turned into a view d elements on: the next head, the next token, ..
        assert _rotate(gl, 19, 8 * heads, 4096, 12 * heads, 4096 + d, 12 * heads) == UNSUPPORTED, d
    assert _rotate(gl, 1, 64, 0, 64, 56, 64) == UNSUPPORTED and _rotate(gl, 1, 64, 56, 64, 0, 64) == UNSUPPORTED
    # other distances: the last token of one, or one in the middle, meets a token of the other
    assert _rotate(gl, 10, 64, 0, 64, 568, 200) == UNSUPPORTED and _rotate(gl, 10, 64, 1800, 64, 0, 200) == UNSUPPORTED
    assert _rotate(gl, 12, 64, 0, 200, 64, 208) == UNSUPPORTED and _rotate(gl, 3, 8, 8, 1000, 0, 504) == UNSUPPORTED


def test_which_tokens_meet(gl):
    """The refusal is exact: against every pair of tokens.  (No call that is not refused reaches a GPU here.)"""
    rng, seen = random.Random(5), {False: 0, True: 0}
    for _ in range(4000):
        n, width = rng.choice([1, 2, 3, 7, 20]), rng.choice([8, 16, 24])
        px, po = (width + rng.choice([0, 8, 16, 24, 40, 64, 200]) for _ in range(2))
        if rng.random() < 0.5:
            po = px
        x, out = 8 * rng.randrange(80), 8 * rng.randrange(80)
        if x == out:
            continue
        meet = any(x + i * px < out + j * po + width and out + j * po < x + i * px + width for i in range(n) for j in range(n))
        assert (_rotate(gl, n, width, x, px, out, po) == UNSUPPORTED) == meet, (n, width, x, px, out, po)
        seen[meet] += 1
    assert min(seen.values()) > 500


# ---- the rotary plan ----

def _two_pi():
    """2 pi to 400 bits: 16 atan(1/5) - 4 atan(1/239), times two."""
    one = 1 << 440

    def atan_inverse(n):
        term, total, k = one // n, 0, 1
        while term:
            total += term // k if k % 4 == 1 else -(term // k)
            term, k = term // (n * n), k + 2
        return total

    return Fraction(2 * (16 * atan_inverse(5) - 4 * atan_inverse(239)), one)


def _off(step, turns):
    """Distance of a step from 2^64 turns, in units, whole turns aside."""
    d = (Fraction(step) - turns * 2 ** 64) % 2 ** 64
    return float(min(d, 2 ** 64 - d))


def test_steps_of_own_frequencies(gl):
    """Off by half a unit of 2^-64 turns and |freq| 2^-62 units, as gl.h has it, whatever whole turns a position makes."""
    freqs = [20.0, 7.0, 1e6, -1e6, 1e12, 1e15 + 0.1, -3e-5, 1e-12, 0.0, 2.0 ** 40 + 0.37, 6.283185307179586, -6.283185307179587, 1.0, -1.0,
             2.0 ** -70] + [(-1) ** i * 1.37 ** (i - 30) for i in range(100)]
    plan, two_pi = gl.rotary_plan(len(freqs), freq=freqs), _two_pi()
    for i, f in enumerate(freqs):
        assert _off(plan.step[i], Fraction(f) / two_pi) <= 0.5 + abs(f) * 2.0 ** -62 + 1e-9, f
    huge = gl.rotary_plan(3, freq=[1e300, -1e300, 2.0 ** 66])     # (finite: some angle, the same every time)
    assert list(huge.step[:3]) == list(gl.rotary_plan(3, freq=[1e300, -1e300, 2.0 ** 66]).step[:3])


def test_steps_of_a_base(gl):
    """Off by two thirds of a unit at most: half a unit of the step and what the power is off by."""
    getcontext().prec = 60
    two_pi = _two_pi()
    two_pi = Decimal(two_pi.numerator) / Decimal(two_pi.denominator)
    for pairs, base in ((128, 10000.0), (64, 500000.0), (128, 1e30), (31, 1.5)):
        plan = gl.rotary_plan(pairs, base)
        for i in range(pairs):
            want = Decimal(base) ** (Decimal(-i) / Decimal(pairs)) / two_pi * 2 ** 64
            assert abs(Decimal(plan.step[i]) - want) <= Decimal(2) / 3, (pairs, base, i)
