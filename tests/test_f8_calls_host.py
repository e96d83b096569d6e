"""Calls on 8-bit operands, the norm and the rotation that are refused or hold on to nothing of their caller's, checked on the host."""
import sys

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
