"""Rotary positions with several axes, against the 64-bit checker (exact fractions of a turn)."""
import numpy as np
import pytest
import torch

from oracle import f8
from paper_2105_09377_b200 import synth

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import binding
    return binding


def _device(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(dtype)


def _np(t):
    return t.double().cpu().numpy()


def _check(got, x, positions, plan, back=False):
    """Angle: rounded to 2^-24 of at most half a turn, pi 2^-24; cosine and sine: two units more, 2^-22 in all; two products and
    their sum: 3 2^-24; then half a unit of the type.  Copied values are equal."""
    p = plan.pairs
    ref = f8.rotate(_np(x), positions.cpu().numpy(), list(plan.step[:p]), list(plan.axis[:p]), bool(plan.adjacent), back)
    mag = np.abs(_np(x))
    first, second = (slice(0, 2 * p, 2), slice(1, 2 * p, 2)) if plan.adjacent else (slice(0, p), slice(p, 2 * p))
    size = np.zeros_like(mag)
    size[..., first] = size[..., second] = mag[..., first] + mag[..., second]
    tol = (np.pi * 2.0 ** -24 + 2.0 ** -22 + 3 * 2.0 ** -24) * size
    tol += (2.0 ** -8 if x.dtype == BF else 2.0 ** -24) * (np.abs(ref) + tol) * (size > 0)
    assert (np.abs(_np(got) - ref) <= tol).all(), np.abs(_np(got) - ref).max()
    assert torch.equal(got[..., 2 * p:], x[..., 2 * p:])


def _positions(axes, b, t, far, seed):
    g = np.random.default_rng(seed)
    return torch.from_numpy(g.integers(-far if far < 2 ** 31 else -2 ** 31, far, (axes, b, t)).astype(np.int32)).cuda()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("b,t,heads,d,pairs,sections", [
    (1, 1, 1, 2, 1, (1,)), (2, 1, 5, 128, 64, (64,)), (1, 3, 2, 64, 32, (12, 10, 10)), (3, 5, 40, 128, 64, (16, 24, 24)),
    (1, 7, 3, 80, 20, (20,)), (2, 2, 4, 48, 24, (6, 6, 6, 6)), (1, 4, 1, 96, 33, (30, 3)), (1, 2, 3, 256, 128, (128,)),
    (2, 3, 3, 10, 3, (1, 1, 1)), (1, 5, 2, 7, 3, (0, 3)), (1, 2, 700, 8, 4, (4,)), (1, 37, 8, 64, 32, (32,))])
def test_against_the_formula(gl, b, t, heads, d, pairs, sections, adjacent, dtype):
    plan = gl.rotary_plan(pairs, 10000.0, sections, adjacent)
    x = _device(synth.normal(31, b * 100 + t * 10 + d, (b, t, heads, d)), dtype)
    pos = _positions(len(sections), b, t, 5000, d)
    _check(gl.gl_compute_rotate(gl.AccessPattern(x, 3), plan, pos).tensor, x, pos, plan)
    back = gl.gl_compute_rotate(gl.AccessPattern(x, 3), plan, pos, flags=gl.GL_ROTATE_BACK).tensor
    _check(back, x, pos, plan, back=True)


def test_far_positions_and_own_frequencies(gl):
    x = _device(synth.normal(33, 1, (1, 300, 2, 64)), F32)
    pos = _positions(1, 1, 300, 2 ** 31, 5)
    pos[0, 0, :4] = torch.tensor([2 ** 31 - 1, -2 ** 31, 0, 1 << 20], dtype=torch.int32)
    for plan in (gl.rotary_plan(32, 500000.0), gl.rotary_plan(32, freq=list(np.linspace(-7.0, 20.0, 32)))):
        _check(gl.gl_compute_rotate(gl.AccessPattern(x, 3), plan, pos[0]).tensor, x, pos, plan)


def test_parts_of_a_projection_in_place_and_out(gl):
    """Queries and keys of a fused projection are turned where they are; values, and what lies between tokens, stay."""
    plan = gl.rotary_plan(32, 10000.0, (8, 12, 12))
    for dtype in (BF, F32):
        qkv = _device(synth.normal(34, 2, (3, 19, 12, 64)), dtype)
        pos = _positions(3, 3, 19, 4000, 6)
        before = qkv.clone()
        dense = gl.gl_compute_rotate(gl.AccessPattern(qkv[:, :, :9], 3), plan, pos).tensor
        _check(dense, before[:, :, :9].contiguous(), pos, plan)
        assert torch.equal(qkv, before)
        part = gl.AccessPattern(qkv[:, :, :9], 3)
        gl.gl_compute_rotate(part, plan, pos, part)
        assert torch.equal(qkv[:, :, :9], dense) and torch.equal(qkv[:, :, 9:], before[:, :, 9:])
        # into the middle of something wider, guarded
        wide = torch.full((3, 19, 20, 64), 7.0, dtype=dtype, device="cuda")
        gl.gl_compute_rotate(gl.AccessPattern(before[:, :, :9], 3), plan, pos, gl.AccessPattern(wide[:, :, 4:13], 3))
        assert torch.equal(wide[:, :, 4:13], dense) and (wide[:, :, :4] == 7).all() and (wide[:, :, 13:] == 7).all()


def test_partial_rotation_in_place(gl):
    """Values behind the pairs are neither read nor written in place."""
    plan = gl.rotary_plan(16, 10000.0)
    x = _device(synth.normal(35, 3, (2, 5, 3, 100)), BF)
    pos = _positions(1, 2, 5, 99, 7)
    before, a = x.clone(), gl.AccessPattern(x, 3)
    gl.gl_compute_rotate(a, plan, pos, a)
    _check(x, before, pos, plan)


def test_odd_distances_between_tokens(gl):
    """A distance that is no multiple of 16 bytes: narrower accesses."""
    plan = gl.rotary_plan(8, 10000.0)
    for extra in (1, 2, 4, 8):
        store = _device(synth.normal(36, extra, (6, 2 * 16 + extra)), BF)
        x = store.as_strided((1, 6, 2, 16), (6 * (32 + extra), 32 + extra, 16, 1))
        pos = _positions(1, 1, 6, 77, extra)
        _check(gl.gl_compute_rotate(gl.AccessPattern(x, 3), plan, pos).tensor, x.contiguous(), pos, plan)


def test_the_gradient_is_the_rotation_back(gl):
    """d/dx of sum(g . rotate(x)) by differences (the rotation is linear: any step is exact) and there and back again."""
    plan = gl.rotary_plan(16, 10000.0, (10, 6), True)
    x, g = (_device(synth.normal(37, i, (1, 4, 2, 40)), F32) for i in (1, 2))
    pos = _positions(2, 1, 4, 1000, 8)
    turn = lambda v, f=0: gl.gl_compute_rotate(gl.AccessPattern(v.contiguous(), 3), plan, pos, flags=f).tensor
    grad = _np(turn(g, gl.GL_ROTATE_BACK))
    base = _np(turn(x))
    for at in ((0, 0, 0, 0), (0, 1, 1, 7), (0, 3, 0, 31), (0, 2, 1, 39)):
        moved = x.clone()
        moved[at] += 1.0
        assert abs(((_np(turn(moved)) - base) * _np(g)).sum() - grad[at]) < 40 * 2.0 ** -22 * 5
    again = turn(turn(x), gl.GL_ROTATE_BACK)
    assert ((again - x).abs() <= 2.0 ** -19 * x.abs().amax()).all()


def test_many_tokens(gl):
    """Several tokens a block, a ragged last block, more than one round of tasks: equal to one token at a time."""
    for b, t, heads, d, dtype in ((2, 4099, 3, 64, BF), (1, 1500, 40, 128, BF), (1, 5000, 1, 32, F32)):
        plan = gl.rotary_plan(d // 2, 500000.0, (d // 2 - 4, 4))
        x = torch.randn((b, t, heads, d), generator=torch.Generator("cuda").manual_seed(t), device="cuda").to(dtype)
        pos = _positions(2, b, t, 100000, 9)
        got = gl.gl_compute_rotate(gl.AccessPattern(x, 3), plan, pos).tensor
        for i in (0, 1, t // 2, t - 1):
            one = x[:, i:i + 1].contiguous()
            want = gl.gl_compute_rotate(gl.AccessPattern(one, 3), plan, pos[:, :, i:i + 1].contiguous()).tensor
            assert torch.equal(got[:, i:i + 1], want)
            _check(want, one, pos[:, :, i:i + 1].contiguous(), plan)


def test_graph_and_stream(gl):
    plan = gl.rotary_plan(32)
    x, pos = torch.randn(4, 1, 6, 64, device="cuda").to(BF), torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    out = gl.AccessPattern(torch.empty_like(x), 3)
    call = gl.prepare_compute_rotate(gl.AccessPattern(x, 3), plan, pos, out)
    call()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        call()
    for step in range(3):
        pos += 1
        torch.cuda.synchronize()
        graph.replay()
        mine = gl.gl_compute_rotate(gl.AccessPattern(x, 3), plan, pos, stream=side).tensor
        torch.cuda.synchronize()
        assert torch.equal(out.tensor, mine)
        _check(mine, x, pos[None], plan)


def test_beyond_two_to_the_31_values(gl):
    plan = gl.rotary_plan(64)
    x = torch.ones((1, 270000, 64, 128), dtype=BF, device="cuda")
    pos = torch.zeros((1, 270000), dtype=torch.int32, device="cuda")
    pos[0, -5:] = 123
    a = gl.AccessPattern(x, 3)
    gl.gl_compute_rotate(a, plan, pos, a)
    assert (x[0, :-5] == 1).all()
    one = torch.ones((1, 5, 64, 128), dtype=BF, device="cuda")
    _check(x[:, -5:].contiguous(), one, pos[None, :, -5:].contiguous(), plan)
