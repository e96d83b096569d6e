"""Calls given a stream of their own, without a workspace: each result is that of the same call alone."""
import numpy as np
import pytest
import torch

from paper_2105_09377_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import binding
    return binding


def _bf16(seed, shape):
    return torch.from_numpy(synth.normal(seed, 1, shape).astype(np.float32)).cuda().to(torch.bfloat16)


def _dense(gl):
    w = gl.gl_mx4_quantize(gl.AccessPattern(_bf16(1, (2048, 2048)), 1))
    xs = [gl.AccessPattern(_bf16(2 + i, (1000, 2048)), 1) for i in range(2)]
    return [lambda s, x=x: gl.gl_dense_mx4(x, w, flags=gl.GL_OUT_BF16, stream=s).tensor for x in xs]


def _attend(gl):
    lens, d, page = [9000, 300], 128, 64
    width = -(-max(lens) // page)
    cache = gl.cache4_empty(2 * width, 2, page, d, "cuda")
    table = torch.arange(2 * width, dtype=torch.int32, device="cuda").view(2, width)
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    gl.gl_cache4_append(cache, _bf16(5, (2, 9000, 2, d)), _bf16(6, (2, 9000, 2, d)), table, lengths)
    qs = [gl.AccessPattern(_bf16(7 + i, (2, 2, 8, d)), 3) for i in range(2)]
    return [lambda s, q=q: gl.gl_attend_cache4(q, cache, table, lengths, stream=s).tensor for q in qs]


def _conv(gl):
    w, win = gl.AccessPattern(_bf16(1, (64, 64, 3, 3)), 1), gl.windows_spec((64, 3, 3), (1, 1, 1))
    xs = [gl.AccessPattern(_bf16(2 + i, (8, 64, 40, 40)), 1) for i in range(2)]
    assert gl.gl_cartesian_dot_workspace(xs[0], win, w) > 0
    return [lambda s, x=x: gl.gl_cartesian_dot(x, win, w, stream=s).tensor for x in xs]


@pytest.mark.parametrize("make", [_dense, _attend, _conv])
def test_two_streams_without_a_workspace(gl, make):
    calls = make(gl)
    alone = []
    for call in calls:
        alone.append(call(None).clone())
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(12):
        for call, s in zip(calls, streams):
            got.append(call(s))
        # what the current stream is handed next is not what the others still use
        torch.empty(64 << 20, dtype=torch.uint8, device="cuda").fill_(0x7F)
    torch.cuda.synchronize()
    for i, y in enumerate(got):
        assert torch.equal(y, alone[i % 2]), i
    # a raw address, as another library has it
    y = calls[0](streams[0].cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(y, alone[0]) and gl.gl_poll_device_status() == 0


def test_prepared_calls_on_two_streams(gl):
    """Prepared calls keep their scratch; dropped while the other stream still runs, it is not handed out."""
    w = gl.gl_mx4_quantize(gl.AccessPattern(_bf16(1, (2048, 2048)), 1))
    x = gl.AccessPattern(_bf16(2, (1000, 2048)), 1)
    want = gl.gl_dense_mx4(x, w).tensor
    torch.cuda.synchronize()
    side, outs = torch.cuda.Stream(), []
    for _ in range(8):
        outs.append(gl.AccessPattern(torch.empty_like(want), 2))
        side.wait_stream(torch.cuda.current_stream())
        call = gl.prepare_dense_mx4(x, w, outs[-1])
        call(side)
        del call
        torch.empty(gl.gl_dense_mx4_workspace(x, w) + 1024, dtype=torch.uint8, device="cuda").fill_(0x7F)
    torch.cuda.synchronize()
    assert all(torch.equal(o.tensor, want) for o in outs)
