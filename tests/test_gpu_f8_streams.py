"""The 8-bit operators, the norm and the rotation on streams of their own and from several host threads: each result is that of
the same call alone."""
import os
import subprocess
import sys

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


def _calls(gl):
    """Every kind of kernel, as functions of the stream; a 4-bit product and a bf16 one in between, whose blocks share the SMs."""
    ap = gl.AccessPattern
    w, w4, wide = gl.gl_f8_quantize(ap(_bf16(1, (2048, 2048)), 1)), gl.gl_mx4_quantize(ap(_bf16(1, (2048, 2048)), 1)), ap(_bf16(1, (2048, 2048)), 1)
    xs = {m: ap(_bf16(2 + m, (m, 2048)), 1) for m in (1, 3, 40, 100, 300, 1500)}
    res, weight = ap(_bf16(5, (300, 2048)), 1), ap(_bf16(6, (2048,)), 0)
    t, pos, plan = ap(_bf16(7, (2, 300, 6, 64)), 3), torch.arange(600, dtype=torch.int32, device="cuda").view(1, 2, 300), gl.rotary_plan(32)
    calls = [lambda s, x=x: gl.gl_dense_f8(x, w, flags=gl.GL_OUT_BF16, stream=s).tensor for x in xs.values()]
    calls += [lambda s: gl.gl_dense_mx4(xs[40], w4, stream=s).tensor, lambda s: gl.gl_cartesian_dot(xs[300], None, wide, stream=s).tensor]
    calls += [lambda s: gl.gl_compute_norm_rms(xs[300], weight, 1e-5, res, stream=s).tensor,
              lambda s: gl.gl_cartesian_dot_f8(gl.gl_compute_norm_rms_f8(xs[300], weight, 1e-5, res, stream=s), w, stream=s).tensor,
              lambda s: gl.gl_compute_rotate(t, plan, pos, stream=s).tensor]
    return calls


def test_three_streams_without_a_workspace(gl):
    calls = _calls(gl)
    alone = []
    for call in calls:
        alone.append(call(None).clone())
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for turn in range(6):
        for i in range(len(calls)):
            for j, s in enumerate(streams):
                k = (i + 4 * j + turn) % len(calls)
                got.append((k, calls[k](s)))
        # what the current stream is handed next is not what the others still use
        torch.empty(64 << 20, dtype=torch.uint8, device="cuda").fill_(0x7F)
    torch.cuda.synchronize()
    for k, y in got:
        assert torch.equal(y, alone[k]), k
    y = calls[4](streams[0].cuda_stream)             # a raw address, as another library has it
    torch.cuda.synchronize()
    assert torch.equal(y, alone[4]) and gl.gl_poll_device_status() == 0


def test_prepared_calls_on_two_streams(gl):
    """Prepared calls keep their scratch; dropped while the other stream still runs, it is not handed out."""
    ap = gl.AccessPattern
    w, x = gl.gl_f8_quantize(ap(_bf16(1, (2048, 2048)), 1)), ap(_bf16(2, (1000, 2048)), 1)
    want = gl.gl_dense_f8(x, w).tensor
    torch.cuda.synchronize()
    side, outs = torch.cuda.Stream(), []
    for _ in range(8):
        outs.append(ap(torch.empty_like(want), 2))
        side.wait_stream(torch.cuda.current_stream())
        call = gl.prepare_dense_f8(x, w, outs[-1])
        call(side)
        del call
        torch.empty(gl.gl_dense_f8_workspace(x, w) + 1024, dtype=torch.uint8, device="cuda").fill_(0x7F)
    torch.cuda.synchronize()
    assert all(torch.equal(o.tensor, want) for o in outs)


def test_a_layer_captured_beside_an_eager_one(gl):
    """Two graphs with workspaces of their own and an eager call, all at once, on changing inputs."""
    ap = gl.AccessPattern
    w, x = gl.gl_f8_quantize(ap(_bf16(1, (1024, 1024)), 1)), torch.empty((200, 1024), dtype=torch.bfloat16, device="cuda")
    outs, graphs, streams = [], [], [torch.cuda.Stream() for _ in range(3)]
    for _ in range(2):
        q, out = gl.f8_empty((200, 1024), 1, "cuda"), ap(torch.empty((200, 1024), device="cuda"), 2)
        steps = [gl.prepare_compute_norm_rms(ap(x, 1), None, q), gl.prepare_cartesian_dot_f8(q, w, out),
                 gl.prepare_dense_f8(ap(out.tensor, 1), w, other := ap(torch.empty((200, 1024), device="cuda"), 2))]
        [step() for step in steps]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            [step() for step in steps]
        graphs.append((g, steps))
        outs.append(other)
    for seed in range(4):
        x.copy_(torch.randn((200, 1024), generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
        torch.cuda.synchronize()
        for (g, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        first = gl.gl_cartesian_dot_f8(gl.gl_compute_norm_rms_f8(ap(x, 1), stream=streams[2]), w, stream=streams[2])
        eager = gl.gl_dense_f8(ap(first.tensor, 1), w, stream=streams[2])
        torch.cuda.synchronize()
        assert torch.equal(outs[0].tensor, eager.tensor) and torch.equal(outs[1].tensor, eager.tensor)


PROGRAM = r"""
import threading
import torch
from paper_2105_09377_b200 import binding as gl
from tests import test_gpu_f8_streams as t

calls = t._calls(gl)
torch.cuda.synchronize()
threads, results, start = 4, {}, threading.Barrier(4)

def run(i, stream):
    start.wait()
    try:
        results[i] = [calls[(k + 3 * i) % len(calls)](stream) for k in range(len(calls))]
    except Exception as e:
        results[i] = e

streams = [torch.cuda.Stream() for _ in range(threads)]
ts = [threading.Thread(target=run, args=(i, s)) for i, s in enumerate(streams)]
[x.start() for x in ts]
[x.join() for x in ts]
torch.cuda.synchronize()
want = [call(None) for call in calls]
torch.cuda.synchronize()
for i in range(threads):
    if isinstance(results[i], Exception):
        raise results[i]
    for k, got in enumerate(results[i]):
        assert torch.equal(got, want[(k + 3 * i) % len(calls)]), (i, k)
assert gl.gl_poll_device_status() == 0
print("ok")
"""


def test_first_calls_from_several_threads():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stderr[-2000:]
