"""The first calls of a process come from several host threads at once, each on a stream of its own."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

PROGRAM = r"""
import threading
import numpy as np
import torch
from paper_2105_09377_b200 import binding as gl, synth

def bf16(seed, shape):
    return torch.from_numpy(synth.normal(seed, 1, shape).astype(np.float32)).cuda().to(torch.bfloat16)

xs = {m: bf16(m, (m, 512)) for m in (3, 40, 300, 2000)}
w = gl.AccessPattern(bf16(1, (2048, 512)), 1)
k, v, table = bf16(2, (2, 500, 2, 128)), bf16(3, (2, 500, 2, 128)), torch.arange(64, dtype=torch.int32).view(2, 32).cuda()
lengths = torch.tensor([500, 77], dtype=torch.int32, device="cuda")
qs = {t: gl.AccessPattern(bf16(10 + t, (2, t, 8, 128)), 3) for t in (1, 3, 20)}
torch.cuda.synchronize()

def work(stream):
    wq = gl.gl_mx4_quantize(w, stream=stream)
    out = [gl.gl_dense_mx4(gl.AccessPattern(x, 1), wq, flags=f, stream=stream).tensor for x in xs.values() for f in (0, gl.GL_OUT_BF16)]
    cache = gl.cache4_empty(64, 2, 16, 128, "cuda")
    gl.gl_cache4_append(cache, k, v, table, lengths, stream=stream)
    out += [gl.gl_attend_cache4(q, cache, table, lengths, flags=f, stream=stream).tensor for q in qs.values() for f in (0, gl.GL_OUT_BF16)]
    return out, (wq, cache)

threads, results, start = 4, {}, threading.Barrier(4)

def run(i, stream):
    start.wait()
    try:
        results[i] = work(stream)
    except Exception as e:
        results[i] = e

streams = [torch.cuda.Stream() for _ in range(threads)]
ts = [threading.Thread(target=run, args=(i, s)) for i, s in enumerate(streams)]
[t.start() for t in ts]
[t.join() for t in ts]
torch.cuda.synchronize()
want, _ = work(None)
torch.cuda.synchronize()
for i in range(threads):
    if isinstance(results[i], Exception):
        raise results[i]
    for got, ref in zip(results[i][0], want):
        assert torch.equal(got, ref), i
assert gl.gl_poll_device_status() == 0
print("ok")
"""


def test_first_calls_from_several_threads():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    for _ in range(2):
        r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0 and r.stdout.strip() == "ok", r.stderr[-2000:]
