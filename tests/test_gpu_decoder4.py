"""The 4-bit operators together, as run_workload.Decoder4 uses them: a prompt and single tokens, every stage against the
checker on the stage's own inputs as the device holds them."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import mx4
from paper_2105_09377_b200 import synth

pytestmark = pytest.mark.gpu


def _close(got, ref, tol):
    """|got - ref| <= tol before the rounding to bf16 (eight significant bits: half a unit is 2^-8 of the value at most)."""
    got = got.double().cpu().numpy().reshape(ref.shape)
    assert (np.abs(got - ref) <= tol + 2.0 ** -8 * (np.abs(ref) + tol)).all()


def _dense(x, w, relu=False):
    a, b = mx4.rounded(x.double().cpu().numpy().reshape(-1, x.shape[-1])), mx4.rounded(w)
    ref, tol = a @ b.T, (a.shape[1] / 32 + 2) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)
    return (np.maximum(ref, 0.0) if relu else ref), tol


def test_prompt_and_tokens():
    from paper_2105_09377_b200 import binding as gl
    from paper_2105_09377_b200 import run_workload as rw
    cfg = dataclasses.replace(synth.DECODER4, name="small", batch=2, prompt=40, heads=4, kv_heads=2, hidden=384, page_tokens=16,
                              capacity=64)
    layer = rw.Decoder4(cfg, torch.device("cuda", 0), seed=9)
    weights = [np.asarray(w, dtype=np.float64) for w in cfg.inputs(9)[1:]]
    x, stored = layer.prompt, []
    for step in range(3):
        got = layer.step(x)
        t = x.shape[1]
        _close(got["qkv"], *_dense(x, weights[0]))
        qkv = got["qkv"].double().cpu().numpy()
        q, k, v = np.split(qkv, [cfg.heads, cfg.heads + cfg.kv_heads], 2)
        stored.append((mx4.rounded(k), mx4.rounded(v)))
        keys, values = (np.concatenate([s[i] for s in stored], 1) for i in (0, 1))
        for b in range(cfg.batch):
            n = keys.shape[1]
            ref, mag = mx4.attend(q[b], keys[b], values[b], cfg.heads // cfg.kv_heads, cfg.head_dim ** -0.5, n - t)
            # scores of 64 products, fp32; weights of 8 bits where more than 32 rows share a kv head
            worst = cfg.head_dim ** -0.5 * np.abs(q[b]).max() * np.abs(keys[b]).max() * cfg.head_dim
            _close(got["seen"][b], ref, (2 * 10 * 2.0 ** -23 * worst + 2.0 ** -8) * mag)
        _close(got["y"], *_dense(got["seen"].reshape(cfg.batch, t, -1), weights[1]))
        _close(got["hidden"], *_dense(got["y"], weights[2], relu=True))
        _close(got["out"], *_dense(got["hidden"], weights[3]))
        x = got["out"][:, -1:].contiguous()
    assert layer.lengths.tolist() == [42, 42] and gl.gl_poll_device_status() == 0
