"""The 8-bit operators, the norms and the rotation together, as run_workload.Decoder8 uses them: a prompt and single tokens, every
stage against the checker on the stage's own inputs as the device holds them."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import f8, mx4
from paper_2105_09377_b200 import synth

pytestmark = pytest.mark.gpu


def _np(t):
    return t.double().cpu().numpy()


def _close(got, ref, tol):
    """|got - ref| <= tol before the rounding to bf16 (eight significant bits: half a unit is 2^-8 of the value at most)."""
    got = _np(got).reshape(ref.shape)
    assert (np.abs(got - ref) <= tol + 2.0 ** -8 * (np.abs(ref) + tol)).all()


def _product(a, w, relu=False):
    """Of rounded values: K exact products, an fp32 unit of sum |a||w| lost for each at most."""
    b = f8.rounded(w)
    ref, tol = a @ b.T, a.shape[1] * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)
    return (np.maximum(ref, 0.0) if relu else ref), tol


def _rounded(x):
    return f8.rounded(_np(x).reshape(-1, x.shape[-1]))


def test_prompt_and_tokens():
    from paper_2105_09377_b200 import binding as gl
    from paper_2105_09377_b200 import run_workload as rw
    cfg = dataclasses.replace(synth.DECODER8, name="small", batch=2, prompt=40, heads=4, kv_heads=2, hidden=384, page_tokens=16,
                              capacity=64)
    layer = rw.Decoder8(cfg, torch.device("cuda", 0), seed=9)
    values = [np.asarray(w, dtype=np.float64) for w in cfg.inputs(9)]
    weights, norms = values[1:5], values[5:]
    x, stored, width = layer.prompt, [], cfg.width
    for step in range(3):
        got = layer.step(x)
        t = x.shape[1]
        flat = lambda name: _np(got[name]).reshape(-1, width)

        def is_norm(result, y, residual, w):
            """Values of an F8 result within half a step of the code (2^-4 of the value, or 2^-10 of a scale that is at most
            2^-7 of the block's largest) of the norm, which itself is exact to 2^-17."""
            _, ref = f8.norm_rms(y, residual, w, cfg.eps)
            val = _np(gl.gl_f8_dequantize(result).tensor).reshape(ref.shape)
            blocks = np.abs(ref).reshape(ref.shape[0], -1, 128).max(-1).repeat(128, -1).reshape(ref.shape)
            assert (np.abs(val - ref) <= (2.0 ** -4 + 2.0 ** -16) * np.abs(ref) + 2.0 ** -16 * blocks).all()
            return val

        a = is_norm(got["first"], _np(x).reshape(-1, width), None, norms[0])
        _close(got["raw"].reshape(a.shape[0], -1), *_product(a, weights[0]))
        raw, turned = _np(got["raw"]), cfg.heads + cfg.kv_heads
        at = np.broadcast_to(np.arange(t) + (0 if step == 0 else cfg.prompt + step - 1), (1, cfg.batch, t))
        ref = f8.rotate(raw[:, :, :turned], at, list(layer.plan.step[:32]), [0] * 32, False)
        mag = np.abs(raw[:, :, :turned])
        size = np.tile(mag[..., :32] + mag[..., 32:], 2)
        _close(got["qkv"][:, :, :turned], ref, 2.0 ** -21 * size)
        assert np.array_equal(_np(got["qkv"])[:, :, turned:], raw[:, :, turned:])
        q, k, v = np.split(_np(got["qkv"]), [cfg.heads, turned], 2)
        stored.append((mx4.rounded(k), mx4.rounded(v)))
        keys, vals = (np.concatenate([s[i] for s in stored], 1) for i in (0, 1))
        for b in range(cfg.batch):
            n = keys.shape[1]
            ref, mag = mx4.attend(q[b], keys[b], vals[b], cfg.heads // cfg.kv_heads, cfg.head_dim ** -0.5, n - t)
            worst = cfg.head_dim ** -0.5 * np.abs(q[b]).max() * np.abs(keys[b]).max() * cfg.head_dim
            _close(got["seen"][b], ref, (2 * 10 * 2.0 ** -23 * worst + 2.0 ** -8) * mag)
        _close(got["y"], *_product(_rounded(got["seen"].reshape(-1, width)), weights[1]))
        h = flat("y") + _np(x).reshape(-1, width)
        assert (np.abs(flat("total") - h) <= (2.0 ** -8 + 2.0 ** -16) * np.abs(h)).all()
        a = is_norm(got["second"], flat("y"), _np(x).reshape(-1, width), norms[1])
        _close(got["hidden"], *_product(a, weights[2], relu=True))
        _close(got["down"], *_product(_rounded(got["hidden"]), weights[3]))
        _, ref = f8.norm_rms(flat("down"), flat("total"), norms[2], cfg.eps)
        _close(got["out"], ref, 2.0 ** -17 * np.abs(ref))
        x = got["out"][:, -1:].contiguous()
    assert layer.lengths.tolist() == [42, 42] and gl.gl_poll_device_status() == 0
