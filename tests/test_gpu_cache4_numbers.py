"""GPU numerics of the attention over 4-bit pages where they are tight: weights and their sum, keys and values near the ends
of the range."""
import numpy as np
import pytest
import torch

from oracle import mx4
from paper_2105_09377_b200 import synth
from tests.test_gpu_cache4 import _to_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import binding
    return binding


def _bf16(seed, shape, std=1.0):
    return (torch.from_numpy(synth.normal(seed, 1, shape)) * std).to(torch.bfloat16).cuda()


def _stored(gl, k, v, page):
    """A cache that holds k and v, [sequences, tokens, kv heads, D] of one length; pages in shuffled order."""
    b, n, hkv, d = k.shape
    width = -(-n // page)
    table = torch.from_numpy(np.random.default_rng(n).permutation(b * width).astype(np.int32).reshape(b, width)).cuda()
    lengths = torch.full((b,), n, dtype=torch.int32, device="cuda")
    cache = gl.cache4_empty(b * width, hkv, page, d, "cuda")
    cache.data.fill_(0xFF)
    gl.gl_cache4_append(cache, k, v, table, lengths)
    return cache, table, lengths


def _row(q, k, v, scale):
    """Weights, result and sum of p |v| of one row over all tokens, in 64 bits."""
    s = scale * (k @ q)
    p = np.exp(s - s.max())
    p /= p.sum()
    return s, p, p @ v, p @ np.abs(v)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("rows,n", [(4, 60), (12, 60), (28, 60), (40, 60), (4, 9000), (28, 3000), (40, 3000)])
def test_keys_near_the_end_of_the_range(gl, rows, n, d, bf16):
    """Keys of about 2^112 under queries of many sizes, in one call: scores that are ordinary numbers (queries of 2^-112),
    scores of up to 2^120 (one token takes all), and zeros.  All of them finite, none beyond fp32."""
    v = _bf16(2, (1, n, 1, d))
    k = _bf16(1, (1, n, 1, d), 2.0 ** 112)
    if n > 100:
        k[0, 40:n - 50] = _bf16(5, (1, n - 90, 1, d))[0]      # ordinary keys before and between
    size = np.resize([2.0 ** -112, 1.0, 0.0, 2.0 ** -118, 2.0 ** -20, 2.0 ** -100], rows)
    q = (torch.from_numpy(synth.normal(3, 1, (rows, d)) * size[:, None])).to(torch.bfloat16).cuda().view(1, 1, rows, d)
    cache, table, lengths = _stored(gl, k, v, 16)
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths, flags=gl.GL_OUT_BF16 if bf16 else 0)
    got = got.tensor[0, 0].double().cpu().numpy()
    kd, vd = (mx4.rounded(x[0, :, 0].double().cpu().numpy()) for x in (k, v))
    qd = q[0, 0].double().cpu().numpy()
    assert np.isfinite(got).all()
    checked = 0
    for h in range(rows):
        s, p, ref, mag = _row(qd[h], kd, vd, d ** -0.5)
        # D products of fp32 partial sums, then two roundings, of terms of q k
        ds = (d / 16 + 6) * 2.0 ** -23 * d ** -0.5 * (np.abs(kd) @ np.abs(qd[h])).max()
        if np.abs(s).max() > 20:             # one token takes all, if it is ahead by more than the scores are off
            top = np.sort(s)[::-1]
            if top[0] - top[1] < 4 * ds + 100:
                continue
            ref, mag, ds = vd[s.argmax()], np.abs(vd[s.argmax()]), 0.0
        rel = 2 * ds + 2.0 ** -20 + (n / 16 + 16) * 2.0 ** -23 + ((2.0 ** -8 if rows > 32 else 2.0 ** -10) if bf16 else 2.0 ** -20)
        tol = rel * mag
        lo, hi = (_to_bf16(ref - tol), _to_bf16(ref + tol)) if bf16 else (ref - tol, ref + tol)
        assert ((got[h] >= lo) & (got[h] <= hi)).all(), (h, size[h], np.abs(got[h] - ref).max())
        checked += 1
    assert checked > rows / 2
    assert gl.gl_poll_device_status() == 0


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("power", [123, -100])
@pytest.mark.parametrize("rows,n", [(4, 60), (12, 130), (28, 60), (40, 200), (4, 20000), (28, 3000), (40, 3000)])
def test_values_near_the_ends_of_the_range(gl, rows, n, power, d, bf16):
    """Values of 2^123 (up to 2^126) and of 2^-100: an average of them is as large as they are, so nothing may overflow or
    get lost on the way."""
    k, q = _bf16(1, (1, n, 1, d)), _bf16(3, (1, 1, rows, d), 1.5)
    v = _bf16(2, (1, n, 1, d), 2.0 ** power)
    cache, table, lengths = _stored(gl, k, v, 16)
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths, flags=gl.GL_OUT_BF16 if bf16 else 0)
    got = got.tensor[0, 0].double().cpu().numpy()
    kd, vd = (mx4.rounded(x[0, :, 0].double().cpu().numpy()) for x in (k, v))
    qd = q[0, 0].double().cpu().numpy()
    for h in range(rows):
        s, p, ref, mag = _row(qd[h], kd, vd, d ** -0.5)
        ds = (d / 16 + 6) * 2.0 ** -23 * d ** -0.5 * (np.abs(kd) @ np.abs(qd[h])).max()
        rel = 2 * ds + 2.0 ** -20 + (n / 16 + 16) * 2.0 ** -23 + ((2.0 ** -8 if rows > 32 else 2.0 ** -10) if bf16 else 2.0 ** -20)
        tol = rel * mag
        lo, hi = (_to_bf16(ref - tol), _to_bf16(ref + tol)) if bf16 else (ref - tol, ref + tol)
        assert ((got[h] >= lo) & (got[h] <= hi)).all(), (h, np.abs(got[h] - ref).max() / mag.min())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("rows", [4, 12, 28, 40])
def test_queries_near_the_ends_of_the_range(gl, rows, d, bf16):
    """Queries of 2^120 (scores of up to 2^125, one token takes all) next to those of 2^-120 (scores that are all the same)."""
    n = 200
    k, v = _bf16(1, (1, n, 1, d)), _bf16(2, (1, n, 1, d))
    size = np.resize([2.0 ** 120, 2.0 ** -120, 1.0], rows)
    q = (torch.from_numpy(synth.normal(3, 1, (rows, d)) * size[:, None])).to(torch.bfloat16).cuda().view(1, 1, rows, d)
    cache, table, lengths = _stored(gl, k, v, 16)
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths, flags=gl.GL_OUT_BF16 if bf16 else 0)
    got = got.tensor[0, 0].double().cpu().numpy()
    kd, vd = (mx4.rounded(x[0, :, 0].double().cpu().numpy()) for x in (k, v))
    qd = q[0, 0].double().cpu().numpy()
    for h in range(rows):
        s, p, ref, mag = _row(qd[h], kd, vd, d ** -0.5)
        ds = (d / 16 + 6) * 2.0 ** -23 * d ** -0.5 * (np.abs(kd) @ np.abs(qd[h])).max()
        if size[h] > 1:
            top = np.sort(s)[::-1]
            if top[0] - top[1] < 4 * ds:
                continue
            ref, mag, ds = vd[s.argmax()], np.abs(vd[s.argmax()]), 0.0
        rel = 2 * ds + 2.0 ** -20 + (n / 16 + 16) * 2.0 ** -23 + ((2.0 ** -8 if rows > 32 else 2.0 ** -10) if bf16 else 2.0 ** -20)
        tol = rel * mag
        lo, hi = (_to_bf16(ref - tol), _to_bf16(ref + tol)) if bf16 else (ref - tol, ref + tol)
        assert ((got[h] >= lo) & (got[h] <= hi)).all(), (h, size[h], np.abs(got[h] - ref).max())


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("t,heads", [(1, 8), (2, 8), (4, 8), (8, 8)])
def test_rounded_weights_are_summed_as_they_are_used(gl, t, heads, d):
    """One late token gets most of the weight, up to 2^7.9 times that of the first ones, so that its weight is no power of
    two when it is rounded.  With weights w (1 + r), |r| <= r0, in both sums the result is off by
    sum p r (V - out) / sum p (1 + r): nothing where the values agree.  r0: 2^-11 (fp16), 2^-8 (bf16, more than 32 rows)."""
    rows = t * heads
    n, loud = (230, 200) if rows > 32 else (64, 40)
    sign = np.sign(synth.normal(3, 1, (d,)))
    k = (synth.normal(4, 1, (n, d)) * 0.02).astype(np.float32)
    k[loud] = sign
    grid = np.array([1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    v = np.tile(grid[np.random.default_rng(d).integers(0, 6, d)], (n, 1))
    v[loud] = grid[np.random.default_rng(d + 1).integers(0, 6, d)]
    v[:, ::32] = 6.0                         # (scales of 1: the values are stored as they are)
    size = np.linspace(2.0, 7.9, rows) / (np.sqrt(d) * np.log2(np.e))
    q = torch.from_numpy(size[:, None] * sign).to(torch.bfloat16).cuda().view(1, t, heads, d)
    kt, vt = (torch.from_numpy(x).to(torch.bfloat16).cuda().view(1, n, 1, d) for x in (k, v))
    cache, table, lengths = _stored(gl, kt, vt, 16)
    # every row sees the loud token: the last `t` positions lie behind it
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths, flags=gl.GL_OUT_BF16).tensor[0].double().cpu().numpy()
    kd, vd, qd = mx4.rounded(kt[0, :, 0].double().cpu().numpy()), mx4.rounded(vt[0, :, 0].double().cpu().numpy()), q[0].double().cpu().numpy()
    r0 = 2.0 ** -8 if rows > 32 else 2.0 ** -11
    for i in range(t):
        for h in range(heads):
            keep = n - t + i + 1
            s, p, ref, mag = _row(qd[i, h], kd[:keep], vd[:keep], d ** -0.5)
            # scores: D products in fp32, two roundings, an error e in a score moves p by e; ex2 to 2 ulp; sums of n / 16 terms
            fp32 = 2 * (d / 16 + 6) * 2.0 ** -23 * np.abs(s).max() + 2.0 ** -20 + (n / 16 + 16) * 2.0 ** -23
            tol = r0 / (1 - r0) * (p[:, None] * np.abs(vd[:keep] - ref)).sum(0) + fp32 * mag
            assert ((got[i, h] >= _to_bf16(ref - tol)) & (got[i, h] <= _to_bf16(ref + tol))).all(), (i, h)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("page,d", [(48, 64), (48, 128), (80, 256), (112, 128)])
@pytest.mark.parametrize("rows", [4, 40])
def test_pages_of_other_sizes(gl, rows, page, d, bf16):
    """Pages of a multiple of 16 tokens that is no power of two: they end inside a tile, at another place in every one."""
    n = 613
    k, v, q = _bf16(1, (2, n, 2, d)), _bf16(2, (2, n, 2, d)), _bf16(3, (2, 1, 2 * rows, d), 1.5)
    cache, table, lengths = _stored(gl, k, v, page)
    rk, rv = gl.gl_cache4_read(cache, n, table, lengths)
    kd, vd = (mx4.rounded(x.double().cpu().numpy()) for x in (k, v))
    assert np.array_equal(rk.double().cpu().numpy(), kd) and np.array_equal(rv.double().cpu().numpy(), vd)
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths, flags=gl.GL_OUT_BF16 if bf16 else 0).tensor
    got, qd = got.double().cpu().numpy(), q.double().cpu().numpy()
    for b in range(2):
        for h in range(2 * rows):
            s, p, ref, mag = _row(qd[b, 0, h], kd[b, :, h // rows], vd[b, :, h // rows], d ** -0.5)
            ds = (d / 16 + 6) * 2.0 ** -23 * d ** -0.5 * (np.abs(kd[b, :, h // rows]) @ np.abs(qd[b, 0, h])).max()
            rel = 2 * ds + 2.0 ** -20 + (n / 16 + 16) * 2.0 ** -23 + ((2.0 ** -8 if rows > 32 else 2.0 ** -10) if bf16 else 2.0 ** -20)
            tol = rel * mag
            lo, hi = (_to_bf16(ref - tol), _to_bf16(ref + tol)) if bf16 else (ref - tol, ref + tol)
            assert ((got[b, 0, h] >= lo) & (got[b, 0, h] <= hi)).all(), (b, h)
