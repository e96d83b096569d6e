"""GPU parity of the pages of 4-bit keys and values and of the attention over them, against 64 bits."""
import numpy as np
import pytest
import torch

from oracle import mx4
from paper_2105_09377_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import binding
    return binding


def _to_bf16(x):
    """Rounded to eight significant bits, ties to even (float64 in and out)."""
    m, e = np.frexp(x)
    return np.ldexp(np.round(m * 256.0), e - 8)


def _within(got, ref, tol, bf16):
    """|result before the last rounding - ref| <= tol, as far as the rounded result can show it: rounding is monotonic."""
    lo, hi = ref - tol, ref + tol
    return (got >= (_to_bf16(lo) if bf16 else lo)) & (got <= (_to_bf16(hi) if bf16 else hi))


def _bf16(seed, shape, std=1.0):
    return torch.from_numpy((synth.normal(seed, 1, shape) * std).astype(np.float32)).cuda().to(torch.bfloat16)


def _filled(gl, lens, hkv, d, page, seed=1, spare=3, k=None, v=None):
    """A cache of 0xFF bytes (NaN scales wherever nothing was stored) with shuffled pages, filled by one append."""
    b, n = len(lens), max(1, max(lens))
    width = -(-n // page)
    order = np.random.default_rng(seed).permutation(b * width + spare)[: b * width].astype(np.int32)
    table = torch.from_numpy(order.reshape(b, width)).cuda()
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    cache = gl.cache4_empty(b * width + spare, hkv, page, d, "cuda")
    cache.data.fill_(0xFF)
    k = _bf16(seed + 10, (b, n, hkv, d)) if k is None else k
    v = _bf16(seed + 20, (b, n, hkv, d)) if v is None else v
    gl.gl_cache4_append(cache, k, v, table, lengths)
    return cache, table, lengths, k, v


@pytest.mark.parametrize("lens,t,hkv,d,page", [
    ([1], 1, 1, 64, 16), ([5, 0, 40], 40, 2, 64, 16), ([33, 64, 17], 64, 3, 128, 32), ([100, 7], 100, 1, 256, 64),
    ([130, 128, 129, 1], 130, 4, 128, 128), ([15, 16, 17, 31, 32, 33], 33, 2, 128, 16)])
def test_append_and_read(gl, lens, t, hkv, d, page):
    cache, table, lengths, k, v = _filled(gl, lens, hkv, d, page)
    rk, rv = gl.gl_cache4_read(cache, t, table, lengths)
    for x, y in ((k, rk), (v, rv)):
        want = mx4.rounded(x.double().cpu().numpy())
        for b, n in enumerate(lens):
            want[b, : t - n] = 0.0
        np.testing.assert_array_equal(y.double().cpu().numpy(), want)
    # token by token, at the same places, gives the same bytes
    again = gl.cache4_empty(cache.pages, hkv, page, d, "cuda")
    again.data.fill_(0xFF)
    wide = k.shape[1]
    for i in range(wide):
        now = (lengths - wide + i + 1).clamp_min(0)
        gl.gl_cache4_append(again, k[:, i:i + 1].contiguous(), v[:, i:i + 1].contiguous(), table, now)
    assert torch.equal(cache.data, again.data)


def _check(gl, cache, table, lengths, k, v, q, lens, scale, bf16, flags=0, out=None, got=None):
    hkv, d = cache.kv_heads, cache.head_dim
    b, t, hq, _ = q.shape
    kd, vd = mx4.rounded(k.double().cpu().numpy()), mx4.rounded(v.double().cpu().numpy())
    qd = q.double().cpu().numpy()
    wide = k.shape[1]
    for i, n in enumerate(lens):
        kk, vv = kd[i, wide - n:], vd[i, wide - n:]
        ref, mag = mx4.attend(qd[i], kk, vv, hq // hkv, scale, n - t)
        # scores: D products of fp32 partial sums, then two roundings; their error enters p twice over (value and sum).
        # p: ex2 to 2 ulp and, for bf16 results, one rounding to 11 bits (8 bits where more than 32 rows share a kv head);
        # result: fp32 sums of n / 16 terms.
        worst = scale * (np.abs(qd[i]).max() * np.abs(kk).max() * d if n else 0.0)
        ds = (d / 16 + 6) * 2.0 ** -23 * worst
        rel = 2 * ds + 2.0 ** -20 + (n / 16 + 16) * 2.0 ** -23 + ((2.0 ** -8 if t * (hq // hkv) > 32 else 2.0 ** -10) if bf16 else 2.0 ** -20)
        tol = rel * mag + 1e-37
        g = got[i].double().cpu().numpy()
        assert np.isfinite(g).all()
        assert _within(g, ref, tol, bf16).all(), (i, n, float(np.max(np.abs(g - ref) / np.maximum(tol, 1e-300))))


ATTEND = [
    # lens, T, heads, kv heads, D, page
    ([1], 1, 1, 1, 64, 16),
    ([33], 1, 8, 8, 64, 16),
    ([0, 1, 31, 32, 33, 64], 1, 4, 2, 128, 32),
    ([700, 3, 129], 1, 5, 1, 128, 64),
    ([1000], 1, 16, 2, 128, 128),
    ([300, 17], 1, 16, 1, 256, 16),
    ([90, 200], 1, 32, 1, 64, 64),
    ([5, 2, 40], 4, 4, 2, 128, 16),          # rows that see nothing: fewer tokens than rows
    ([64, 100], 33, 6, 2, 64, 32),
    ([150, 9], 21, 8, 4, 256, 16),
    ([257, 130], 130, 4, 4, 128, 64),
    ([2500, 1200, 30], 3, 8, 4, 128, 16),    # cut over many blocks
    ([200], 40, 1, 1, 128, 16),              # more than 32 rows: tcgen05
    ([128, 129, 127, 1, 0], 128, 2, 1, 128, 64),
    ([300, 700, 20], 150, 4, 2, 64, 32),
    ([260, 64, 65], 33, 2, 2, 256, 128),
    ([3000], 70, 8, 1, 128, 16),             # 560 rows of one kv head over many blocks
    ([900, 1100], 300, 3, 3, 128, 64),
    ([0, 256, 3, 129], 1, 6, 2, 64, 256),    # at most 256 tokens: a block per sequence and head
    ([128, 0, 77], 2, 3, 3, 256, 128),       # (128 of them for 256-wide heads)
    ([512, 1, 0, 400], 35, 4, 2, 128, 512),  # (512 for more than 32 rows)
    ([0, 257], 1, 6, 2, 64, 16),
]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("lens,t,hq,hkv,d,page", ATTEND)
def test_attend(gl, lens, t, hq, hkv, d, page, bf16):
    cache, table, lengths, k, v = _filled(gl, lens, hkv, d, page, seed=hq + d)
    q = _bf16(77, (len(lens), t, hq, d), 1.5)
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths, flags=gl.GL_OUT_BF16 if bf16 else 0)
    _check(gl, cache, table, lengths, k, v, q, lens, d ** -0.5, bf16, got=got.tensor)
    again = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths, flags=gl.GL_OUT_BF16 if bf16 else 0)
    assert torch.equal(got.tensor, again.tensor)
    assert gl.gl_poll_device_status() == 0


@pytest.mark.parametrize("d", [64, 128, 256])
def test_values_of_many_binades(gl, d):
    """Scales of V that span far more than fp16 within a tile, and a loud token that has next to no weight."""
    lens = [96, 50]
    k, v = _bf16(5, (2, 96, 2, d)), _bf16(6, (2, 96, 2, d))
    v = v * torch.from_numpy(np.exp2(np.round(synth.uniform(9, 1, (2, 96, 2, d), -60, 60)[..., :1]))).cuda().to(torch.bfloat16)
    v[:, 60:70] = 0
    cache, table, lengths, k, v = _filled(gl, lens, 2, d, 32, k=k, v=v)
    for bf16, t in ((False, 2), (True, 2), (False, 20), (True, 20)):
        q = _bf16(7, (2, t, 4, d), 3.0)
        got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths, flags=gl.GL_OUT_BF16 if bf16 else 0)
        _check(gl, cache, table, lengths, k, v, q, lens, d ** -0.5, bf16, got=got.tensor)


@pytest.mark.parametrize("t", [1, 9])
def test_queries_of_many_sizes(gl, t):
    cache, table, lengths, k, v = _filled(gl, [70], 1, 128, 16, k=_bf16(5, (1, 70, 1, 128), 1e-3))
    q = _bf16(8, (1, t, 4, 128)) * torch.tensor([0.0, 1e-30, 1e6, 300.0], device="cuda").view(1, 1, 4, 1).to(torch.bfloat16)
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths, scale=1e-3)
    _check(gl, cache, table, lengths, k, v, q, [70], 1e-3, False, got=got.tensor)


@pytest.mark.parametrize("t", [5, 40])
def test_parts_of_a_fused_projection(gl, t):
    """q, k and v as slices of one [B, T, (heads + 2 kv heads) D] result."""
    lens, hq, hkv, d = [t, t - 3], 6, 2, 64
    fused = _bf16(3, (2, t, hq + 2 * hkv, d))
    q, k, v = fused[:, :, :hq], fused[:, :, hq:hq + hkv], fused[:, :, hq + hkv:]
    cache, table, lengths, _, _ = _filled(gl, lens, hkv, d, 16, k=k, v=v)
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths)
    dense = gl.gl_attend_cache4(gl.AccessPattern(q.contiguous(), 3), cache, table, lengths)
    assert torch.equal(got.tensor, dense.tensor)
    _check(gl, cache, table, lengths, k, v, q, lens, d ** -0.5, False, got=got.tensor)


@pytest.mark.parametrize("heads", [4, 80])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_pages_that_do_not_exist_are_not_seen(gl, d, heads):
    lens = [64, 80]
    cache, table, lengths, k, v = _filled(gl, lens, 2, d, 16)
    bad = table.clone()
    bad[0, 1], bad[0, 2], bad[1, 4] = -1, cache.pages, 2 ** 31 - 1
    q = _bf16(4, (2, 1, heads, d))
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, bad, lengths).tensor
    kd, vd = mx4.rounded(k.double().cpu().numpy()), mx4.rounded(v.double().cpu().numpy())
    for i, keep in enumerate((list(range(16)) + list(range(48, 64)), list(range(64)))):
        off = k.shape[1] - lens[i]
        ref, mag = mx4.attend(q[i].double().cpu().numpy(), kd[i, off:][keep], vd[i, off:][keep], heads // 2, d ** -0.5, len(keep) - 1)
        assert (np.abs(got[i].double().cpu().numpy() - ref) <= 2.0 ** -14 * mag).all()
    before = cache.data.clone()
    gl.gl_cache4_append(cache, k[:, -1:].contiguous(), v[:, -1:].contiguous(), torch.full_like(table, cache.pages), lengths)
    assert torch.equal(before, cache.data)
    rk, _ = gl.gl_cache4_read(cache, 20, bad, lengths)
    assert not rk[1, 4:].any() and rk[1, :4].any()
    # lengths out of range count as empty, or as all that the table can hold
    wild = torch.tensor([-5, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, wild).tensor
    assert not got[0].any() and torch.isfinite(got[1]).all()


@pytest.mark.parametrize("heads", [2, 24])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_nan_reaches_the_rows_that_see_it_and_no_others(gl, d, heads):
    lens, t = [40], 3
    k, v = _bf16(5, (1, 40, 1, d)), _bf16(6, (1, 40, 1, d))
    v[0, 38, 0, 40] = float("nan")                        # token 38: seen by rows 1 and 2, second block of dims
    cache, table, lengths, k, v = _filled(gl, lens, 1, d, 16, k=k, v=v)
    q = _bf16(7, (1, t, heads, d))
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths).tensor[0]
    nan = torch.isnan(got)
    assert not nan[0].any() and nan[1:, :, 32:64].all()
    nan[1:, :, 32:64] = False
    assert not nan.any()
    k[0, 39, 0, 0] = float("inf")                         # token 39: a key that is NaN makes row 2 NaN
    cache, table, lengths, k, v = _filled(gl, lens, 1, d, 16, k=k, v=v.nan_to_num())
    nan = torch.isnan(gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths).tensor[0])
    assert not nan[:2].any() and nan[2].all()


def test_a_cache_beyond_4_gib(gl):
    d, hkv, page = 128, 8, 128
    per_page = hkv * (page // 16) * 17 * d
    pages = (5 << 30) // per_page
    cache = gl.cache4_empty(pages, hkv, page, d, "cuda")
    lens = [300, 140]
    table = torch.tensor([[pages - 1, 3, pages - 2], [pages - 3, pages - 4, 0]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    k, v = _bf16(1, (2, 300, hkv, d)), _bf16(2, (2, 300, hkv, d))
    gl.gl_cache4_append(cache, k, v, table, lengths)
    q = _bf16(3, (2, 1, 8, d))
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths)
    _check(gl, cache, table, lengths, k, v, q, lens, d ** -0.5, False, got=got.tensor)


def test_long_sequences_on_another_stream(gl):
    lens, d = [20000, 5], 128
    cache, table, lengths, k, v = _filled(gl, lens, 1, d, 64)
    q = _bf16(3, (2, 1, 3, d), 2.0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths, flags=gl.GL_OUT_BF16)
    side.synchronize()
    _check(gl, cache, table, lengths, k, v, q, lens, d ** -0.5, True, got=got.tensor)


@pytest.mark.parametrize("heads,batch", [(1, 300), (40, 1200)])
def test_more_sequences_than_threads(gl, heads, batch):
    """The blocks find their place in rounds; every length from none to a few tiles."""
    lens = [(7 * i) % 90 for i in range(batch)]
    cache, table, lengths, k, v = _filled(gl, lens, 1, 64, 16)
    q = _bf16(4, (batch, 1, heads, 64))
    got = gl.gl_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths).tensor
    some = list(range(0, 20)) + list(range(120, 140)) + list(range(batch - 20, batch))
    at = torch.tensor(some)
    _check(gl, cache, table, lengths, k[at], v[at], q[at], [lens[i] for i in some], 0.125, False, got=got[at])
    assert not got[[i for i, n in enumerate(lens) if n == 0]].any()


def test_prepared_calls_in_a_graph(gl):
    lens, d = [50, 20], 64
    cache, table, lengths, k, v = _filled(gl, lens, 1, d, 64)
    q, k1, v1 = (_bf16(s, (2, 1, h, d)) for s, h in ((4, 2), (5, 1), (6, 1)))
    out = gl.AccessPattern(torch.zeros(2, 1, 2, d, device="cuda"), 3)
    calls = [gl.prepare_cache4_append(cache, k1, v1, table, lengths),
             gl.prepare_attend_cache4(gl.AccessPattern(q, 3), cache, table, lengths, out)]
    lengths += 1                       # both are read on the device: the graph goes on with the lengths it finds
    for call in calls:
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in calls:
            call()
    lengths += 1
    k1.copy_(_bf16(7, (2, 1, 1, d)))
    graph.replay()
    first = torch.cat([k, _bf16(5, (2, 1, 1, d)), k1], 1), torch.cat([v, v1, v1], 1)
    # (left-padded: the padding moves along)
    _check(gl, cache, table, lengths, first[0], first[1], q, [52, 22], d ** -0.5, False, got=out.tensor)
