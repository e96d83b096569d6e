"""Where the rules of the 8-bit operators, the norm and the rotation change from one kernel to the next; places that are shared."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import binding
    return binding


def _rows(rows, k, dtype, seed=1):
    g = torch.Generator("cuda").manual_seed(seed + rows + k)
    return (torch.randn((rows, k), generator=g, device="cuda") * torch.rand((rows, 1), generator=g, device="cuda").add_(0.25)).to(dtype)


def _norm_is_right(gl, rows, k, dtype, res=None, eps=1e-5):
    """The fp32 result against 64 bits, the bf16 and F8 results as its roundings."""
    ap = gl.AccessPattern
    x, r, w = _rows(rows, k, dtype), None if res is None else _rows(rows, k, res, 2), torch.randn(k, device="cuda")
    opt = None if r is None else ap(r, 1)
    plain = gl.gl_compute_norm_rms(ap(x, 1), ap(w, 0), eps, opt, None, ap(torch.empty((rows, k), device="cuda"), 1))
    # 32 products in a lane, 5 steps over lanes, 32 warps, halved by the root; the mean, eps, the root and three products 12, h 1
    for at in range(0, rows, 1 << 18):
        part = slice(at, at + (1 << 18))
        h = x[part].double() + (0 if r is None else r[part].double())
        y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + eps) * w.double()
        assert ((plain.tensor[part].double() - y).abs() <= (69 / 2 + 13) * U * y.abs()).all()
    half = gl.gl_compute_norm_rms(ap(x, 1), ap(w, 0), eps, opt, None, ap(torch.empty((rows, k), dtype=BF, device="cuda"), 1)).tensor
    assert torch.equal(half, plain.tensor.to(BF))
    q, want = gl.gl_compute_norm_rms_f8(ap(x, 1), ap(w, 0), eps, opt), gl.gl_f8_quantize(plain)
    assert torch.equal(gl.gl_f8_dequantize(q).tensor, gl.gl_f8_dequantize(want).tensor)


@pytest.mark.parametrize("rows,k", [(600, 16384), (600, 16640), (1000, 12288), (700, 14336), (840, 10240), (600, 16376), (530, 16384), (100, 16384)])
def test_norm_of_rows_of_forty_to_sixty_five_units(gl, rows, k):
    """bf16 without a residual into F8: eight units a warp in five to eight warps, and what lies beyond."""
    _norm_is_right(gl, rows, k, BF)


@pytest.mark.parametrize("rows,k", [(1250003, 8), (620001, 16), (1212416, 8), (1212415, 8)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_four_groups_of_one_or_two_lanes(gl, rows, k, dtype):
    _norm_is_right(gl, rows, k, dtype)
    _norm_is_right(gl, rows, k, BF, dtype)
    ap, x = gl.AccessPattern, _rows(rows, k, dtype)
    back = gl.gl_f8_dequantize(gl.gl_f8_quantize(ap(x, 1)), ap(torch.empty_like(x), 1)).tensor
    # a row is one block: codes of the values over the smallest power of two that brings the largest to 448 or below
    top = torch.frexp(x.double().abs().amax(-1, keepdim=True))
    scale = torch.exp2((top.exponent - 9 + (top.mantissa > 0.875).int()).double())
    want = ((x.double() / scale).float().to(torch.float8_e4m3fn).double() * scale).to(dtype)
    assert torch.equal(back, want)


def test_a_prepared_call_shared_by_threads(gl):
    """Each thread's work follows what its own stream holds: inputs that its stream makes, results that it reads."""
    ap, calls, failed = gl.AccessPattern, [], []
    for i in range(4):                                   # (an operand and a result of its own for each, one plan, one weight)
        x = torch.empty((64, 1024), dtype=BF, device="cuda")
        calls.append((x, ap(torch.empty_like(x), 1)))
    w = ap(torch.randn(1024, device="cuda"), 0)
    prepared = [gl.prepare_compute_norm_rms(ap(x, 1), w, out) for x, out in calls]
    start, streams = threading.Barrier(4), [torch.cuda.Stream() for _ in range(4)]

    def run(i):
        try:
            start.wait()
            with torch.cuda.stream(streams[i]):
                for turn in range(200):
                    x, out = calls[i]
                    x.fill_(float(turn % 7 + 1))
                    prepared[(i + 1) % 4](streams[(i + 1) % 4])          # another thread's call, on that thread's stream
                    prepared[i]()
                    if turn % 50 == 49:
                        want = gl.gl_compute_norm_rms(ap(x, 1), w).tensor
                        streams[i].synchronize()
                        assert torch.equal(out.tensor, want), (i, turn)
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert not failed, failed[0]


def _turned(gl, x, plan, pos):
    return gl.gl_compute_rotate(gl.AccessPattern(x.contiguous(), 3), plan, pos).tensor


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_rotation_into_the_gaps_of_its_operand(gl, dtype):
    """Queries turned into where the keys of the same projection lie; every second token into the places between."""
    ap, plan = gl.AccessPattern, gl.rotary_plan(32)
    qkv, pos = torch.randn(2, 19, 12, 64, device="cuda").to(dtype), torch.arange(38, dtype=torch.int32, device="cuda").view(2, 19)
    want, before = _turned(gl, qkv[:, :, :4], plan, pos), qkv.clone()
    gl.gl_compute_rotate(ap(qkv[:, :, :4], 3), plan, pos, ap(qkv[:, :, 4:8], 3))
    assert torch.equal(qkv[:, :, 4:8], want) and torch.equal(qkv[:, :, :4], before[:, :, :4]) and torch.equal(qkv[:, :, 8:], before[:, :, 8:])
    gl.gl_compute_rotate(ap(qkv[:, :, 8:], 3), plan, pos, ap(qkv[:, :, :4], 3))
    assert torch.equal(qkv[:, :, :4], _turned(gl, before[:, :, 8:], plan, pos)) and torch.equal(qkv[:, :, 8:], before[:, :, 8:])
    tokens = torch.randn(1, 40, 2, 64, device="cuda").to(dtype)
    kept = tokens.clone()
    gl.gl_compute_rotate(ap(tokens[:, 0::2], 3), plan, pos[:1, :1].expand(1, 20).contiguous(), ap(tokens[:, 1::2], 3))
    assert torch.equal(tokens[:, 0::2], kept[:, 0::2])
    assert torch.equal(tokens[:, 1::2], _turned(gl, kept[:, 0::2], plan, pos[:1, :1].expand(1, 20).contiguous()))
    # another distance: the first tokens of what is twice as far apart
    wide = torch.randn(1, 24, 4, 64, device="cuda").to(dtype)
    kept = wide.clone()
    gl.gl_compute_rotate(ap(wide[:, :12, :2], 3), plan, pos[:1, :12].contiguous(), ap(wide[:, 0::2, 2:], 3))
    assert torch.equal(wide[:, 0::2, 2:], _turned(gl, kept[:, :12, :2], plan, pos[:1, :12].contiguous())) and torch.equal(wide[:, :, :2], kept[:, :, :2])


def test_neighbours_of_one_projection_are_refused(gl):
    ap, plan = gl.AccessPattern, gl.rotary_plan(32)
    qkv, pos = torch.randn(2, 19, 12, 64, device="cuda").to(BF), torch.arange(38, dtype=torch.int32, device="cuda").view(2, 19)
    before = qkv.clone()
    for out in (qkv[:, :, 1:9], qkv[:, :, 4:]):
        with pytest.raises(gl.GlError):
            gl.gl_compute_rotate(ap(qkv[:, :, :8], 3), plan, pos, ap(out, 3))
    x = torch.randn(9, 512, device="cuda")
    with pytest.raises(gl.GlError):
        gl.gl_compute_norm_rms(ap(x[:8], 1), out=ap(x[1:], 1))
    with pytest.raises(gl.GlError):
        gl.gl_compute_norm_rms(ap(x, 1), out=ap(x.view(-1).view(BF)[: 9 * 512].view(9, 512), 1))
    torch.cuda.synchronize()
    assert torch.equal(qkv, before)
