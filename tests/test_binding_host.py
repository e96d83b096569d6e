"""Host-only checks of what the Python binding hands to the library: views it cannot describe, where tensors live."""
import pytest
import torch


@pytest.fixture(scope="module")
def gl():
    from paper_2105_09377_b200 import build
    build.build()
    from paper_2105_09377_b200 import binding
    return binding


@pytest.mark.parametrize("shape,view", [
    ((1, 1, 4, 64), (8, 1, 4, 64)),      # one token for every sequence
    ((1, 1, 4, 64), (1, 8, 4, 64)),      # for every token
    ((1, 1, 4, 64), (3, 5, 4, 64)),
    ((3, 1, 4, 64), (3, 5, 4, 64)),
    ((1, 5, 4, 64), (3, 5, 4, 64))])
def test_broadcast_tokens_are_refused(gl, shape, view):
    """A distance of 0 between tokens would be read as `dense`, far behind the storage."""
    t = torch.zeros(shape, dtype=torch.bfloat16).expand(view)
    with pytest.raises(ValueError):
        gl._tokens_struct(t)


def test_overlapping_tokens_are_refused(gl):
    t = torch.zeros(4096, dtype=torch.bfloat16).as_strided((1, 8, 4, 64), (1024, 128, 64, 1))
    with pytest.raises(ValueError):
        gl._tokens_struct(t)


def test_distances_that_can_be_described(gl):
    one = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16)
    assert gl._tokens_struct(one)[1] == 256
    assert gl._tokens_struct(one.expand(1, 1, 4, 64))[1] == 256
    fused = torch.zeros(6, 1, 12, 64, dtype=torch.bfloat16)
    assert gl._tokens_struct(fused[:, :, 4:8])[1] == 12 * 64
    assert gl._tokens_struct(fused.transpose(0, 1)[:, :, 8:])[1] == 12 * 64


def _calls(gl):
    """Every call on 4-bit operands as a function of where its tensors live, one tensor at a time on the host."""
    bf, f32, u8, i32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32

    def made(shape, dtype):
        return torch.zeros(shape, dtype=dtype)

    def mx(rows, k):
        s = gl._mx4_meta((rows, k), 1)
        import ctypes
        return gl.Mx4(made(gl.LIB.gl_mx4_data_bytes(ctypes.byref(s)), u8), made(gl.LIB.gl_mx4_scale_bytes(ctypes.byref(s)), u8),
                      (rows, k), 1)

    ap = gl.AccessPattern
    x, out = ap(made((4, 64), bf), 1), ap(made((4, 6), f32), 2)
    cache = gl.cache4_empty(2, 1, 16, 64, "cpu")
    k, q = made((1, 3, 1, 64), bf), ap(made((1, 3, 2, 64), bf), 3)
    table, lengths = made((1, 2), i32), made((1,), i32)
    ws = made(1 << 20, u8)
    return {
        "quantize": lambda: gl.gl_mx4_quantize(x, mx(4, 64)), "dequantize": lambda: gl.gl_mx4_dequantize(mx(4, 64), x),
        "product": lambda: gl.gl_cartesian_dot_mx4(mx(4, 64), mx(6, 64), out), "dense": lambda: gl.gl_dense_mx4(x, mx(6, 64), out),
        "append": lambda: gl.gl_cache4_append(cache, k, k, table, lengths), "read": lambda: gl.gl_cache4_read(cache, 3, table, lengths),
        "attend": lambda: gl.gl_attend_cache4(q, cache, table, lengths),
        "prepare_quantize": lambda: gl.prepare_mx4_quantize(x, mx(4, 64)),
        "prepare_dequantize": lambda: gl.prepare_mx4_dequantize(mx(4, 64), x),
        "prepare_product": lambda: gl.prepare_cartesian_dot_mx4(mx(4, 64), mx(6, 64), out),
        "prepare_dense": lambda: gl.prepare_dense_mx4(x, mx(6, 64), out, workspace=ws),
        "prepare_append": lambda: gl.prepare_cache4_append(cache, k, k, table, lengths),
        "prepare_read": lambda: gl.prepare_cache4_read(cache, k, k, table, lengths),
        "prepare_attend": lambda: gl.prepare_attend_cache4(q, cache, table, lengths, ap(made((1, 3, 2, 64), f32), 3), workspace=ws),
    }


@pytest.mark.parametrize("name", ["quantize", "dequantize", "product", "dense", "append", "read", "attend", "prepare_quantize",
                                  "prepare_dequantize", "prepare_product", "prepare_dense", "prepare_append", "prepare_read",
                                  "prepare_attend"])
def test_host_tensors_are_refused(gl, name):
    """A host address would be read by a kernel."""
    with pytest.raises(ValueError, match="GPU"):
        _calls(gl)[name]()


def test_tensors_are_on_one_gpu(gl):
    class T:                                       # (what the check looks at; this machine has no GPU)
        def __init__(self, device):
            self.device, self.is_cuda = torch.device(device), device != "cpu"
    gl._on_gpu(T("cuda:0"), T("cuda:0"))
    gl._on_gpu(T("cuda:1"), None, T("cuda:1"))     # no workspace given
    for devices in (("cuda:0", "cpu"), ("cpu", "cuda:0"), ("cuda:0", "cuda:1")):
        with pytest.raises(ValueError):
            gl._on_gpu(*(T(d) for d in devices))


class _Stream:
    cuda_stream = 7


def _storing_calls(gl):
    """Calls that take storage for their result or their scratch, as functions of the stream."""
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    ap = gl.AccessPattern
    a, win = ap(torch.zeros(2, 6, 6, 6), 1), gl.windows_spec((6, 3, 3), (1, 1, 1))
    b = ap(torch.zeros(2, 6, 6, 6), 1)
    x, w = ap(torch.zeros(2, 64, 9, 9, dtype=bf), 1), ap(torch.zeros(5, 64, 3, 3, dtype=bf), 1)
    conv = gl.windows_spec((64, 3, 3), (1, 1, 1))
    assert gl.gl_cartesian_dot_workspace(x, conv, w) > 0
    rows = ap(torch.zeros(4, 64, dtype=bf), 1)
    m0, m1 = gl.mx4_empty((4, 64), 1, "cpu"), gl.mx4_empty((6, 64), 1, "cpu")
    cache = gl.cache4_empty(2, 1, 16, 64, "cpu")
    q = ap(torch.zeros(1, 3, 2, 64, dtype=bf), 3)
    table, lengths = torch.zeros(1, 2, dtype=i32), torch.zeros(1, dtype=i32)
    return [lambda s: gl.gl_access_windows(a, win, stream=s), lambda s: gl.gl_access_transpose(a, (1, 0, 2, 3), stream=s),
            lambda s: gl.gl_access_pad(a, 1, 1, 1, stream=s), lambda s: gl.gl_access_slice(a, 1, 0, 2, stream=s),
            lambda s: gl.gl_access_concat(a, b, 1, stream=s), lambda s: gl.gl_access_pair(a, b, stream=s),
            lambda s: gl.gl_compute_reduce_max(a, None, stream=s), lambda s: gl.gl_compute_reduce_sum(a, stream=s),
            lambda s: gl.gl_compute_relu(a, stream=s), lambda s: gl.gl_cartesian_dot(x, conv, w, stream=s),
            lambda s: gl.gl_mx4_quantize(rows, stream=s), lambda s: gl.gl_mx4_dequantize(m0, stream=s),
            lambda s: gl.gl_cartesian_dot_mx4(m0, m1, stream=s), lambda s: gl.gl_dense_mx4(rows, m1, stream=s),
            lambda s: gl.gl_cache4_read(cache, 3, table, lengths, stream=s),
            lambda s: gl.gl_attend_cache4(q, cache, table, lengths, stream=s)]


def test_storage_is_taken_on_the_stream_of_the_call(gl, monkeypatch):
    """torch hands a block out again in the order of the stream that it was taken on: scratch that is dropped on return may
    only have been taken on the stream that still uses it."""
    import contextlib
    calls = _storing_calls(gl)
    now, taken, launched = [], [], []

    @contextlib.contextmanager
    def stream(s):
        now.append(s.cuda_stream)
        yield
        now.pop()

    class Lib:                              # host functions as they are, device calls recorded
        def __getattr__(self, name):
            f = getattr(real, name)
            if name.endswith(("_workspace", "_bytes")) or name.startswith("gl_shape"):
                return f
            return lambda *args: launched.append(args[-1]) or 0

    real, empty = gl.LIB, torch.empty
    monkeypatch.setattr(gl, "LIB", Lib())
    monkeypatch.setattr(gl, "_on_gpu", lambda *t: None)
    monkeypatch.setattr(gl, "_stream", lambda s: 3 if s is None else s if isinstance(s, int) else s.cuda_stream)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda raw: _Stream() if raw == 7 else None)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: taken.append(now[-1] if now else 3) or empty(*a, **k))
    monkeypatch.setattr(torch, "empty_like", lambda t: taken.append(now[-1] if now else 3) or empty(t.shape, dtype=t.dtype))
    for given, raw in ((None, 3), (_Stream(), 7), (7, 7)):
        for i, call in enumerate(calls):
            del taken[:], launched[:]
            call(given)
            assert launched == [raw] and taken and set(taken) == {raw}, (i, given, taken)


def test_prepared_scratch_tells_torch_of_other_streams(gl, monkeypatch):
    told = []

    class Scratch:
        def record_stream(self, s):
            told.append(s.cuda_stream)

    monkeypatch.setattr(gl, "_stream", lambda s: 3 if s is None else s.cuda_stream)
    call = gl.Prepared(lambda raw: 0, (), (), Scratch())
    for s in (None, _Stream(), None, _Stream()):
        call(s)
    assert told == [7]


def test_attention_checks_the_split_and_the_scale(gl, monkeypatch):
    monkeypatch.setattr(gl, "_on_gpu", lambda *t: None)
    cache = gl.cache4_empty(2, 1, 16, 64, "cpu")
    table, lengths = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    out = gl.AccessPattern(torch.zeros(1, 3, 2, 64), 3)

    def call(access, scale):
        q = gl.AccessPattern(torch.zeros(1, 3, 2, 64, dtype=torch.bfloat16), access)
        ws = torch.zeros(gl.gl_attend_cache4_workspace(q, cache) + 1024, dtype=torch.uint8)
        return gl.LIB.gl_attend_cache4(*gl._attend_args(q, cache, table, lengths, out, scale, 0, ws), None)

    assert call(2, 0.125) == 3 and call(4, 0.125) == 3              # ((B, T, heads),(head_dim)) and nothing else
    for scale in (1.8e38, 2.5e38, 3.3e38):                          # times log2(e) these may leave fp32's range
        assert call(3, scale) == 4
