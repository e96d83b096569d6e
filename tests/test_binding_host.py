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
