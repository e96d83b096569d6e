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
