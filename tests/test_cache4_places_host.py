"""Where the threads of an append or a read look for their tokens, run on the host: right, and never past an array."""
import os
import subprocess

import pytest

from paper_2105_09377_b200 import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("places") / "cache4_places")
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-std=c++17", "-gencode",
                           "arch=compute_100a,code=sm_100a", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                           os.path.join(HERE, "cache4_places.cu"), "-o", exe])
    return exe


# batch, T, kv heads, D, page, pages per sequence, items per block (256 threads of one or two items)
@pytest.mark.parametrize("args", [
    (1, 1, 1, 64, 16, 1, 256), (1, 1, 1, 128, 16, 1, 512), (3, 5, 2, 64, 16, 3, 256), (64, 1, 8, 128, 64, 3, 512),
    (1024, 1, 1, 64, 16, 1, 256), (7, 33, 3, 256, 48, 2, 512), (2, 129, 1, 64, 112, 2, 256)])
def test_places(program, args):
    r = subprocess.run([program] + [str(a) for a in args], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.startswith("ok"), (r.returncode, r.stdout)
