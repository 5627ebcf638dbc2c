"""The AdamW kernels' own square root and reciprocal equal CUDA's correctly rounded ones: the codes of 8-bit states are those of the
formula in fp32, and the same from both forms of a block's step, because of it."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from gpu_util import require_cuda
from paper_1908_06077_b200 import build as cuda_build

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    require_cuda()
    path = str(tmp_path_factory.mktemp("roots") / "libroots.so")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc] + cuda_build.NVCC_FLAGS + ["-shared", "-o", path, os.path.join(HERE, "roots.cu")], check=True)
    lib = C.CDLL(path)
    lib.compare_range.argtypes = [C.c_uint32, C.c_uint32, C.c_void_p, C.c_void_p]
    return lib


def _bits(x):
    return int(np.float32(x).view(np.uint32))


def _differ(lib, low, high):
    torch, _ = require_cuda()
    counts, last = torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    assert lib.compare_range(low, high, counts.data_ptr(), last.data_ptr()) == 0
    return [(c, hex(x & 0xFFFFFFFF)) if c else (0, None) for c, x in zip(counts.tolist(), last.tolist())]


def test_every_root_from_2_to_the_minus_100_on(lib):
    """up to the largest number"""
    assert _differ(lib, _bits(2.0 ** -100), _bits(np.finfo(np.float32).max))[0] == (0, None)


def test_every_reciprocal_from_2_to_the_minus_100_to_2_to_the_126(lib):
    assert _differ(lib, _bits(2.0 ** -100), _bits(2.0 ** 126))[1] == (0, None)


def test_what_differs_is_found(lib):
    """zero and infinity are not the functions' to answer: NaN, where CUDA's root is a number"""
    assert _differ(lib, 0, 0)[0] == (1, "0x0")
    assert _differ(lib, _bits(np.inf), _bits(np.inf))[0][0] == 1
