"""What nuq_grad_norm and nuq_adamw refuse and launch, without a GPU: the library's objects linked with a runtime that runs
nothing (fake_cudart.cpp)."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

import adamw_reference as R
from paper_1908_06077_b200 import build as cuda_build

HERE = os.path.dirname(os.path.abspath(__file__))
STREAM = 0x10
G, W, COPY, M, V, SCALES, CONTROL = (0x100000 * i for i in range(1, 8))


class Tensor(C.Structure):
    _fields_ = [("g", C.c_void_p), ("w", C.c_void_p), ("copy", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("scales", C.c_void_p), ("n", C.c_uint64), ("weight_decay", C.c_float), ("types", C.c_uint32)]


class Config(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("scale", C.c_double),
                ("step", C.c_uint64), ("seed", C.c_uint64)]


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    if not all(os.path.exists(o) for o in cuda_build.OBJECTS):
        cuda_build.build(force=True)
    path = str(tmp_path_factory.mktemp("host") / "libnuq_host.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I/usr/local/cuda/include", "-Wl,-Bsymbolic", "-o", path,
                    os.path.join(HERE, "fake_cudart.cpp")] + cuda_build.OBJECTS, check=True)
    return path


@pytest.fixture()
def lib(built, tmp_path):
    lib = C.CDLL(shutil.copy(built, tmp_path))
    lib.nuq_grad_norm.argtypes = [C.c_void_p, C.c_uint32, C.c_float, C.c_float, C.c_void_p, C.c_void_p]
    lib.nuq_adamw.argtypes = [C.c_void_p, C.c_uint32, C.POINTER(Config), C.c_void_p, C.c_void_p]
    lib.fake_events.restype = C.c_char_p
    return lib


def _launches(lib):
    return [e for e in lib.fake_events().decode().splitlines() if e.startswith("launch")]


def _tensor(**kw):
    return Tensor(**{"g": G, "w": W, "copy": COPY, "m": M, "v": V, "scales": SCALES, "n": 1000, "weight_decay": 0.1, "types": 0, **kw})


def _array(*tensors):
    return (Tensor * max(1, len(tensors)))(*tensors)


def _config(**kw):
    return Config(**{"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "scale": 1.0, "step": 1, "seed": 0, **kw})


BITS8, BF16, COPY16 = 1 << 16, 1, 1 << 8
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw", [dict(g=None), dict(g=G + 2), dict(types=BF16, g=G + 1), dict(w=None), dict(w=W + 2), dict(m=None), dict(m=M + 1), dict(v=None),
                                dict(v=V + 2), dict(types=COPY16, copy=None), dict(types=COPY16, copy=COPY + 1), dict(types=BITS8, scales=None),
                                dict(types=BITS8, scales=SCALES + 4), dict(types=3), dict(types=3 << 8), dict(types=2 << 16), dict(types=1 << 24),
                                dict(n=1 << 40), dict(weight_decay=NAN), dict(weight_decay=-1.0), dict(weight_decay=INF)])
def test_adamw_refuses_a_tensor(lib, kw):
    bad = _tensor(**kw)
    assert lib.nuq_adamw(_array(_tensor(), bad), 2, _config(), None, STREAM) == -1
    assert not _launches(lib)


@pytest.mark.parametrize("kw", [dict(lr=NAN), dict(lr=-1e-9), dict(lr=INF), dict(lr=1e13), dict(beta1=1.0), dict(beta1=-0.5), dict(beta1=NAN), dict(beta2=1.0), dict(beta2=NAN),
                                dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(scale=NAN), dict(scale=INF), dict(scale=-INF), dict(step=0)])
def test_adamw_refuses_constants(lib, kw):
    assert lib.nuq_adamw(_array(_tensor()), 1, _config(**kw), None, STREAM) == -1
    if "step" not in kw:
        assert lib.nuq_adamw(_array(_tensor()), 1, _config(**kw), CONTROL, STREAM) == -1
    assert not _launches(lib)


def test_adamw_refuses_other_arguments(lib):
    assert lib.nuq_adamw(None, 1, _config(), None, STREAM) == -1
    assert lib.nuq_adamw(_array(_tensor()), 1, None, None, STREAM) == -1
    assert lib.nuq_adamw(_array(_tensor()), 1, _config(), CONTROL + 8, STREAM) == -1
    assert not _launches(lib)


@pytest.mark.parametrize("kw", [dict(g=None), dict(g=G + 2), dict(types=BF16, g=G + 1), dict(types=3), dict(n=1 << 40)])
def test_norm_refuses_a_tensor(lib, kw):
    assert lib.nuq_grad_norm(_array(_tensor(), _tensor(**kw)), 2, 1.0, 1.0, CONTROL, STREAM) == -1
    assert not _launches(lib)


@pytest.mark.parametrize("scale,max_norm,control", [(NAN, 1.0, CONTROL), (INF, 1.0, CONTROL), (1.0, 0.0, CONTROL), (1.0, -1.0, CONTROL), (1.0, NAN, CONTROL),
                                                    (1.0, 1.0, None), (1.0, 1.0, CONTROL + 8)])
def test_norm_refuses_other_arguments(lib, scale, max_norm, control):
    assert lib.nuq_grad_norm(_array(_tensor()), 1, scale, max_norm, control, STREAM) == -1
    assert lib.nuq_grad_norm(None, 1, 1.0, 1.0, CONTROL, STREAM) == -1
    assert not _launches(lib)


def test_what_is_looked_at(lib):
    """the norm looks at gradients alone; pointers that a tensor's types or its length make no use of may be anything"""
    only = Tensor(g=G + 2, n=1, types=BF16, weight_decay=NAN)
    assert lib.nuq_grad_norm(_array(only), 1, 1.0, INF, CONTROL, STREAM) == 0
    assert lib.nuq_adamw(_array(_tensor(copy=None, scales=None), _tensor(types=BITS8, copy=1, m=M + 1, v=V + 3), Tensor()), 3, _config(), None, STREAM) == 0
    assert lib.nuq_adamw(_array(_tensor()), 1, _config(step=0), CONTROL, STREAM) == 0
    assert lib.nuq_grad_norm(None, 0, 1.0, INF, CONTROL, STREAM) == 0 and lib.nuq_adamw(None, 0, _config(), None, STREAM) == 0


@pytest.mark.parametrize("count,types,launches", [(0, 0, 0), (1, 0, 1), (400, 0, 1), (401, 0, 2), (400, BITS8, 1), (801, BITS8, 3)])
def test_launches_of_a_step(lib, count, types, launches):
    lib.fake_capture(1)                                     # (nothing is asked for that a capture does not allow)
    assert lib.nuq_adamw(_array(*[_tensor(types=types, n=1 + i) for i in range(count)]), count, _config(), None, STREAM) == 0
    assert len(_launches(lib)) == launches and "refused" not in lib.fake_events().decode()


def test_both_kinds_of_states_take_a_launch_each(lib):
    assert lib.nuq_adamw(_array(_tensor(), _tensor(types=BITS8), _tensor(), _tensor(n=0, types=BITS8)), 4, _config(), None, STREAM) == 0
    assert len(_launches(lib)) == 2


@pytest.mark.parametrize("count,n,launches", [(0, 5, 1), (1, 0, 1), (1536, 5, 1), (1537, 5, 2), (3, (1 << 40) - 1, 1), (9, (1 << 40) - 1, 2)])
def test_launches_of_a_norm(lib, count, n, launches):
    lib.fake_capture(1)
    assert lib.nuq_grad_norm(_array(*[_tensor(n=n) for _ in range(count)]), count, 1.0, 1.0, CONTROL, STREAM) == 0
    assert len(_launches(lib)) == launches and "refused" not in lib.fake_events().decode()


# ---- the reference that the GPU tests compare with ----

def test_the_reference_s_codes_are_e4m3():
    torch = pytest.importorskip("torch")
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(R.CODES, want, equal_nan=True)


def test_the_reference_rounds_to_neighbours_and_keeps_the_mean():
    rng = np.random.default_rng(0)
    x = rng.standard_normal(4096) * 10.0 ** rng.uniform(-5, 0, 4096)
    unit = (R.largest(x) / 448.0)[np.arange(4096) // R.BLOCK]
    grid = np.sort(R.CODES[:127])
    above = np.searchsorted(grid, np.abs(x) / unit, side="right")
    low, high = grid[above - 1], grid[np.minimum(above, 126)]
    p = (np.abs(x) / unit - low) / np.where(high > low, high - low, 1.0)
    ups = np.zeros(4096)
    for bits in range(0, 1 << 16, 257):                     # 256 evenly spaced draws
        code, _ = R.coded(x, np.zeros(4096), np.full(4096, bits))
        got = np.abs(R.CODES[code])
        assert ((got == low) | (got == high)).all() and np.array_equal(np.signbit(R.CODES[code]), np.signbit(x))
        ups += got == high
    # (a block's largest magnitude lies on the grid's end, up to the rounding of its quotient: there low is as good as high)
    assert (np.abs(ups / 256 - p) <= 1.5 / 256)[high > low].all()


def test_the_reference_s_random_bits_are_philox():
    oracle = pytest.importorskip("oracle")
    seed = 0xABCDEF0123456789
    got = R.philox(np.array([0, 5, (3 << 32) + 7]), 11, 2, seed)
    for q, row in zip((0, 5, (3 << 32) + 7), got):
        want = oracle.philox4x32_10([q & 0xFFFFFFFF, q >> 32, 11, 2], [seed & 0xFFFFFFFF, seed >> 32])
        assert list(row) == list(want)


# ---- the decoder with the step ----

def _decode(lib, K=3, d=100_000, bucket=1024, s=4, likely=0xFFFFFFFF, acc=None, w=W, m=M, v=V, decay=0.1, config=None, control=None, streams=None):
    lib.nuq_decode_adamw.argtypes = [C.POINTER(C.c_void_p), C.c_uint32, C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint32, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_void_p, C.c_float, C.POINTER(Config), C.c_void_p, C.c_void_p]
    array = (C.c_void_p * max(1, K))(*(streams or [0x2000] * max(1, K)))
    return lib.nuq_decode_adamw(array, K, d, bucket, s, likely, acc, w, m, v, decay, config or _config(), control, STREAM)


@pytest.mark.parametrize("kw", [dict(K=0), dict(K=65), dict(d=0), dict(d=1 << 40), dict(bucket=1000), dict(s=0), dict(s=15), dict(w=None), dict(m=None), dict(v=None),
                                dict(w=W + 4), dict(m=M + 8), dict(v=V + 4), dict(acc=G + 4), dict(decay=-1.0), dict(decay=NAN), dict(likely=3 << 16), dict(likely=3 << 8),
                                dict(likely=1), dict(likely=1 << 24), dict(config=_config(step=0)), dict(config=_config(lr=NAN)), dict(config=_config(scale=INF)),
                                dict(control=CONTROL + 4), dict(streams=[0x2000, None, 0x2000]), dict(streams=[0x2000, 0x2008, 0x2000])])
def test_decode_adamw_refuses(lib, kw):
    assert _decode(lib, **kw) == -1
    assert not _launches(lib)


@pytest.mark.parametrize("likely,kernel", [(0, "decode_chains_kernel"), (1 << 16, "decode_fields_kernel"), (2 << 16, "decode_chains_kernel"), (1 << 16 | 1 << 8, "decode_chains_kernel"),
                                           (0xFFFFFFFF, "decode_chains_kernel")])
def test_decode_adamw_takes_the_likely_kernel(lib, likely, kernel):
    for K in (1, 2, 3, 40):                                 # (the sum is needed by nobody, however many streams there are)
        assert _decode(lib, K=K, likely=likely) == 0
    assert len(_launches(lib)) == 4 and all(kernel in e and "AdamwSum" in e and e.endswith("unordered 0") for e in _launches(lib))


def test_decode_adamw_in_a_capture_needs_a_call_before(lib):
    lib.fake_capture(1)
    assert _decode(lib) == -4
    lib.fake_capture(0)
    assert _decode(lib) == 0
    lib.fake_capture(1)
    assert _decode(lib, control=CONTROL, config=_config(step=0)) == 0


@pytest.mark.parametrize("lr,decay,rc", [(2.0, 1e38, 0), (2.0, 3e38, -1), (2.0 ** 40, 2.0 ** 87, 0), (2.0 ** 40, 2.0 ** 88, -1), (0.0, 3.4e38, 0), (1e-3, 3.4e38, 0)])
def test_a_decay_that_fp32_cannot_hold_is_refused(lib, lr, decay, rc):
    """lr weight_decay is formed once for all of a tensor's elements: infinite, it would make NaN of every parameter that is 0"""
    for n in (1000, 0):
        assert lib.nuq_adamw(_array(_tensor(), _tensor(weight_decay=decay, n=n)), 2, _config(lr=lr), None, STREAM) == rc
    assert lib.nuq_adamw(_array(_tensor(weight_decay=decay)), 1, _config(lr=lr), CONTROL, STREAM) == rc
    assert len(_launches(lib)) == (0 if rc else 3)
    assert _decode(lib, decay=decay, config=_config(lr=lr)) == rc
    assert lib.nuq_grad_norm(_array(_tensor(weight_decay=decay)), 1, 1.0, 1.0, CONTROL, STREAM) == 0


# ---- the binding ----

def test_containers_in_host_memory_are_refused():
    """their addresses went to the kernels as they were"""
    torch = pytest.importorskip("torch")
    from paper_1908_06077_b200 import nuq
    host = [torch.zeros(64, dtype=torch.int32)] * 2
    x = [torch.zeros(256) for _ in range(4)]
    for bad in (lambda: nuq.decode_accumulate(host, 256, 256, 3), lambda: nuq.decode_accumulate(host, 256, 256, 3, acc=x[0]),
                lambda: nuq.decode_update(host, 256, 256, 3, x[0], acc=x[1]), lambda: nuq.decode_adamw(host, 256, 256, 3, *x[:3], lr=0.1, step=1)):
        with pytest.raises(ValueError):
            bad()


def test_containers_on_another_device_are_refused():
    from paper_1908_06077_b200 import nuq

    class On:
        def __init__(self, index):
            self.index = index

        def get_device(self):
            return self.index

        def data_ptr(self):
            return 4096

    assert list(nuq._pointers([On(1), On(1)], On(1), None, On(1))) == [4096, 4096]
    for streams, others in (([On(0)], [On(1)]), ([On(1), On(0)], [On(1)]), ([On(1), On(-1)], [On(1)]), ([On(-1)], [On(-1)]), ([On(0)], [On(0), On(1)]), ([On(0)], [On(0), None, On(-1)])):
        with pytest.raises(ValueError):
            nuq._pointers(streams, *others)
