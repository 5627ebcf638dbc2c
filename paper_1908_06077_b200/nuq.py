"""Thin ctypes binding of libnuq.so: argument marshalling only.

Every function has the name and the argument order of its C counterpart in
include/nuq.h; tensors are passed as raw device pointers and the current torch
CUDA stream is used unless one is given.  There is no CPU path: importing this
module fails if the CUDA library cannot be built or loaded.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

from . import build as _build

NUQ_OK, ERR_INVALID_ARG, ERR_CAPACITY, ERR_BAD_STREAM, ERR_CUDA, ERR_TIMEOUT, ERR_INTERNAL = 0, -1, -2, -3, -4, -5, -6
WARN_NONFINITE = 1
NORM_L2, NORM_LINF = 0, 1
LEVELS_EXP, LEVELS_UNIFORM, LEVELS_TABLE = 0 << 8, 1 << 8, 2 << 8
MODE_ERC, MODE_FIXED, MODE_CODED = 0 << 16, 1 << 16, 2 << 16
TEST_NORMS = 1 << 24
TEST_SHORT_PATIENCE = 1 << 25
HEADER_WORDS = 16
STATIC_SCRATCH_BYTES = 512 * 1024
GRAD_F32, GRAD_BF16, GRAD_F16 = 0, 1, 2
COPY_NONE, COPY_BF16, COPY_F16 = 0 << 8, 1 << 8, 2 << 8
STATES_F32, STATES_8BIT = 0 << 16, 1 << 16
STATE_BLOCK = 256
CONTROL_BYTES = 16384
LIKELY_AS_KNOWN = 0xFFFFFFFF


class NuqError(RuntimeError):
    def __init__(self, where, code):
        super().__init__(f"{where} failed with status {code}")
        self.code = code


class _Info(C.Structure):
    _fields_ = [("d", C.c_uint64), ("bucket", C.c_uint32), ("s", C.c_uint32), ("flags", C.c_uint32),
                ("sub_block", C.c_uint32), ("nblk", C.c_uint64), ("container_bits", C.c_uint64),
                ("code_bits", C.c_uint64), ("nnz", C.c_uint64)]


class _Tensor(C.Structure):
    _fields_ = [("g", C.c_void_p), ("w", C.c_void_p), ("copy", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("scales", C.c_void_p), ("n", C.c_uint64), ("weight_decay", C.c_float), ("types", C.c_uint32)]


class _AdamwConfig(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("scale", C.c_double),
                ("step", C.c_uint64), ("seed", C.c_uint64)]


def _load():
    path = _build.LIB
    if not os.path.exists(path):
        _build.build()
    lib = C.CDLL(path)
    lib.nuq_encode.restype = C.c_int
    lib.nuq_encode.argtypes = [C.c_void_p, C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint32, C.c_uint64, C.c_uint64,
                               C.c_void_p, C.c_void_p, C.c_void_p]
    lib.nuq_encode_static.restype = C.c_int
    lib.nuq_encode_static.argtypes = lib.nuq_encode.argtypes
    lib.nuq_decode_accumulate.restype = C.c_int
    lib.nuq_decode_accumulate.argtypes = [C.POINTER(C.c_void_p), C.c_uint32, C.c_uint64, C.c_uint32, C.c_uint32,
                                          C.c_void_p, C.c_void_p]
    lib.nuq_decode_update.restype = C.c_int
    lib.nuq_decode_update.argtypes = [C.POINTER(C.c_void_p), C.c_uint32, C.c_uint64, C.c_uint32, C.c_uint32,
                                      C.c_void_p, C.c_void_p, C.c_void_p, C.c_float, C.c_float, C.c_float, C.c_void_p]
    lib.nuq_grad_norm.restype = C.c_int
    lib.nuq_grad_norm.argtypes = [C.c_void_p, C.c_uint32, C.c_float, C.c_float, C.c_void_p, C.c_void_p]
    lib.nuq_adamw.restype = C.c_int
    lib.nuq_adamw.argtypes = [C.c_void_p, C.c_uint32, C.POINTER(_AdamwConfig), C.c_void_p, C.c_void_p]
    lib.nuq_decode_adamw.restype = C.c_int
    lib.nuq_decode_adamw.argtypes = [C.POINTER(C.c_void_p), C.c_uint32, C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint32,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float, C.POINTER(_AdamwConfig),
                                     C.c_void_p, C.c_void_p]
    lib.nuq_encode_bound.restype = C.c_uint64
    lib.nuq_encode_bound.argtypes = [C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint32]
    lib.nuq_set_level_table.restype = C.c_int
    lib.nuq_set_level_table.argtypes = [C.POINTER(C.c_float), C.c_uint32]
    lib.nuq_level_histogram.restype = C.c_int
    lib.nuq_level_histogram.argtypes = [C.c_void_p, C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint32, C.c_uint64,
                                        C.c_uint64, C.c_void_p, C.c_void_p]
    lib.nuq_fit_level_code.restype = C.c_int
    lib.nuq_fit_level_code.argtypes = [C.POINTER(C.c_uint64), C.c_uint32, C.POINTER(C.c_uint8)]
    lib.nuq_set_level_code.restype = C.c_int
    lib.nuq_set_level_code.argtypes = [C.POINTER(C.c_uint8), C.c_uint32]
    lib.nuq_set_test_norms.restype = C.c_int
    lib.nuq_set_test_norms.argtypes = [C.c_void_p]
    lib.nuq_last_status.restype = C.c_int
    lib.nuq_last_status.argtypes = [C.c_void_p]
    lib.nuq_stream_info.restype = C.c_int
    lib.nuq_stream_info.argtypes = [C.c_void_p, C.POINTER(_Info), C.c_void_p]
    lib.nuq_shutdown.restype = None
    lib.nuq_shutdown.argtypes = []
    lib.nuq_version.restype = C.c_char_p
    lib.nuq_version.argtypes = []
    return lib


_lib = _load()
LIBRARY_PATH = _build.LIB


_current_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _stream(stream):
    """A cudaStream_t as an integer: the current torch stream of the current device unless one is given."""
    if stream is None:
        return _current_raw_stream(_current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def version() -> str:
    return _lib.nuq_version().decode()


def encode_bound(d, bucket, s, norm_kind=0) -> int:
    return int(_lib.nuq_encode_bound(d, bucket, s, norm_kind))


def set_level_table(interior_levels):
    """interior levels l_1 < ... < l_s of the level sequence (0, l_1, ..., l_s, 1) used with LEVELS_TABLE"""
    vals = [float(x) for x in interior_levels]
    arr = (C.c_float * len(vals))(*vals)
    rc = _lib.nuq_set_level_table(arr, len(vals))
    if rc != NUQ_OK:
        raise NuqError("nuq_set_level_table", rc)


def level_histogram(g: torch.Tensor, bucket, s, norm_kind=0, seed=0, offset=0, hist=None, stream=None):
    """how often each level index 0..s+1 comes out of the quantizer for g: int64 CUDA tensor of s + 2 counters"""
    assert g.is_cuda and g.dtype == torch.float32 and g.is_contiguous()
    if hist is None:
        hist = torch.empty(s + 2, dtype=torch.int64, device=g.device)
    rc = _lib.nuq_level_histogram(g.data_ptr(), g.numel(), bucket, s, norm_kind, seed, offset,
                                  hist.data_ptr(), _stream(stream))
    if rc != NUQ_OK:
        raise NuqError("nuq_level_histogram", rc)
    return hist


def fit_level_code(hist, s):
    """code lengths of the level indices 1..s+1 (Huffman) from the s + 2 counts of level_histogram (host values)"""
    vals = [int(x) for x in hist]
    assert len(vals) == s + 2
    arr = (C.c_uint64 * len(vals))(*vals)
    out = (C.c_uint8 * (s + 1))()
    rc = _lib.nuq_fit_level_code(arr, s, out)
    if rc != NUQ_OK:
        raise NuqError("nuq_fit_level_code", rc)
    return list(out)


def set_level_code(lengths):
    """code lengths of the level indices 1..s+1 that MODE_CODED calls use from now on"""
    vals = [int(x) for x in lengths]
    arr = (C.c_uint8 * len(vals))(*vals)
    rc = _lib.nuq_set_level_code(arr, len(vals) - 1)
    if rc != NUQ_OK:
        raise NuqError("nuq_set_level_code", rc)


def set_test_norms(norms: torch.Tensor | None):
    """norms: CUDA float32 tensor of ceil(d/bucket) bucket norms (kept by reference), or None."""
    rc = _lib.nuq_set_test_norms(norms.data_ptr() if norms is not None else None)
    if rc != NUQ_OK:
        raise NuqError("nuq_set_test_norms", rc)


def encode(g: torch.Tensor, bucket, s, norm_kind=0, seed=0, offset=0, out=None, out_bits=None, stream=None):
    """c <- ENCODE(g).  Returns (out, out_bits): the container as an int32 CUDA tensor of
    nuq_encode_bound bytes and a one-element int64 CUDA tensor that receives container_bits."""
    assert g.is_cuda and g.dtype == torch.float32 and g.is_contiguous()
    d = g.numel()
    if out is None:
        nbytes = encode_bound(d, bucket, s, norm_kind)
        if nbytes == 0:
            raise NuqError("nuq_encode_bound", ERR_INVALID_ARG)
        out = torch.empty(nbytes // 4, dtype=torch.int32, device=g.device)
    if out_bits is None:
        out_bits = torch.empty(1, dtype=torch.int64, device=g.device)
    rc = _lib.nuq_encode(g.data_ptr(), d, bucket, s, norm_kind, seed, offset, out.data_ptr(),
                         out_bits.data_ptr(), _stream(stream))
    if rc != NUQ_OK:
        raise NuqError("nuq_encode", rc)
    return out, out_bits


def encode_static(g: torch.Tensor, bucket, s, norm_kind=0, seed=0, offset=0, *, out, out_bits, stream=None):
    """nuq_encode_static: the encoder for callers that may not allocate device memory.  Its
    scan state lives in a fixed array inside the library instead of a cudaMalloc'ed workspace,
    so `out` (encode_bound bytes) and `out_bits` (one int64) must be passed in and nothing is
    allocated here either.  Raises NuqError(ERR_CAPACITY) when d is too long for that array.
    Calls that could overlap on the GPU must be serialised by the caller."""
    assert g.is_cuda and g.dtype == torch.float32 and g.is_contiguous()
    rc = _lib.nuq_encode_static(g.data_ptr(), g.numel(), bucket, s, norm_kind, seed, offset,
                                out.data_ptr(), out_bits.data_ptr(), _stream(stream))
    if rc != NUQ_OK:
        raise NuqError("nuq_encode_static", rc)
    return out, out_bits


_pointer_arrays = {}


def _pointers(streams, *others):
    """the containers' addresses as a C array (copied by the call it is handed to); others: what has to be on the same CUDA device"""
    n = len(streams)
    index = others[0].get_device()
    found = [t.get_device() for t in streams] + [x.get_device() for x in others if x is not None]
    if index < 0 or found.count(index) != len(found):
        raise ValueError("containers, sums and parameters: CUDA tensors on one device are wanted")
    array = _pointer_arrays.get(n)
    if array is None:
        array = _pointer_arrays[n] = C.c_void_p * n
    return array(*[t.data_ptr() for t in streams])


def decode_accumulate(streams, d, bucket, s, acc=None, stream=None):
    """acc <- sum_k DECODE(streams[k]); acc is overwritten."""
    if acc is None:
        acc = torch.empty(d, dtype=torch.float32, device=streams[0].device)
    ptrs = _pointers(streams, acc)
    rc = _lib.nuq_decode_accumulate(ptrs, len(streams), d, bucket, s, acc.data_ptr(), _stream(stream))
    if rc != NUQ_OK:
        raise NuqError("nuq_decode_accumulate", rc)
    return acc


# Parameters are written through their addresses.  Autograd hears of it here, as of any write in place: a backward pass through
# a graph that saved them before the step is an error, not a wrong gradient.  (A replayed graph passes this by.)
_written = torch._C._increment_version


def decode_update(streams, d, bucket, s, w, yl=None, alpha=1.0, mu=0.0, l=0.0, acc=None, stream=None):
    """w <- w - (alpha / K) sum_k DECODE(streams[k]), or the momentum rule with yl when mu != 0; in place."""
    ptrs = _pointers(streams, w, yl, acc)
    rc = _lib.nuq_decode_update(ptrs, len(streams), d, bucket, s, acc.data_ptr() if acc is not None else None,
                                w.data_ptr(), yl.data_ptr() if yl is not None else None,
                                alpha, mu, l, _stream(stream))
    if rc != NUQ_OK:
        raise NuqError("nuq_decode_update", rc)
    _written((w,))
    return w


_GRADS = {torch.float32: GRAD_F32, torch.bfloat16: GRAD_BF16, torch.float16: GRAD_F16}
_COPIES = {torch.bfloat16: COPY_BF16, torch.float16: COPY_F16}
_STATES = {torch.float32: STATES_F32, torch.uint8: STATES_8BIT}
_F32 = (torch.float32,)
_ITEM = {torch.float32: 4, torch.bfloat16: 2, torch.float16: 2, torch.uint8: 1}


class Tensors:
    """A list of tensors as grad_norm and adamw take it (see `tensors`).  It holds their addresses and keeps the tensors alive; their
    contents are looked at by the calls it is given to.  So it serves step after step as long as the tensors stay where they are: a
    gradient that is allocated anew in every step (zero_grad(set_to_none=True), decode_accumulate without acc) needs a new list
    each time, the old one would go on with the old gradient."""

    def __init__(self, array, device, kept, states, written):
        self.array, self.device, self.kept, self.states, self.written = array, device, kept, states, written
        self.count, self.address = len(array), C.addressof(array)

    def __len__(self):
        return self.count


def tensors(g, w=None, m=None, v=None, scales=None, copy=None, weight_decay=0.0) -> Tensors:
    """The list of tensors for grad_norm (gradients alone) and adamw.

    g     gradients: contiguous CUDA tensors of float32, bfloat16 or float16
    w     parameters, float32, as many elements each
    m, v  states: both float32, or both uint8 (codes) with `scales`, float32 of 2 * ceil(n / 256) elements
    copy  bfloat16 or float16 copies of the parameters; the list or an entry may be None
    weight_decay  one number, or one per tensor
    Raises ValueError where shapes, types, devices or alignment do not fit, or where written memory is given twice."""
    g = list(g)
    count = len(g)
    lists = {"g": g, "w": w, "m": m, "v": v, "scales": scales, "copy": copy}
    for name, x in lists.items():
        x = lists[name] = [None] * count if x is None else list(x)
        if len(x) != count:
            raise ValueError(f"{name}: {len(x)} tensors for {count} gradients")
    decays = [float(weight_decay)] * count if isinstance(weight_decay, (int, float)) else [float(x) for x in weight_decay]
    if len(decays) != count:
        raise ValueError(f"weight_decay: {len(decays)} numbers for {count} gradients")
    states = w is not None
    if not states and any(x is not None for x in (m, v, scales, copy)):
        raise ValueError("states or copies without parameters")
    device = g[0].device if count and isinstance(g[0], torch.Tensor) else None
    on = -1 if device is None or device.type != "cuda" else device.index
    rows, spans = [], []                                    # the C array, eight words a tensor; what memory holds what

    def place(name, i, types, n, writes=True):
        x = lists[name][i]
        if not isinstance(x, torch.Tensor) or x.dtype not in types or x.numel() != n or not x.is_contiguous() or on < 0 or x.get_device() != on:
            raise ValueError(f"{name}[{i}]: a contiguous tensor of {n} elements, {' or '.join(map(str, types))}, on the CUDA device of the first gradient is wanted")
        p = x.data_ptr()
        if n:
            spans.append((p, p + n * _ITEM[x.dtype], writes, name, i))
        return p

    for i, x in enumerate(g):
        n = x.numel() if isinstance(x, torch.Tensor) else 0
        row = [place("g", i, _GRADS, n, False), 0, 0, 0, 0, 0, n, 0]
        types = _GRADS[x.dtype]
        if states:
            row[1] = place("w", i, _F32, n)
            row[3] = place("m", i, _STATES, n)
            kind = lists["m"][i].dtype
            row[4] = place("v", i, (kind,), n)
            types |= _STATES[kind]
            if kind is torch.uint8:
                row[5] = place("scales", i, _F32, 2 * -(-n // STATE_BLOCK))
                if row[5] % 8:
                    raise ValueError(f"scales[{i}]: 8-byte alignment is wanted")
            if lists["copy"][i] is not None:
                row[2] = place("copy", i, _COPIES, n)
                types |= _COPIES[lists["copy"][i].dtype]
        row[7] = types << 32 | int.from_bytes(C.c_float(decays[i]), "little")
        rows += row
    written = read = (0, 0, False, "", 0)                   # the spans that reach furthest, of what is written and of what is read
    for span in sorted(spans):
        for other in (written, read) if span[2] else (written,):    # (gradients may be given twice)
            if span[0] < other[1]:
                raise ValueError(f"{span[3]}[{span[4]}] and {other[3]}[{other[4]}] overlap")
        if span[2]:
            written = span
        elif span[1] > read[1]:
            read = span
    words = (C.c_uint64 * len(rows))(*rows)
    array = (_Tensor * count).from_buffer(words)
    # (a tensor and the parts of it share one version)
    versions = {}
    for x in (*lists["w"], *lists["copy"]):
        if x is not None:
            x = x if (base := x._base) is None else base
            versions[id(x)] = x
    return Tensors(array, device, (g, lists), states, tuple(versions.values()))


def step_control(step=0, device=None) -> torch.Tensor:
    """A step's record on the device (nuq_control): an int64 CUDA tensor, steps taken set to `step`, the learning rate's factor to 1.
    grad_norm begins the next step; until it has, steps with the record change nothing."""
    control = torch.zeros(CONTROL_BYTES // 8, dtype=torch.int64, device="cuda" if device is None else device)
    control[0] = int(step)
    control.view(torch.float32)[4] = 1.0
    return control


def control_fields(control) -> dict:
    """The record's fields as views of it (CUDA tensors of one element): step, norm, scale, lr_factor, skip."""
    f = control.view(torch.float32)
    return {"step": control[0], "norm": f[2], "scale": f[3], "lr_factor": f[4], "skip": control.view(torch.int32)[5]}


def _control(control, device):
    if control is None:
        return None
    if not control.is_cuda or control.dtype is not torch.int64 or not control.is_contiguous() or 8 * control.numel() < CONTROL_BYTES:
        raise ValueError(f"control: a contiguous int64 CUDA tensor of {CONTROL_BYTES // 8} elements is wanted")
    if device is not None and control.get_device() != device.index:
        raise ValueError(f"control: on {control.device}, the tensors are on {device}")
    return control.data_ptr()


def _config(lr, beta1, beta2, eps, scale, step, seed):
    if not 0 <= step < 1 << 64:                             # (ctypes would take what is left of it)
        raise ValueError(f"step: {step}")
    return _AdamwConfig(lr, beta1, beta2, eps, scale, step, seed & 0xFFFFFFFFFFFFFFFF)


def _on_device(index, stream, function, *args):
    """function(*args, raw stream) with device `index` current (the stream, if none is given, is its current one)"""
    if index is None or index == _current_device():
        return function(*args, _stream(stream))
    with torch.cuda.device(index):
        return function(*args, _stream(stream))


def grad_norm(list_, control, max_norm=float("inf"), scale=1.0, stream=None):
    """The gradients' Euclidean norm, the factor that clips it to max_norm and the beginning of the next step, all into
    `control` (see control_fields).  list_: from `tensors`."""
    where = _control(control, list_.device)
    rc = _on_device(control.get_device(), stream, _lib.nuq_grad_norm, list_.address, list_.count, scale, max_norm, where)
    if rc != NUQ_OK:
        raise NuqError("nuq_grad_norm", rc)
    return control


def adamw(list_, lr, beta1=0.9, beta2=0.999, eps=1e-8, step=0, scale=1.0, seed=0, control=None, stream=None):
    """One AdamW step over the tensors of list_ (from `tensors`), in place.  step: its number, from 1 on, or `control`."""
    if not list_.states:
        raise ValueError("a list of gradients alone")
    where = _control(control, list_.device)
    config = _config(lr, beta1, beta2, eps, scale, step, seed)
    rc = _on_device(list_.device and list_.device.index, stream, _lib.nuq_adamw, list_.address, list_.count, C.byref(config), where)
    if rc != NUQ_OK:
        raise NuqError("nuq_adamw", rc)
    _written(list_.written)


def decode_adamw(streams, d, bucket, s, w, m, v, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=0, scale=1.0,
                 control=None, likely=LIKELY_AS_KNOWN, acc=None, stream=None):
    """An AdamW step with the mean of DECODE(streams[k]) as the gradient; w, m and v (float32, d elements) in place.
    step: its number, from 1 on, or `control`.  likely: what the streams most likely are, as encode was told (MODE_* | LEVELS_*);
    received containers are not known by their addresses."""
    index = w.get_device()
    for name, x in (("w", w), ("m", m), ("v", v)) + ((("acc", acc),) if acc is not None else ()):
        if x.get_device() != index or index < 0 or x.dtype is not torch.float32 or not x.is_contiguous() or x.numel() != d:
            raise ValueError(f"{name}: a contiguous float32 CUDA tensor of {d} elements is wanted, all on one device")
    places = sorted((x.data_ptr(), x.data_ptr() + 4 * d) for x in (w, m, v, acc) if x is not None)
    if any(a[1] > b[0] for a, b in zip(places, places[1:])):
        raise ValueError("w, m, v and acc overlap")
    where = _control(control, w.device)
    config = _config(lr, beta1, beta2, eps, scale, step, 0)
    ptrs = _pointers(streams, w)
    rc = _on_device(index, stream, _lib.nuq_decode_adamw, ptrs, len(streams), d, bucket, s, likely,
                    acc.data_ptr() if acc is not None else None, w.data_ptr(), m.data_ptr(), v.data_ptr(), weight_decay,
                    C.byref(config), where)
    if rc != NUQ_OK:
        raise NuqError("nuq_decode_adamw", rc)
    _written((w,))
    return w


def last_status(stream=None) -> int:
    return int(_lib.nuq_last_status(_stream(stream)))


def stream_info(out: torch.Tensor, stream=None) -> dict:
    info = _Info()
    rc = _lib.nuq_stream_info(out.data_ptr(), C.byref(info), _stream(stream))
    if rc != NUQ_OK:
        raise NuqError("nuq_stream_info", rc)
    return {k: int(getattr(info, k)) for k, _ in _Info._fields_}


def shutdown():
    _lib.nuq_shutdown()
