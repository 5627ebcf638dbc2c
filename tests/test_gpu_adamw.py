"""AdamW over lists of tensors (nuq_adamw) and the gradients' norm (nuq_grad_norm) against their formulas in 64 bits."""
import numpy as np
import pytest

import adamw_reference as R
from gpu_util import require_cuda

pytestmark = pytest.mark.gpu

GUARD = 64
GRADS = ["float32", "bfloat16", "float16"]
# one element, less than a block, a block, its ends, a tile's ends, several tiles
SIZES = [1, 3, 255, 256, 257, 2047, 2048, 2049, 6000, 0, 20011]


class Guarded:
    """`host` on the device, `skew` elements behind an aligned address, with a pattern around it that has to stay."""

    def __init__(self, torch, host, skew=0):
        self.torch, self.n, self.at = torch, host.numel(), GUARD + skew
        self.buf = torch.full((self.n + 2 * GUARD + skew,), 77, dtype=host.dtype, device="cuda")
        self.view = self.buf[self.at:self.at + self.n]
        self.view.copy_(host)

    def read(self):
        around = self.torch.cat([self.buf[:self.at], self.buf[self.at + self.n:]])
        assert bool((around == 77).all()), "written outside"
        return self.view.cpu()


def _list(torch, nuq, sizes, grad="float32", copy=None, bits=32, skew=0, seed=0, zero=False, decays=None, magnitude=1.0, skews=None):
    """tensors of the given sizes with states as in training (or zero), and their list"""
    rng = np.random.default_rng(seed)
    t = []
    for i, n in enumerate(sizes):
        k = skew if skews is None else skews[i % len(skews)]
        size = 10.0 ** rng.uniform(-3, 0) * magnitude
        x = {"g": torch.from_numpy((rng.standard_normal(n) * size).astype(np.float32)).to(getattr(torch, grad)),
             "w": torch.from_numpy(rng.standard_normal(n).astype(np.float32) * np.float32(0.1))}
        m, r = rng.standard_normal(n) * 0.3 * size, (np.abs(rng.standard_normal(n)) + 0.2) * size
        blocks = -(-n // R.BLOCK)
        if bits == 32:
            x["m"], x["v"] = torch.from_numpy(m.astype(np.float32) * (not zero)), torch.from_numpy((r * r).astype(np.float32) * (not zero))
        else:
            scales = rng.uniform(0.5, 2.0, (blocks, 2)) * size / 448.0 * (not zero)
            x["m"] = torch.from_numpy(rng.integers(0, 256, n).astype(np.uint8) * np.uint8(not zero))
            x["v"] = torch.from_numpy(rng.integers(0, 127, n).astype(np.uint8) * np.uint8(not zero))
            x["m"][(x["m"] & 127) == 127] = 5                # (NaN is tested by itself)
            x["scales"] = torch.from_numpy(scales.astype(np.float32).reshape(-1))
        if copy:
            x["copy"] = torch.zeros(n, dtype=getattr(torch, copy))
        t.append({name: Guarded(torch, y, k if name != "scales" else 0) for name, y in x.items()})
    decays = [0.1 * (i % 2) for i in range(len(sizes))] if decays is None else decays
    col = lambda name: [x[name].view for x in t]  # noqa: E731
    lst = nuq.tensors(col("g"), col("w"), col("m"), col("v"), scales=col("scales") if bits == 8 else None,
                      copy=col("copy") if copy else None, weight_decay=decays)
    return t, lst, decays


def _numpy(x):
    return x.float().numpy() if x.dtype.is_floating_point else x.numpy()


def _read(t):
    return [{name: _numpy(y.read()) for name, y in x.items()} for x in t]


def _copy_bound(copy, w):
    """half a step of the copy's type"""
    return np.abs(w) * (2.0 ** -8 if copy == "bfloat16" else 2.0 ** -11) + 2.0 ** -25


def _check(before, after, decays, t, bits, scale=1.0, copy=None, seed=0, lr=R.LR, beta1=R.BETA1, beta2=R.BETA2, eps=R.EPS, first=0):
    """every array of every tensor against the 64-bit step from what the device held before; returns how many codes were undecided"""
    undecided = total = 0
    for j, (a, b, decay) in enumerate(zip(before, after, decays)):
        n = a["w"].size
        if bits == 32:
            m0, v0 = a["m"], a["v"]
        else:
            m0, v0 = R.held(a["m"], a["scales"][0::2]), R.held(a["v"], a["scales"][1::2]) ** 2
        m, v, dm, dv = R.moments(a["g"], m0, v0, scale, beta1, beta2)
        if bits == 8:                                        # (what the codes stand for is rounded too, v's root before it is squared)
            dm, dv = dm + 2 * R.U * np.abs(m0), dv + 6 * R.U * v0
        w, dw = R.step(a["w"], m, v, dm, dv, t, np.float32(decay), lr, beta1, beta2, eps)
        assert (np.abs(b["w"] - w) <= dw).all(), (j, n, np.max(np.abs(b["w"] - w) / dw))
        assert np.array_equal(a["g"], b["g"])
        if copy:
            assert (np.abs(b["copy"] - b["w"]) <= _copy_bound(copy, b["w"])).all()
        if bits == 32:
            assert (np.abs(b["m"] - m) <= dm).all() and (np.abs(b["v"] - v) <= dv).all(), (j, n)
            continue
        if n == 0:
            continue
        words = R.philox(np.arange(-(-n // 4)) + first // 4, t, j, seed).reshape(-1)[:n].astype(np.int64)
        root, droot = np.sqrt(v), dv / (2.0 * np.sqrt(np.maximum(v, 1e-300))) + R.U * np.sqrt(v)
        for name, x, dx, random, k in (("m", m, dm, words & 0xFFFF, 0), ("v", root, droot, words >> 16, 1)):
            most = R.largest(x)
            assert (np.abs(b["scales"][k::2] - most / 448.0) <= (8 * R.U * most + dx.max()) / 448.0).all()
            code, sure = R.coded(x, dx, random, root=name == "v")
            got = b[name].astype(np.int64)
            assert np.array_equal(got[sure], code[sure]), (j, name, np.flatnonzero(sure & (got != code))[:5])
            # one code further at most, where 64 bits cannot tell (the sign can only differ where m is as good as zero)
            near = (np.abs((got & 127) - (code & 127)) <= 1) & (((got ^ code) < 128) | (np.abs(x) <= dx))
            assert near.all()
            undecided += int((~sure & (got != code)).sum())
            total += n
    assert undecided <= 4 + 2e-4 * total, (undecided, total)
    return undecided


@pytest.mark.parametrize("skew", [0, 1, 2])
@pytest.mark.parametrize("grad", GRADS)
@pytest.mark.parametrize("copy", [None, "bfloat16", "float16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_of_every_type_and_alignment(bits, copy, grad, skew):
    torch, nuq = require_cuda()
    t, lst, decays = _list(torch, nuq, SIZES, grad, copy, bits, skew, seed=3 * skew + bits)
    before = _read(t)
    nuq.adamw(lst, lr=R.LR, step=7, scale=0.5, seed=0xABCDEF0123456789)
    _check(before, _read(t), decays, 7, bits, 0.5, copy, 0xABCDEF0123456789)


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_of_different_alignment_in_one_list(bits):
    torch, nuq = require_cuda()
    t, lst, decays = _list(torch, nuq, [5000, 5000, 5000, 5000, 5000, 300], "float32", "bfloat16", bits, skews=[0, 1, 4, 3, 8, 2], seed=5)
    before = _read(t)
    nuq.adamw(lst, lr=R.LR, step=1, seed=1)
    _check(before, _read(t), decays, 1, bits, 1.0, "bfloat16", 1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kw", [dict(beta1=0.0), dict(beta2=0.0), dict(beta1=0.0, beta2=0.0), dict(lr=0.0), dict(eps=1.0), dict(beta1=0.95, beta2=0.99, lr=0.3),
                                dict(step=1 << 40), dict(step=2)])
def test_constants(bits, kw):
    torch, nuq = require_cuda()
    kw = {"lr": R.LR, "step": 3, **kw}
    t, lst, decays = _list(torch, nuq, [1000, 4096], bits=bits, seed=8)
    before = _read(t)
    nuq.adamw(lst, seed=2, **kw)
    step = kw.pop("step")
    _check(before, _read(t), decays, step, bits, seed=2, **kw)


@pytest.mark.parametrize("bits", [32, 8])
def test_first_steps_from_zero_states(bits):
    """states of all zeros are the ones before the first step; ten steps, each checked from where the device was"""
    torch, nuq = require_cuda()
    t, lst, decays = _list(torch, nuq, [257, 3000], bits=bits, zero=True, seed=11)
    rng = np.random.default_rng(1)
    for step in range(1, 11):
        for x in t:
            x["g"].view.copy_(torch.from_numpy(rng.standard_normal(x["g"].n).astype(np.float32)))
        before = _read(t)
        nuq.adamw(lst, lr=0.01, step=step, seed=step)
        _check(before, _read(t), decays, step, bits, seed=step, lr=0.01)


@pytest.mark.parametrize("bits,count", [(32, 17), (32, 177), (32, 401), (32, 1000), (8, 401), (8, 16)])
def test_more_tensors_than_a_launch_takes(bits, count):
    torch, nuq = require_cuda()
    sizes = [1 + (37 * i) % 700 for i in range(count)]
    t, lst, decays = _list(torch, nuq, sizes, bits=bits, seed=13)
    before = _read(t)
    nuq.adamw(lst, lr=R.LR, step=5, seed=3)
    _check(before, _read(t), decays, 5, bits, seed=3)


def test_states_of_both_kinds_in_one_list():
    torch, nuq = require_cuda()
    a, _, _ = _list(torch, nuq, [500, 70], bits=32, seed=1)
    b, _, _ = _list(torch, nuq, [3000, 256], bits=8, seed=2)
    every = [a[0], b[0], a[1], b[1]]
    lst = nuq.tensors([x["g"].view for x in every], [x["w"].view for x in every], [x["m"].view for x in every], [x["v"].view for x in every],
                      scales=[x["scales"].view if "scales" in x else None for x in every], weight_decay=[0.0, 0.1, 0.2, 0.3])
    before = _read(every)
    nuq.adamw(lst, lr=R.LR, step=4, seed=6)
    after = _read(every)
    _check([before[0], before[2]], [after[0], after[2]], [0.0, 0.2], 4, 32)
    # (the random bits go by a tensor's place in the list)
    nothing = {k: np.zeros(0, v.dtype) for k, v in before[1].items()}
    _check([nothing, before[1], nothing, before[3]], [nothing, after[1], nothing, after[3]], [0, 0.1, 0, 0.3], 4, 8, seed=6)


def test_8_bit_states_keep_their_mean():
    """The same step from the same states with 400 seeds: the mean of what is stored is the moment itself.  A rounding's variance is
    at most a quarter of its spacing squared, so the mean of 400 lies within 6 / sqrt(400) / 2 = 0.15 spacings of it."""
    torch, nuq = require_cuda()
    t, lst, _ = _list(torch, nuq, [2048], bits=8, seed=21)
    start = {k: x.view.clone() for k, x in t[0].items()}
    m0, v0 = R.held(start["m"].cpu().numpy(), start["scales"].cpu().numpy()[0::2]), R.held(start["v"].cpu().numpy(), start["scales"].cpu().numpy()[1::2]) ** 2
    m, v, _, _ = R.moments(start["g"].cpu().numpy(), m0, v0)
    sums = np.zeros((2, 2048))
    for seed in range(400):
        for k, x in t[0].items():
            x.view.copy_(start[k])
        nuq.adamw(lst, lr=R.LR, step=9, seed=seed * 0x9E3779B97F4A7C15 & (2 ** 64 - 1))
        b = _read(t)[0]
        sums += [R.held(b["m"], b["scales"][0::2]), R.held(b["v"], b["scales"][1::2])]
    for x, mean in zip((m, np.sqrt(v)), sums / 400):
        unit = (R.largest(x) / 448.0)[np.arange(2048) // 256]
        spacing = np.maximum(2.0 ** (np.frexp(np.abs(x) / unit)[1] - 4.0), 2.0 ** -9) * unit
        tiny = np.abs(x) < 2.0 ** -9 * unit                  # (a root that would be rounded to 0 is not)
        assert (np.abs(mean - x)[~tiny] <= 0.16 * spacing[~tiny]).all()


def test_8_bit_states_decay_and_never_forget_a_root():
    """Without gradients v falls by 0.1 % a step, far less than half a code's spacing: its mean follows all the same.  No root becomes 0."""
    torch, nuq = require_cuda()
    n = 1 << 14
    g, w = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.full((n,), 0x70, dtype=torch.uint8, device="cuda")
    v[::256] = 0x7E
    v[1::256] = 1
    scales = torch.full((n // 128,), 1.0 / 448.0, device="cuda")
    lst = nuq.tensors([g], [w], [m], [v], scales=[scales])
    before = R.held(v.cpu().numpy(), scales.cpu().numpy()[1::2])
    steps = 200
    for t in range(steps):
        nuq.adamw(lst, lr=R.LR, step=1000 + t, seed=5)
    after = R.held(v.cpu().numpy(), scales.cpu().numpy()[1::2])
    assert (after > 0).all()
    body = np.arange(n) % 256 >= 2
    # each step's rounding adds less than a spacing (1/8) squared over four in variance, relative to the root: sqrt(200) / 16 a lane
    want = before[body] * 0.999 ** (steps / 2)
    assert abs(after[body].mean() / want.mean() - 1) <= 6 * np.sqrt(steps) / 16 / np.sqrt(body.sum()) + 1e-3


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("grad", GRADS)
def test_gradients_that_are_not_finite_reach_their_elements_only(bits, bad, grad):
    torch, nuq = require_cuda()
    t, lst, decays = _list(torch, nuq, [1000], grad, None, bits, seed=31)
    t[0]["g"].view[300] = bad
    before = _read(t)
    nuq.adamw(lst, lr=R.LR, step=3, seed=4)
    after = _read(t)
    other = np.arange(1000) != 300
    assert np.isnan(after[0]["w"][300])                      # inf / inf, or NaN itself
    if bits == 32:
        assert not np.isfinite(after[0]["m"][300]) and not np.isfinite(after[0]["v"][300])
    else:
        assert after[0]["m"][300] & 127 == 127 and after[0]["v"][300] & 127 == 127
        assert np.isfinite(after[0]["scales"]).all()
    # everybody else's step is what it is without that element
    clean = [{k: x.copy() for k, x in before[0].items()}]
    clean[0]["g"][300] = 0.0
    clean[0]["m"][300] = clean[0]["v"][300] = 0
    for x in t[0].values():
        x.view
    for k, x in t[0].items():
        x.view.copy_(torch.from_numpy(clean[0][k]).to(x.view.dtype))
    nuq.adamw(lst, lr=R.LR, step=3, seed=4)
    for k, x in _read(t)[0].items():
        if k == "scales":
            assert np.array_equal(x, after[0][k])
        elif k != "g":
            assert np.array_equal(x[other], after[0][k][other]), k
    # and a state that is NaN stays so, with the others still as they were
    if bits == 8:
        t[0]["m"].view[5] = 0xFF
        before = _read(t)
        nuq.adamw(lst, lr=R.LR, step=4, seed=4)
        after = _read(t)
        assert after[0]["m"][5] & 127 == 127 and np.isnan(after[0]["w"][5]) and not np.isnan(np.delete(after[0]["w"], 5)).any()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("magnitude", [1e-30, 1e-15, 1e15])
def test_magnitudes(bits, magnitude):
    torch, nuq = require_cuda()
    t, lst, decays = _list(torch, nuq, [777, 256], bits=bits, seed=41, magnitude=magnitude)
    before = _read(t)
    nuq.adamw(lst, lr=R.LR, step=3, seed=4)
    after = _read(t)
    if magnitude == 1e-30 and bits == 8:                     # (v underflows, the root with it: nothing but finite numbers is asked)
        assert all(np.isfinite(x["w"]).all() and np.isfinite(x["scales"]).all() for x in after)
        return
    _check(before, after, decays, 3, bits, seed=4)


# ---- the norm ----

def _norm(torch, nuq, grads, max_norm=float("inf"), scale=1.0, step=0):
    control = nuq.step_control(step)
    nuq.grad_norm(nuq.tensors(grads), control, max_norm=max_norm, scale=scale)
    return {k: v.item() for k, v in nuq.control_fields(control).items()}


@pytest.mark.parametrize("grad", GRADS)
@pytest.mark.parametrize("skew", [0, 1, 3, 5])
@pytest.mark.parametrize("sizes", [[1], [0], [0, 5, 0], SIZES, [8191], [8192], [8193], [3_000_001], [70_000, 1, 8192 * 3]])
def test_norm(grad, skew, sizes):
    torch, nuq = require_cuda()
    rng = np.random.default_rng(sum(sizes) + skew)
    t = [Guarded(torch, torch.from_numpy(rng.standard_normal(n).astype(np.float32)).to(getattr(torch, grad)), skew) for n in sizes]
    want = np.sqrt(sum(float((x.read().double() ** 2).sum()) for x in t))
    got = _norm(torch, nuq, [x.view for x in t], max_norm=0.5, scale=-2.0, step=41)
    # eights in fp32 (seven roundings of a sum that grows: 7 U of the square, 4 U of the root at most), the root rounded
    assert abs(got["norm"] - 2.0 * want) <= 5 * R.U * 2.0 * want
    assert got["skip"] == 0 and got["step"] == 42 and got["lr_factor"] == 1.0
    factor = min(1.0, 0.5 / (2.0 * want)) if want else 1.0
    assert abs(got["scale"] + 2.0 * factor) <= 8 * R.U * 2.0 * factor


@pytest.mark.parametrize("value", [1e-45, 1e-38, 1e-30, 1e-20, 1e18, 1e25, 3e38])
def test_norm_of_extreme_values(value):
    torch, nuq = require_cuda()
    x = torch.full((1000,), value, device="cuda")
    x[::3] = 0.0
    want = np.sqrt(float((x.double() ** 2).sum()))
    got = _norm(torch, nuq, [x, torch.zeros(100, device="cuda")])
    if want > 3.4028234e38:
        assert got["skip"] == 1 and got["step"] == 0
    else:
        assert got["skip"] == 0 and abs(got["norm"] - want) <= 5 * R.U * want + 1e-45


@pytest.mark.parametrize("grad", GRADS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("at", [0, 12345, 29_999])
def test_norm_finds_what_is_not_finite(grad, bad, at):
    torch, nuq = require_cuda()
    x = torch.ones(30_000, device="cuda", dtype=getattr(torch, grad))
    x[at] = bad
    got = _norm(torch, nuq, [torch.ones(5, device="cuda"), x], max_norm=1.0, step=3)
    assert got["skip"] == 1 and got["step"] == 3
    got = _norm(torch, nuq, [torch.ones(5, device="cuda"), torch.ones(30_000, device="cuda")], max_norm=1.0, step=3)
    assert got["skip"] == 0 and got["step"] == 4


def test_norm_of_thousands_of_tensors_repeats_bit_for_bit():
    torch, nuq = require_cuda()
    rng = np.random.default_rng(3)
    sizes = [1 + (i * 131) % 3000 for i in range(3500)]      # three launches
    x = torch.from_numpy(rng.standard_normal(sum(sizes)).astype(np.float32)).cuda()
    grads = list(torch.split(x, sizes))
    want = np.sqrt(float((x.double() ** 2).sum()))
    control = nuq.step_control(0)
    lst = nuq.tensors(grads)
    seen = set()
    for _ in range(5):
        nuq.grad_norm(lst, control)
        seen.add(nuq.control_fields(control)["norm"].item())
    assert len(seen) == 1 and abs(seen.pop() - want) <= 5 * R.U * want
    assert control[0].item() == 5


def test_no_tensors():
    torch, nuq = require_cuda()
    control = nuq.step_control(6)
    nuq.grad_norm(nuq.tensors([]), control, max_norm=1.0, scale=0.25)
    f = nuq.control_fields(control)
    assert (f["step"].item(), f["norm"].item(), f["scale"].item(), f["skip"].item()) == (7, 0.0, 0.25, 0)
    nuq.adamw(nuq.tensors([], []), lr=1.0, step=1)


# ---- together ----

@pytest.mark.parametrize("bits", [32, 8])
def test_clipped_steps_follow_the_record(bits):
    """norm and step in turn: clipped, not clipped, skipped, with a schedule"""
    torch, nuq = require_cuda()
    t, lst, decays = _list(torch, nuq, [3000, 129], "float32", "bfloat16", bits, zero=True, seed=51)
    control = nuq.step_control(0)
    f = nuq.control_fields(control)
    rng = np.random.default_rng(5)
    taken = 0
    for k, (size, factor, bad) in enumerate([(1.0, 1.0, False), (1e-3, 0.5, False), (1.0, 0.25, True), (2.0, 0.125, False)]):
        for x in t:
            x["g"].view.copy_(torch.from_numpy((size * rng.standard_normal(x["g"].n)).astype(np.float32)))
        if bad:
            t[1]["g"].view[100] = float("inf")
        f["lr_factor"].fill_(factor)
        before = _read(t)
        nuq.grad_norm(lst, control, max_norm=1.0, scale=0.5)
        nuq.adamw(lst, lr=0.01, control=control, seed=9)
        after = _read(t)
        if bad:
            assert f["skip"].item() == 1
            for a, b in zip(before, after):
                assert all(np.array_equal(a[n], b[n], equal_nan=True) for n in a)
            continue
        taken += 1
        norm = 0.5 * np.sqrt(sum((x["g"].astype(np.float64) ** 2).sum() for x in before))
        scale = f["scale"].item()
        assert f["step"].item() == taken and abs(scale - 0.5 * min(1.0, 1.0 / norm)) <= 8 * R.U
        _check(before, after, decays, taken, bits, scale, "bfloat16", 9, lr=0.01 * factor)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_goes_on_counting(bits):
    """norm and step in one graph, replayed on changing gradients and learning rates: what the same calls give outside it"""
    torch, nuq = require_cuda()
    make = lambda: _list(torch, nuq, [3000, 129, 0, 5001], "bfloat16", "bfloat16", bits, zero=True, seed=61)  # noqa: E731
    (a, la, _), (b, lb, _) = make(), make()
    ca, cb = nuq.step_control(0), nuq.step_control(0)

    def call(lst, control):
        nuq.grad_norm(lst, control, max_norm=1.0)
        nuq.adamw(lst, lr=0.01, control=control, seed=9)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call(la, ca)
    torch.cuda.current_stream().wait_stream(side)
    rng = np.random.default_rng(5)
    for k in range(4):
        for x, y in zip(a, b):
            new = torch.from_numpy((10.0 ** (k - 2) * rng.standard_normal(x["g"].n)).astype(np.float32))
            if k == 2 and x["g"].n == 129:
                new[7] = float("nan")
            x["g"].view.copy_(new)
            y["g"].view.copy_(new)
        for c in (ca, cb):
            nuq.control_fields(c)["lr_factor"].fill_(1.0 / (k + 1))
        graph.replay()
        call(lb, cb)
        torch.cuda.synchronize()
        assert torch.equal(ca[:3], cb[:3])
        for x, y in zip(_read(a), _read(b)):
            assert all(np.array_equal(x[n], y[n], equal_nan=True) for n in x)
    assert ca[0].item() == 3


def test_steps_on_several_streams_at_once():
    torch, nuq = require_cuda()
    lists = [_list(torch, nuq, [400_000, 77], bits=bits, seed=70 + i) for i, bits in enumerate((32, 8, 32, 8))]
    before = [_read(t) for t, _, _ in lists]
    controls = [nuq.step_control(4) for _ in lists]
    streams = [torch.cuda.Stream() for _ in lists]
    torch.cuda.synchronize()
    for (_, lst, _), control, stream in zip(lists, controls, streams):
        nuq.grad_norm(lst, control, max_norm=1.0, stream=stream)
        nuq.adamw(lst, lr=R.LR, control=control, seed=1, stream=stream)
    torch.cuda.synchronize()
    for (t, _, decays), a, control, bits in zip(lists, before, controls, (32, 8, 32, 8)):
        f = nuq.control_fields(control)
        want = np.sqrt(sum((x["g"].astype(np.float64) ** 2).sum() for x in a))
        assert abs(f["norm"].item() - want) <= 5 * R.U * want
        _check(a, _read(t), decays, 5, bits, f["scale"].item(), seed=1)


def test_a_step_without_a_begun_one_changes_nothing():
    torch, nuq = require_cuda()
    t, lst, _ = _list(torch, nuq, [1000], seed=81)
    before = _read(t)
    nuq.adamw(lst, lr=1.0, control=nuq.step_control(0))
    for a, b in zip(before, _read(t)):
        assert all(np.array_equal(a[n], b[n]) for n in a)


def test_encoded_decoded_clipped_and_applied():
    """the path of a step: K gradients encoded, decoded and summed, the norm of the sum's parts, AdamW on parts that start anywhere"""
    torch, nuq = require_cuda()
    sizes = [10_001, 64, 300, 77_777, 1]
    d, K, bucket, s = sum(sizes), 4, 8192, 4
    gen = torch.Generator(device="cuda").manual_seed(1)
    streams = [nuq.encode(torch.randn(d, generator=gen, device="cuda"), bucket, s, seed=k)[0] for k in range(K)]
    total = nuq.decode_accumulate(streams, d, bucket, s)
    assert nuq.last_status() == 0
    parts = list(torch.split(total, sizes))
    w = list(torch.split(torch.randn(d, generator=gen, device="cuda"), sizes))
    m, v = [torch.zeros(n, device="cuda") for n in sizes], [torch.zeros(n, device="cuda") for n in sizes]
    lst = nuq.tensors(parts, w, m, v, weight_decay=0.01)
    control = nuq.step_control(0)
    before = [{"g": g.cpu().numpy(), "w": x.cpu().numpy(), "m": np.zeros(n, np.float32), "v": np.zeros(n, np.float32)} for g, x, n in zip(parts, w, sizes)]
    nuq.grad_norm(lst, control, max_norm=1.0, scale=1.0 / K)
    nuq.adamw(lst, lr=R.LR, control=control)
    f = nuq.control_fields(control)
    want = np.sqrt(float((total.double() ** 2).sum())) / K
    assert abs(f["norm"].item() - want) <= 5 * R.U * want
    after = [{"g": g.cpu().numpy(), "w": x.cpu().numpy(), "m": y.cpu().numpy(), "v": z.cpu().numpy()} for g, x, y, z in zip(parts, w, m, v)]
    _check(before, after, [0.01] * len(sizes), 1, 32, f["scale"].item())


def test_a_training_loop_with_8_bit_states():
    """sums of encoded gradients of a quadratic, clipped, states in 8 bits, weights of several shapes: as the README has it"""
    torch, nuq = require_cuda()
    shapes, K, bucket, s = [(64, 33), (33,), (7, 5, 3), (1,)], 2, 256, 4
    sizes = [int(np.prod(x)) for x in shapes]
    d = sum(sizes)
    gen = torch.Generator(device="cuda").manual_seed(3)
    weights = [torch.randn(x, generator=gen, device="cuda") for x in shapes]
    copies = [w.to(torch.bfloat16) for w in weights]
    states = [[torch.zeros(n, dtype=torch.uint8, device="cuda") for n in sizes] for _ in range(2)]
    scales = [torch.zeros(2 * -(-n // nuq.STATE_BLOCK), device="cuda") for n in sizes]
    total = torch.zeros(d, device="cuda")
    parts = list(torch.split(total, sizes))
    tensors = nuq.tensors(parts, weights, *states, scales=scales, copy=copies, weight_decay=[0.05 if w.dim() > 1 else 0.0 for w in weights])
    control = nuq.step_control()
    for step in range(1, 6):
        flat = torch.cat([w.reshape(-1) for w in weights])
        containers = [nuq.encode(flat + 0.1 * torch.randn(d, generator=gen, device="cuda"), bucket, s, seed=k, offset=step)[0] for k in range(K)]
        nuq.decode_accumulate(containers, d, bucket, s, acc=total)
        before = [{"g": g.cpu().numpy(), "w": w.reshape(-1).cpu().numpy(), "m": m.cpu().numpy(), "v": v.cpu().numpy(), "scales": c.cpu().numpy()}
                  for g, w, m, v, c in zip(parts, weights, *states, scales)]
        nuq.grad_norm(tensors, control, max_norm=1.0, scale=1.0 / K)
        nuq.adamw(tensors, lr=R.LR, seed=7, control=control)
        assert nuq.last_status() == 0
        f = {k: x.item() for k, x in nuq.control_fields(control).items()}
        want = np.sqrt(sum((x["g"].astype(np.float64) ** 2).sum() for x in before)) / K
        assert f["step"] == step and abs(f["norm"] - want) <= 5 * R.U * want
        after = [{"g": g.cpu().numpy(), "w": w.reshape(-1).cpu().numpy(), "copy": c16.float().reshape(-1).cpu().numpy(), "m": m.cpu().numpy(), "v": v.cpu().numpy(), "scales": c.cpu().numpy()}
                 for g, w, c16, m, v, c in zip(parts, weights, copies, *states, scales)]
        _check(before, after, [0.05, 0.0, 0.05, 0.0], step, 8, f["scale"], "bfloat16", 7)


@pytest.mark.parametrize("bits", [32, 8])
def test_offsets_beyond_32_bits(bits):
    """a tensor of more than 2^32 elements: the elements on both sides of 2^32 and the last ones, and the norm of all"""
    torch, nuq = require_cuda()
    n = (1 << 32) + 4099
    need = n * (14 if bits == 32 else 8) + (4 << 30)
    if torch.cuda.mem_get_info()[0] < need:
        pytest.skip("not enough memory free")
    rng = np.random.default_rng(3)
    g, w = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, device="cuda")
    dtype = torch.float32 if bits == 32 else torch.uint8
    m, v = torch.zeros(n, dtype=dtype, device="cuda"), torch.zeros(n, dtype=dtype, device="cuda")
    blocks = -(-n // R.BLOCK)
    scales = torch.full((2 * blocks,), 1.0 / 448.0, device="cuda") if bits == 8 else None
    # whole blocks each: the random bits go by an element's place, so the reference gets the places in front as if they were there
    parts = [slice(0, 512), slice((1 << 31) - 512, (1 << 31) + 512), slice((1 << 32) - 512, (1 << 32) + 1024), slice((1 << 32) + 3840, n)]
    for p in parts:
        k = p.stop - p.start
        g[p] = torch.from_numpy(rng.standard_normal(k).astype(np.float32)).cuda().to(torch.bfloat16)
        w[p] = torch.from_numpy(rng.standard_normal(k).astype(np.float32)).cuda()
        for x in (m, v):
            x[p] = torch.from_numpy((rng.random(k) if bits == 32 else rng.integers(1, 126, k)).astype(np.float32)).cuda().to(dtype)
    read = lambda: [{**{name: x[p].float().cpu().numpy() if x.dtype != torch.uint8 else x[p].cpu().numpy() for name, x in (("g", g), ("w", w), ("m", m), ("v", v))},  # noqa: E731
                     **({"scales": scales[2 * (p.start // 256):2 * -(-p.stop // 256)].cpu().numpy()} if bits == 8 else {})} for p in parts]
    before = read()
    lst = nuq.tensors([g], [w], [m], [v], scales=[scales] if bits == 8 else None, weight_decay=0.1)
    control = nuq.step_control(2)
    nuq.grad_norm(lst, control, scale=1.0)
    want = np.sqrt(sum((x["g"].astype(np.float64) ** 2).sum() for x in before))
    assert abs(nuq.control_fields(control)["norm"].item() - want) <= 5 * R.U * want
    nuq.adamw(lst, lr=R.LR, control=control, seed=77)
    for p, a, b in zip(parts, before, read()):
        _check([a], [b], [0.1], 3, bits, seed=77, first=p.start)


def test_lists_refuse_what_does_not_fit():
    torch, nuq = require_cuda()
    z = lambda n, dtype=torch.float32: torch.zeros(n, dtype=dtype, device="cuda")  # noqa: E731
    g, w, m, v = z(300), z(300), z(300), z(300)
    codes, scales = z(300, torch.uint8), z(4)
    nuq.tensors([g], [w], [m], [v])
    nuq.tensors([g], [w], [codes], [z(300, torch.uint8)], scales=[scales])
    for bad in (lambda: nuq.tensors([g.cpu()]), lambda: nuq.tensors([z(300, torch.float64)]), lambda: nuq.tensors([z((300, 2))[:, 0]]),
                lambda: nuq.tensors([g], [z(299)], [m], [v]), lambda: nuq.tensors([g], [w], [m], [z(300, torch.uint8)]),
                lambda: nuq.tensors([g], [w], [codes], [z(300, torch.uint8)]), lambda: nuq.tensors([g], [w], [codes], [z(300, torch.uint8)], scales=[z(3)]),
                lambda: nuq.tensors([g], [w], [codes], [z(300, torch.uint8)], scales=[z(5)[1:]]),
                lambda: nuq.tensors([g], [w.half()], [m], [v]), lambda: nuq.tensors([g], [w], [m], [m]), lambda: nuq.tensors([w], [w], [m], [v]),
                lambda: nuq.tensors([g, g], [w, w], [m, z(300)], [v, z(300)]), lambda: nuq.tensors([g], [w], [m], [v], copy=[z(300)]),
                lambda: nuq.tensors([g], [w], [m], [v], weight_decay=[0.1, 0.2]), lambda: nuq.tensors([g], [w, w], [m], [v]),
                lambda: nuq.tensors([z(600)[:300]], [w], [z(600)[299:599]], [z(600)[:300]], copy=[z(299, torch.bfloat16)]),
                lambda: nuq.tensors([g], m=[m]), lambda: nuq.adamw(nuq.tensors([g]), lr=1.0, step=1),
                lambda: nuq.grad_norm(nuq.tensors([g]), z(2048, torch.int32)), lambda: nuq.grad_norm(nuq.tensors([g]), z(100, torch.int64))):
        with pytest.raises((ValueError, AttributeError)):
            bad()
    lst, control = nuq.tensors([g], [w], [m], [v]), nuq.step_control()
    nan, inf = float("nan"), float("inf")
    for kw in (dict(lr=nan), dict(lr=-1.0), dict(lr=inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan), dict(eps=-1e-8), dict(eps=nan),
               dict(scale=nan), dict(scale=inf), dict(step=0), dict(step=-1), dict(step=1 << 64)):
        with pytest.raises((nuq.NuqError, ValueError)):
            nuq.adamw(lst, **{"lr": 0.1, "step": 1, **kw})
    for kw in (dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=nan), dict(scale=inf), dict(scale=nan)):
        with pytest.raises(nuq.NuqError):
            nuq.grad_norm(lst, control, **kw)
    assert not w.any().item() and control[0].item() == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_a_record_whose_step_no_norm_has_begun_changes_nothing(bits):
    """a record with a number of steps and no scale, as step_control makes it, is not a step's: gradients were multiplied by 0"""
    torch, nuq = require_cuda()
    t, lst, decays = _list(torch, nuq, [1000, 257], bits=bits, seed=82)
    control = nuq.step_control(999)
    f = nuq.control_fields(control)
    before = _read(t)
    nuq.adamw(lst, lr=1.0, control=control, seed=3)
    for a, b in zip(before, _read(t)):
        assert all(np.array_equal(a[n], b[n]) for n in a)
    nuq.grad_norm(lst, control)
    nuq.adamw(lst, lr=R.LR, control=control, seed=3)
    assert f["step"].item() == 1000
    after = _read(t)
    _check(before, after, decays, 1000, bits, seed=3)
    # a scale of 0 that grad_norm has written is one: the moments decay
    nuq.grad_norm(lst, control, scale=0.0)
    nuq.adamw(lst, lr=R.LR, control=control, seed=4)
    assert f["step"].item() == 1001 and f["scale"].item() == 0.0 and f["skip"].item() == 0
    _check(after, _read(t), decays, 1001, bits, 0.0, seed=4)


def test_a_record_with_a_scale_of_the_caller_s_own():
    torch, nuq = require_cuda()
    t, lst, decays = _list(torch, nuq, [1000], seed=83)
    control = nuq.step_control(6)
    nuq.control_fields(control)["scale"].fill_(0.25)
    before = _read(t)
    nuq.adamw(lst, lr=R.LR, control=control)
    _check(before, _read(t), decays, 6, 32, 0.25)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("factor", [-1.0, -1e-30, float("nan"), float("inf"), 2.0 ** 50])
def test_a_learning_rate_s_factor_out_of_range_changes_nothing(bits, factor):
    """a negative one would take the decay with the wrong sign, the others leave NaN or infinity in every parameter"""
    torch, nuq = require_cuda()
    t, lst, _ = _list(torch, nuq, [1000, 257], bits=bits, seed=84)
    control = nuq.step_control(4)
    before = _read(t)
    nuq.grad_norm(lst, control)
    nuq.control_fields(control)["lr_factor"].fill_(factor)
    nuq.adamw(lst, lr=R.LR, control=control, seed=3)
    for a, b in zip(before, _read(t)):
        assert all(np.array_equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("bits", [32, 8])
def test_the_largest_decays(bits):
    """lr_factor = 0 moves no parameter, whatever the decay; a product of factor and decay that leaves fp32 leaves zeros zero"""
    torch, nuq = require_cuda()
    t, lst, decays = _list(torch, nuq, [1000, 257], bits=bits, seed=85, decays=[3e38, 1e30])
    control = nuq.step_control(4)
    f = nuq.control_fields(control)
    f["lr_factor"].fill_(0.0)
    before = _read(t)
    nuq.grad_norm(lst, control)
    nuq.adamw(lst, lr=1.0, control=control, seed=3)
    after = _read(t)
    _check(before, after, decays, 5, bits, seed=3, lr=0.0)
    assert all(np.array_equal(a["w"], b["w"]) for a, b in zip(before, after))
    for x in t:
        x["w"].view.zero_()
    f["lr_factor"].fill_(2.0)
    before = _read(t)
    nuq.grad_norm(lst, control)
    nuq.adamw(lst, lr=1.0, control=control, seed=3)
    _check(before, _read(t), [0.0, 0.0], 6, bits, seed=3, lr=2.0)


@pytest.mark.parametrize("which", ["w", "copy", "part of w"])
def test_a_backward_pass_through_parameters_from_before_the_step_is_an_error(which):
    """the step writes parameters through their addresses; autograd has to hear of it, or it takes the new ones for those it has saved"""
    torch, nuq = require_cuda()
    whole = torch.randn(600, device="cuda")
    if which == "part of w":
        whole.requires_grad_()
        parts = list(torch.split(whole, [300, 300]))
        w = [x.detach() for x in parts]
    else:
        w = [torch.randn(300, device="cuda", requires_grad=which == "w") for _ in range(2)]
    copies = [x.detach().to(torch.bfloat16).requires_grad_(which == "copy") for x in w]
    zeros = lambda: [torch.zeros(300, device="cuda") for _ in range(2)]  # noqa: E731
    lst = nuq.tensors(zeros(), w, zeros(), zeros(), copy=copies)
    loss = whole.square().sum() if which == "part of w" else sum(x.float().square().sum() if which == "w" else (x * x).sum() for x in (w if which == "w" else copies))
    nuq.adamw(lst, lr=R.LR, step=1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    # and one from after it is as ever
    x = whole if which == "part of w" else (w if which == "w" else copies)[0]
    x.square().sum().backward()
    assert torch.equal(x.grad, 2 * x.detach())


def test_parameters_made_in_inference_mode():
    torch, nuq = require_cuda()
    with torch.inference_mode():
        g, w, m, v = (torch.ones(300, device="cuda") for _ in range(4))
    nuq.adamw(nuq.tensors([g], [w], [m], [v]), lr=0.5, step=1)
    assert float(w.max()) < 1.0


@pytest.mark.parametrize("skew", [0, 1])
@pytest.mark.parametrize("total,count", [(9_000_001, 4), (20_000_003, 7), (70_000_001, 23)])
def test_long_lists_of_8_bit_states_are_stepped_like_their_tensors(total, count, skew):
    """A warp of a long call takes several blocks one after the other (2, 4 and 16 here, where an SM has seven CTAs).  Each tensor
    in a call of its own, with as many empty ones in front (the random bits go by the place in the list), is short enough for
    one block to a warp: equal bits are wanted."""
    torch, nuq = require_cuda()
    rng = np.random.default_rng(total)
    share = rng.uniform(0.2, 1.0, count)
    sizes = [int((total - 3000) * x / share.sum()) for x in share]
    sizes[count // 2] = 1531                                 # a short one between the others
    assert max(sizes) < 2 * torch.cuda.get_device_properties(0).multi_processor_count * 7 * 4 * 1024
    starts, end = [], skew
    for n in sizes:
        starts.append(end)
        end = end + n + 3 if skew else (end + n + 63) // 64 * 64 + 64
    blocks = [-(-n // R.BLOCK) for n in sizes]
    gen = torch.Generator(device="cuda").manual_seed(count)
    g = torch.randn(end, generator=gen, device="cuda").to(torch.bfloat16)
    first = {"w": torch.randn(end, generator=gen, device="cuda"), "copy": torch.zeros(end, dtype=torch.bfloat16, device="cuda"),
             "m": torch.randint(0, 127, (end,), generator=gen, device="cuda").to(torch.uint8), "v": torch.randint(0, 127, (end,), generator=gen, device="cuda").to(torch.uint8),
             "scales": torch.rand(2 * sum(blocks), generator=gen, device="cuda") / 448.0 + 1e-4}
    one, each = ({k: x.clone() for k, x in first.items()} for _ in range(2))

    def lists(x):
        cut = lambda y: [y[a:a + n] for a, n in zip(starts, sizes)]  # noqa: E731
        at = [2 * sum(blocks[:i]) for i in range(count)]
        return cut(g), cut(x["w"]), cut(x["m"]), cut(x["v"]), [x["scales"][a:a + 2 * b] for a, b in zip(at, blocks)], cut(x["copy"])

    def list_of(x, keep):
        return nuq.tensors(*[[y[:0] if not keep(i) else y for i, y in enumerate(col)] for col in lists(x)[:4]],
                           scales=[y[:0] if not keep(i) else y for i, y in enumerate(lists(x)[4])],
                           copy=[y[:0] if not keep(i) else y for i, y in enumerate(lists(x)[5])], weight_decay=[0.1 * (i % 3) for i in range(count)])

    nuq.adamw(list_of(one, lambda i: True), lr=R.LR, step=3, seed=5)
    for j in range(count):
        nuq.adamw(list_of(each, lambda i: i == j), lr=R.LR, step=3, seed=5)
    for k in first:
        assert not torch.equal(one[k], first[k]), k
        assert torch.equal(one[k].view(torch.int32) if k in ("w", "scales") else one[k].view(torch.int16) if k == "copy" else one[k],
                           each[k].view(torch.int32) if k in ("w", "scales") else each[k].view(torch.int16) if k == "copy" else each[k]), k
    # the gaps are as they were, and two of the tensors are what the formula gives
    inside = torch.zeros(end, dtype=torch.bool, device="cuda")
    for a, n in zip(starts, sizes):
        inside[a:a + n] = True
    for k in ("w", "copy", "m", "v"):
        assert torch.equal(one[k][~inside], first[k][~inside]), k
    row = lambda x, i: {k: _numpy(y[i].cpu()) for k, y in zip(("g", "w", "m", "v", "scales", "copy"), lists(x))}  # noqa: E731
    for i in (count // 2, int(np.argmin([n if n != 1531 else total for n in sizes]))):
        nothing = [{k: np.zeros(0, y.dtype) for k, y in row(first, i).items()}] * i
        _check(nothing + [row(first, i)], nothing + [row(one, i)], [0.1 * (j % 3) for j in range(i + 1)], 3, 8, copy="bfloat16", seed=5)


def test_a_long_run_of_8_bit_states_with_gradients():
    """8000 steps on normal gradients of constant size 1, beta2 = 0.999, beside the rounding rule in 64 bits with random numbers of
    its own: both wander alike.  Where the states have settled, E v = 1 + E var / (1 - beta2), and a rounding's variance is at most
    its spacing (an eighth of the root) times how far the root has moved against its block's scale in a step, on average no
    more than 3/2 (1 - beta2) of it: v is at most 3/16 of itself too high.  Blocks are independent of each other, so a mean is
    off by the spread of the blocks' means / sqrt(blocks); six times that is allowed for."""
    torch, nuq = require_cuda()
    blocks, steps = 256, 8000
    n = blocks * R.BLOCK
    gen = torch.Generator(device="cuda").manual_seed(12)
    g, w = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(2 * blocks, device="cuda")
    lst = nuq.tensors([g], [w], [m], [v], scales=[scales])
    root, mean = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    for t in range(1, steps + 1):
        g.normal_(generator=gen)
        nuq.adamw(lst, lr=R.LR, step=t, seed=5)
        x = (R.BETA2 * root * root + (1.0 - R.BETA2) * g.double() ** 2).sqrt()
        unit = (x.view(blocks, -1).amax(1) / 448.0).repeat_interleave(R.BLOCK)
        spacing = torch.exp2(torch.floor(torch.log2((x / unit).clamp(min=2.0 ** -6))) - 3.0)
        root = torch.floor(x / unit / spacing + torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)) * spacing * unit
        y = R.BETA1 * mean + (1.0 - R.BETA1) * g.double()
        unit = (y.abs().view(blocks, -1).amax(1) / 448.0).repeat_interleave(R.BLOCK)
        spacing = torch.exp2(torch.floor(torch.log2((y.abs() / unit).clamp(min=2.0 ** -6))) - 3.0)
        mean = torch.floor(y / unit / spacing + torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)) * spacing * unit
    got = {"root": torch.from_numpy(R.held(v.cpu().numpy(), scales.cpu().numpy()[1::2])), "m": torch.from_numpy(R.held(m.cpu().numpy(), scales.cpu().numpy()[0::2]))}
    want = {"root": root.cpu(), "m": mean.cpu()}
    for name, power in (("root", 1), ("root", 2), ("m", 1), ("m", 2)):
        a, b = ((x[name] ** power).view(blocks, -1).mean(1) for x in (got, want))
        off = 6.0 * float(((a.var() + b.var()) / blocks).sqrt())
        print(f"{name}^{power}: {float(a.mean()):.4f}, rule {float(b.mean()):.4f}, allowed {off:.4f}")
        assert abs(float(a.mean() - b.mean())) <= off, (name, power)
    a = (got["root"] ** 2).view(blocks, -1).mean(1)
    off = 6.0 * float((a.var() / blocks).sqrt())
    assert 1.0 - off <= float(a.mean()) <= 1.0 / (1.0 - 3.0 / 16.0) + off
    print(f"sd of the root {float(got['root'].std()):.4f}, mean of v {float(a.mean()):.4f}")


@pytest.mark.parametrize("bits,skew", [(32, 0), (8, 0), (8, 1)])
@pytest.mark.parametrize("count", [16, 17, 64, 65, 256, 257, 400])
def test_tables_of_every_size(count, bits, skew):
    """lists at the ends of the tables in which they travel"""
    torch, nuq = require_cuda()
    t, lst, decays = _list(torch, nuq, [1 + (53 * i) % 300 for i in range(count)], bits=bits, skew=skew, seed=count)
    before = _read(t)
    nuq.adamw(lst, lr=R.LR, step=5, seed=3)
    _check(before, _read(t), decays, 5, bits, seed=3)


def test_a_record_kept_from_before_it_was_marked_as_begun():
    """the norm's scratch has its old places: words 24 to 31 its carried sum, 32 the count of CTAs, 36 zero"""
    torch, nuq = require_cuda()
    t, lst, decays = _list(torch, nuq, [1000, 70_000], seed=86)
    control = nuq.step_control(6)
    control.view(torch.float64)[3] = 123.456
    nuq.control_fields(control)["scale"].fill_(0.25)
    before = _read(t)
    nuq.adamw(lst, lr=R.LR, control=control)
    after = _read(t)
    _check(before, after, decays, 6, 32, 0.25)
    nuq.grad_norm(lst, control)
    nuq.adamw(lst, lr=R.LR, control=control)
    assert control[0].item() == 7
    _check(after, _read(t), decays, 7, 32)


def test_autograd_hears_of_every_buffer_that_parameters_are_parts_of():
    torch, nuq = require_cuda()
    bases = [torch.zeros(40, device="cuda") for _ in range(20)]
    w = [x[i:i + 10] for x in bases for i in (0, 10, 25)]
    make = lambda dtype=torch.float32: [torch.zeros(10, dtype=dtype, device="cuda") for _ in w]  # noqa: E731
    copies = make(torch.bfloat16)
    lst = nuq.tensors(make(), w, make(), make(), copy=[x if i % 2 else None for i, x in enumerate(copies)])
    versions = [x._version for x in (*bases, *w, *copies)]
    nuq.adamw(lst, lr=R.LR, step=1)
    assert all(x._version > a for x, a in zip((*bases, *w), versions))
    assert [x._version > a for x, a in zip(copies, versions[80:])] == [i % 2 == 1 for i in range(60)]
