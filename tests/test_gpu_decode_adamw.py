"""AdamW applied where the decoder finishes a sum (nuq_decode_adamw): the sums are the oracle's, the step is the formula's in 64 bits."""
import numpy as np
import pytest

import adamw_reference as R
import oracle as O
from gpu_util import require_cuda

pytestmark = pytest.mark.gpu

GUARD = 64
LIKELY = {O.MODE_ERC: 0, O.MODE_FIXED: 1 << 16, O.MODE_CODED: 2 << 16}


def _gradient(d, seed):
    rng = np.random.default_rng(seed)
    g = rng.standard_normal(d) * 10.0 ** rng.uniform(-3, 0, d)
    g[rng.random(d) < 0.02] = 0.0
    return g.astype(np.float32)


def _streams(torch, nuq, d, bucket, s, flags, K, seed=0):
    """K containers as the library writes them, and as the oracle reads them"""
    if (flags >> 8) & 0xFF == 2:
        nuq.set_level_table([0.6 ** (s + 1 - j) for j in range(1, s + 1)])
    if (flags >> 16) & 0xFF == 2:
        nuq.set_level_code([min(j + 1, s) for j in range(s + 1)])
    outs, hosts = [], []
    for k in range(K):
        out, bits = nuq.encode(torch.from_numpy(_gradient(d, 1000 * seed + k)).cuda(), bucket, s, flags, seed=k + 1)
        outs.append(out)
        hosts.append(out.cpu().numpy().view(np.uint32)[: int(bits.item()) // 32].copy())
    assert nuq.last_status() == 0
    return outs, hosts


def _guarded(torch, host):
    buf = torch.full((host.size + 2 * GUARD,), float("nan"), device="cuda")
    buf[GUARD:GUARD + host.size] = torch.from_numpy(host).cuda()
    return buf, buf[GUARD:GUARD + host.size]


def _inside(buf, d, what):
    host = buf.cpu().numpy()
    assert np.isnan(host[:GUARD]).all() and np.isnan(host[GUARD + d:]).all(), f"written outside {what}"
    return host[GUARD:GUARD + d].copy()


def _states(d, seed):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal(d).astype(np.float32), (0.1 * rng.standard_normal(d)).astype(np.float32),
            (np.square(rng.standard_normal(d)) * 0.1).astype(np.float32))


def _check(total, K, before, after, t, decay, scale=1.0, lr=R.LR):
    w0, m0, v0 = before
    m, v, dm, dv = R.moments(total, m0, v0, scale / K)
    w, dw = R.step(w0, m, v, dm, dv, t, np.float32(decay), lr)
    assert (np.abs(after[1] - m) <= dm).all() and (np.abs(after[2] - v) <= dv).all()
    assert (np.abs(after[0] - w) <= dw).all(), np.max(np.abs(after[0] - w) / dw)


@pytest.mark.parametrize("K,d,bucket,s,mode,levels,norm", [
    (1, 1, 256, 4, O.MODE_ERC, 0, 0), (1, 1, 256, 4, O.MODE_FIXED, 0, 0), (1, 3, 256, 3, O.MODE_FIXED, 0, 0),
    (1, 70001, 1024, 4, O.MODE_ERC, 0, 0), (2, 8192 * 3 + 17, 8192, 3, O.MODE_ERC, 0, 0), (8, 200000, 8192, 4, O.MODE_ERC, 0, 0),
    (9, 50000, 512, 4, O.MODE_ERC, 0, 0), (16, 9600 * 256 + 77, 1024, 3, O.MODE_ERC, 0, 0),
    (33, 60001, 512, 4, O.MODE_ERC, 0, 0), (64, 20000, 768, 3, O.MODE_FIXED, 0, 0),        # in two groups of streams, in eight
    (8, 100000, 8192, 4, O.MODE_FIXED, 0, 0), (4, 1_000_003, 8192, 4, O.MODE_FIXED, 0, 0),  # fields of 4, 3, 5 bits
    (3, 70001, 768, 2, O.MODE_FIXED, 0, 0), (3, 70001, 1024, 9, O.MODE_FIXED, 0, 0), (1, 255, 256, 4, O.MODE_FIXED, 0, 0),
    (3, 70001, 2048, 4, O.MODE_FIXED, 1, 1), (2, 70001, 2048, 7, O.MODE_FIXED, 1, 1), (3, 30001, 2048, 4, O.MODE_FIXED, 2, 0),
    (5, 70001, 4096, 4, O.MODE_ERC, 1, 1), (2, 70001, 4096, 8, O.MODE_ERC, 1, 0), (3, 30001, 2048, 4, O.MODE_ERC, 2, 0),
    (4, 100037, 8192, 3, O.MODE_CODED, 0, 0), (3, 200000, 65536, 4, O.MODE_ERC, 0, 0), (3, 200000, 65536, 4, O.MODE_FIXED, 0, 0),
])
@pytest.mark.parametrize("told", ["right", "as known", "wrong"])
def test_decode_adamw_matches_the_oracle_s_sum_and_the_formula(K, d, bucket, s, mode, levels, norm, told):
    torch, nuq = require_cuda()
    flags = O.make_flags(norm, levels, mode)
    outs, hosts = _streams(torch, nuq, d, bucket, s, flags, K, seed=d + K)
    rc, total = O.decode_accumulate(hosts, d, bucket, s)
    assert rc == 0
    if told != "as known":                                   # at addresses that no encode call has written
        outs = [x.clone() for x in outs]
    likely = {"right": flags & 0xFFFF00, "as known": nuq.LIKELY_AS_KNOWN, "wrong": O.MODE_FIXED << 16 if mode != O.MODE_FIXED else 0}[told]
    before = _states(d, d)
    bufs = [_guarded(torch, x) for x in before]
    accbuf, acc = _guarded(torch, np.zeros(d, np.float32))
    with_acc = (d + K) % 2 == 0
    nuq.decode_adamw(outs, d, bucket, s, *(x for _, x in bufs), lr=R.LR, weight_decay=0.1, step=5, scale=0.5, likely=likely, acc=acc if with_acc else None)
    assert nuq.last_status() == 0
    got = _inside(accbuf, d, "acc")
    assert np.array_equal(got.view(np.uint32), total.view(np.uint32)) if with_acc else not got.any()
    _check(total, K, before, [_inside(b, d, n) for (b, _), n in zip(bufs, "wmv")], 5, 0.1, 0.5)


@pytest.mark.parametrize("skew", [4, 8, 20])
@pytest.mark.parametrize("K,mode", [(3, O.MODE_ERC), (8, O.MODE_FIXED)])
def test_states_at_multiples_of_16_bytes(K, mode, skew):
    """w, m, v and acc need 16 bytes' alignment only, each its own"""
    torch, nuq = require_cuda()
    d, bucket, s = 70_001, 1024, 4
    outs, hosts = _streams(torch, nuq, d, bucket, s, O.make_flags(mode=mode), K)
    total = O.decode_accumulate(hosts, d, bucket, s)[1]
    before = _states(d, 3)
    bufs = [torch.full((d + 64,), float("nan"), device="cuda") for _ in range(4)]
    places = [b[k:k + d] for b, k in zip(bufs, (skew, 0, 4, skew + 4))]
    for x, y in zip(places, before):
        x.copy_(torch.from_numpy(y))
    nuq.decode_adamw(outs, d, bucket, s, *places[:3], lr=R.LR, step=2, acc=places[3], likely=LIKELY[mode])
    assert nuq.last_status() == 0
    assert np.array_equal(places[3].cpu().numpy().view(np.uint32), total.view(np.uint32))
    _check(total, K, before, [x.cpu().numpy() for x in places[:3]], 2, 0.0)
    for b in bufs:
        assert int(torch.isnan(b).sum()) == 64               # nothing else was written


def test_steps_on_two_streams_at_once():
    torch, nuq = require_cuda()
    d, bucket, s, K = 300_001, 8192, 4, 4
    work = []
    for mode in (O.MODE_ERC, O.MODE_FIXED):
        outs, hosts = _streams(torch, nuq, d, bucket, s, O.make_flags(mode=mode), K, seed=mode)
        before = _states(d, mode)
        work.append((mode, outs, O.decode_accumulate(hosts, d, bucket, s)[1], before, [torch.from_numpy(x).cuda() for x in before], torch.cuda.Stream(), nuq.step_control(mode + 3)))
    torch.cuda.synchronize()
    for mode, outs, _, _, state, stream, control in work:
        nuq.grad_norm(nuq.tensors([]), control, scale=0.5, stream=stream)
        nuq.decode_adamw(outs, d, bucket, s, *state, lr=R.LR, weight_decay=0.1, control=control, likely=LIKELY[mode], stream=stream)
    for mode, _, total, before, state, stream, _ in work:
        assert nuq.last_status(stream) == 0
        _check(total, K, before, [x.cpu().numpy() for x in state], mode + 4, 0.1, 0.5)


def test_streams_of_several_kinds():
    torch, nuq = require_cuda()
    d, bucket, s = 50_001, 1024, 4
    outs, hosts = [], []
    for mode in (O.MODE_ERC, O.MODE_FIXED, O.MODE_CODED, O.MODE_FIXED):
        a, b = _streams(torch, nuq, d, bucket, s, O.make_flags(mode=mode), 1, seed=mode)
        outs += a
        hosts += b
    total = O.decode_accumulate(hosts, d, bucket, s)[1]
    before = _states(d, 3)
    for likely in (nuq.LIKELY_AS_KNOWN, 0, 1 << 16):
        bufs = [_guarded(torch, x) for x in before]
        nuq.decode_adamw(outs, d, bucket, s, *(x for _, x in bufs), lr=R.LR, step=1, likely=likely)
        assert nuq.last_status() == 0
        _check(total, 4, before, [_inside(b, d, n) for (b, _), n in zip(bufs, "wmv")], 1, 0.0)


@pytest.mark.parametrize("mode", [O.MODE_ERC, O.MODE_FIXED])
def test_a_container_that_is_not_one(mode):
    torch, nuq = require_cuda()
    d, bucket, s = 30_000, 1024, 4
    outs, _ = _streams(torch, nuq, d, bucket, s, O.make_flags(mode=mode), 3)
    bad = [x.clone() for x in outs]
    bad[1][0] = 0                                            # the magic word
    bufs = [_guarded(torch, x) for x in _states(d, 3)]
    nuq.decode_adamw(bad, d, bucket, s, *(x for _, x in bufs), lr=R.LR, step=1, likely=LIKELY[mode])
    assert nuq.last_status() == nuq.ERR_BAD_STREAM
    for (b, _), n in zip(bufs, "wmv"):
        _inside(b, d, n)
    before = _states(d, 4)
    bufs = [_guarded(torch, x) for x in before]              # and the next call is as ever
    nuq.decode_adamw(outs, d, bucket, s, *(x for _, x in bufs), lr=R.LR, step=1, likely=LIKELY[mode])
    assert nuq.last_status() == 0


@pytest.mark.parametrize("mode", [O.MODE_ERC, O.MODE_FIXED])
def test_states_that_are_zero_infinite_or_nan(mode):
    torch, nuq = require_cuda()
    d, bucket, s, K = 4099, 256, 4, 2
    outs, hosts = _streams(torch, nuq, d, bucket, s, O.make_flags(mode=mode), K)
    total = O.decode_accumulate(hosts, d, bucket, s)[1]
    w, m, v = (x.copy() for x in _states(d, 3))
    m[:1000] = v[:1000] = 0.0
    m[2000], v[2001], w[2002] = np.nan, np.inf, np.nan
    bufs = [_guarded(torch, x) for x in (w, m, v)]
    nuq.decode_adamw(outs, d, bucket, s, *(x for _, x in bufs), lr=R.LR, step=1, likely=LIKELY[mode])
    after = [b.cpu().numpy()[GUARD:GUARD + d] for b, _ in bufs]
    assert np.isnan(after[0][2000]) and np.isnan(after[1][2000]) and np.isinf(after[2][2001]) and np.isnan(after[0][2002])
    rest = np.ones(d, bool)
    rest[2000:2003] = False
    _check(total[rest], K, [x[rest] for x in (w, m, v)], [x[rest] for x in after], 1, 0.0)
    assert abs(after[0][2001] - w[2001]) == 0.0              # an infinite root: no step


@pytest.mark.parametrize("mode", [O.MODE_ERC, O.MODE_FIXED])
@pytest.mark.parametrize("K", [2, 9])
def test_buckets_with_tiny_and_with_no_norms(mode, K):
    """norms below 2^-100, infinite and NaN ones: the slow way through a unit, with the step behind it"""
    torch, nuq = require_cuda()
    d, bucket, s = 256 * 40 + 77, 256, 4
    outs, hosts = [], []
    for k in range(K):
        g = _gradient(d, 50 + k)
        g[512:2048] *= np.float32(1e-33)
        if k == 1:
            g[2600], g[5000] = np.inf, np.nan
        out, bits = nuq.encode(torch.from_numpy(g).cuda(), bucket, s, O.make_flags(mode=mode), seed=k + 1)
        outs.append(out)
        hosts.append(out.cpu().numpy().view(np.uint32)[: int(bits.item()) // 32].copy())
    assert nuq.last_status() == nuq.WARN_NONFINITE
    rc, total = O.decode_accumulate(hosts, d, bucket, s)
    assert rc == 0 and np.isfinite(total).all()
    before = _states(d, 3)
    bufs = [_guarded(torch, x) for x in before]
    accbuf, acc = _guarded(torch, np.zeros(d, np.float32))
    nuq.decode_adamw(outs, d, bucket, s, *(x for _, x in bufs), lr=R.LR, step=1, likely=LIKELY[mode], acc=acc)
    assert nuq.last_status() == 0
    assert np.array_equal(_inside(accbuf, d, "acc").view(np.uint32), total.view(np.uint32))
    _check(total, K, before, [_inside(b, d, n) for (b, _), n in zip(bufs, "wmv")], 1, 0.0)


def test_record_skips_counts_and_scales():
    torch, nuq = require_cuda()
    d, bucket, s, K = 20_003, 1024, 4, 3
    for mode in (O.MODE_ERC, O.MODE_FIXED):
        outs, hosts = _streams(torch, nuq, d, bucket, s, O.make_flags(mode=mode), K)
        total = O.decode_accumulate(hosts, d, bucket, s)[1]
        before = _states(d, 3)
        bufs = [_guarded(torch, x) for x in before]
        accbuf, acc = _guarded(torch, np.zeros(d, np.float32))
        control = nuq.step_control(7)
        f = nuq.control_fields(control)
        f["skip"].fill_(1)
        f["scale"].fill_(1.0)
        nuq.decode_adamw(outs, d, bucket, s, *(x for _, x in bufs), lr=R.LR, control=control, likely=LIKELY[mode], acc=acc)
        for (b, _), x, n in zip(bufs, before, "wmv"):
            assert np.array_equal(_inside(b, d, n), x)
        assert np.array_equal(_inside(accbuf, d, "acc").view(np.uint32), total.view(np.uint32))
        nuq.grad_norm(nuq.tensors([]), control, scale=0.25)  # the step begins, without a norm
        f["lr_factor"].fill_(0.5)
        nuq.decode_adamw(outs, d, bucket, s, *(x for _, x in bufs), lr=R.LR, weight_decay=0.2, scale=2.0, control=control, likely=LIKELY[mode])
        assert nuq.last_status() == 0 and f["step"].item() == 8
        _check(total, K, before, [_inside(b, d, n) for (b, _), n in zip(bufs, "wmv")], 8, 0.2, 0.5, lr=0.5 * R.LR)


@pytest.mark.parametrize("mode", [O.MODE_ERC, O.MODE_FIXED])
def test_a_captured_exchange_step(mode):
    """encode, the step's beginning, decode and AdamW in one graph, replayed on changing gradients"""
    torch, nuq = require_cuda()
    d, bucket, s, K = 100_003, 1024, 4, 2
    flags = O.make_flags(mode=mode)
    grads = [torch.zeros(d, device="cuda") for _ in range(K)]
    make = lambda: [torch.from_numpy(x).cuda() for x in _states(d, 3)]  # noqa: E731
    outs = [torch.zeros(nuq.encode_bound(d, bucket, s, flags) // 4, dtype=torch.int32, device="cuda") for _ in range(K)]
    bits = torch.zeros(1, dtype=torch.int64, device="cuda")

    def call(state, control, stream=None):
        for k, g in enumerate(grads):
            nuq.encode(g, bucket, s, flags, seed=k, out=outs[k], out_bits=bits)
        nuq.grad_norm(nuq.tensors([]), control)
        nuq.decode_adamw(outs, d, bucket, s, *state, lr=0.01, control=control, likely=LIKELY[mode])

    a, b = make(), make()
    ca, cb = nuq.step_control(0), nuq.step_control(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        for g in grads:
            g.normal_()
        call(make(), nuq.step_control(0))                    # (what a capture does not allow is done by a call before it)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            call(a, ca)
    torch.cuda.current_stream().wait_stream(side)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(3):
        for g in grads:
            g.normal_(generator=gen)
        graph.replay()
        call(b, cb)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a, b)) and torch.equal(ca[:3], cb[:3])
    assert ca[0].item() == 3 and nuq.last_status() == 0


def test_decode_adamw_is_decode_then_adamw():
    """to rounding: w, m, v of the one call and of the three"""
    torch, nuq = require_cuda()
    d, bucket, s, K = 300_001, 8192, 4, 4
    outs, _ = _streams(torch, nuq, d, bucket, s, 0, K)
    a, b = ([torch.from_numpy(x).cuda() for x in _states(d, 3)] for _ in range(2))
    nuq.decode_adamw(outs, d, bucket, s, *a, lr=R.LR, weight_decay=0.1, step=3)
    total = nuq.decode_accumulate(outs, d, bucket, s)
    nuq.adamw(nuq.tensors([total], [b[0]], [b[1]], [b[2]], weight_decay=0.1), lr=R.LR, step=3, scale=1.0 / K)
    assert nuq.last_status() == 0
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])          # (the same roundings: 1 / 4 is exact)
    assert float((a[0] - b[0]).abs().max()) <= 2.0 ** -22 * float(a[0].abs().max())


def test_decode_adamw_refuses_what_does_not_fit():
    torch, nuq = require_cuda()
    d, bucket, s = 5000, 256, 3
    outs, _ = _streams(torch, nuq, d, bucket, s, 0, 2)
    z = lambda n=d, dtype=torch.float32: torch.zeros(n, dtype=dtype, device="cuda")  # noqa: E731
    w, m, v = z(), z(), z()
    both = z(2 * d - 4)
    for bad in (dict(w=z(d - 1)), dict(m=z(d, torch.float16)), dict(v=m), dict(acc=w), dict(m=both[:d], v=both[d - 4:]), dict(w=z(d + 1)[1:]), dict(step=0), dict(lr=-1.0)):
        args = {"w": w, "m": m, "v": v, "lr": 0.1, "step": 1, **bad}
        with pytest.raises((ValueError, nuq.NuqError)):
            nuq.decode_adamw(outs, d, bucket, s, args.pop("w"), args.pop("m"), args.pop("v"), **args)
    assert not w.any().item()


@pytest.mark.parametrize("mode", [O.MODE_ERC, O.MODE_FIXED])
def test_a_record_whose_step_no_norm_has_begun(mode):
    torch, nuq = require_cuda()
    d, bucket, s, K = 20_003, 1024, 4, 3
    outs, hosts = _streams(torch, nuq, d, bucket, s, O.make_flags(mode=mode), K)
    total = O.decode_accumulate(hosts, d, bucket, s)[1]
    before = _states(d, 3)
    bufs = [_guarded(torch, x) for x in before]
    accbuf, acc = _guarded(torch, np.zeros(d, np.float32))
    control = nuq.step_control(999)
    nuq.decode_adamw(outs, d, bucket, s, *(x for _, x in bufs), lr=R.LR, control=control, likely=LIKELY[mode], acc=acc)
    assert nuq.last_status() == 0
    for (b, _), x, n in zip(bufs, before, "wmv"):
        assert np.array_equal(_inside(b, d, n), x)
    assert np.array_equal(_inside(accbuf, d, "acc").view(np.uint32), total.view(np.uint32))
    nuq.grad_norm(nuq.tensors([]), control)
    nuq.decode_adamw(outs, d, bucket, s, *(x for _, x in bufs), lr=R.LR, control=control, likely=LIKELY[mode])
    _check(total, K, before, [_inside(b, d, n) for (b, _), n in zip(bufs, "wmv")], 1000, 0.0)


@pytest.mark.parametrize("call", ["decode_adamw", "decode_update"])
def test_a_backward_pass_through_parameters_from_before_the_step_is_an_error(call):
    torch, nuq = require_cuda()
    d, bucket, s = 5000, 256, 3
    outs, _ = _streams(torch, nuq, d, bucket, s, 0, 3)
    w = torch.randn(d, device="cuda", requires_grad=True)
    m, v = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    loss = w.square().sum()
    if call == "decode_adamw":
        nuq.decode_adamw(outs, d, bucket, s, w, m, v, lr=R.LR, step=1)
    else:
        nuq.decode_update(outs, d, bucket, s, w, alpha=0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    w.square().sum().backward()
    assert torch.equal(w.grad, 2 * w.detach())


def test_containers_in_host_memory_are_refused():
    torch, nuq = require_cuda()
    d, bucket, s = 5000, 256, 3
    outs, _ = _streams(torch, nuq, d, bucket, s, 0, 2)
    mixed = [outs[0], outs[1].cpu()]
    x = [torch.zeros(d, device="cuda") for _ in range(3)]
    for bad in (lambda: nuq.decode_adamw(mixed, d, bucket, s, *x, lr=0.1, step=1), lambda: nuq.decode_update(mixed, d, bucket, s, x[0], acc=x[1]),
                lambda: nuq.decode_update(outs, d, bucket, s, x[0], acc=x[1].cpu()), lambda: nuq.decode_accumulate(mixed, d, bucket, s, acc=x[0]),
                lambda: nuq.decode_accumulate(mixed, d, bucket, s)):
        with pytest.raises(ValueError):
            bad()
    assert not any(y.any().item() for y in x)
