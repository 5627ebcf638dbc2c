"""The optimizer's operators of this package, as cases to be timed and compared.

A case is one call on a list of tensors (`do`):

    norm     the Euclidean norm of all gradients together, the factor that clips it, the next step's number (grad_norm)
    adamw    an AdamW step over all tensors with states in 32 or in 8 bits; with `clip`, behind the norm and by its factor
             (adamw, or grad_norm and adamw)
    decode   the 4-bit containers of K workers decoded, averaged and applied as an AdamW step (decode_adamw)

Tensors are described by `sizes` (one, resnet18, resnet50: those networks' parameters; ragged: `count` tensors of very
different odd lengths that add up to `total`) and `layout`: packed (back to back in one buffer, as tensor fusion has
them, so that they start at any element) or aligned (each starts at a multiple of 64 elements). `grad` is the gradients'
type, `copy` the type of the low-precision copy of the fp32 parameters ("" for none).

Where `own` is false, the operators are computed from elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

BLOCK = 256                                                 # elements that share the scales of their 8-bit states
LR, BETA1, BETA2, EPS, DECAY, MAX_NORM = 1e-3, 0.9, 0.999, 1e-8, 0.05, 1.0
SEED = 0x1234567890ABCDEF                                   # of the 8-bit states' roundings
CONTROL_WORDS = 2048                                        # int64 words of the device's step record and its scratch
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
RESNET18, RESNET50 = 11_689_512, 25_557_032
LARGEST = 1 << 28


def _case(name, do, sizes, total, count=1, layout="aligned", grad="f32", copy="", state=32, clip=False, k=0, bucket=0, s=0):
    c = {"name": name} if name else {}
    c.update(do=do, sizes=sizes, total=total, count=count, layout=layout, grad=grad, copy=copy, state=state, clip=clip,
             k=k, bucket=bucket, s=s)
    return c


def listed():
    return [
        # the unquantized tensors of a network, biases and the like: launches and latency are all there is
        _case("norm small", "norm", "ragged", 30_011, 53, "packed"),
        # the decoded sum of a ResNet-50 step, before it is clipped
        _case("norm resnet50", "norm", "resnet50", RESNET50, 161, "packed"),
        # a large mixed-precision model's gradients
        _case("norm flat bf16", "norm", "one", LARGEST, grad="bf16"),
        # one small tensor: the smallest benchmark configuration's length
        _case("adamw small", "adamw", "one", 65536),
        # a ResNet-50 step on the decoded sum, parameters and states in one buffer each, clipped by the norm
        _case("adamw resnet50 clipped", "adamw", "resnet50", RESNET50, 161, "packed", clip=True),
        # several hundred tensors of any length, mixed precision: 16-bit gradients and copy, tensors allocated one by one
        _case("adamw ragged bf16", "adamw", "ragged", 50_000_003, 300, "aligned", "bf16", "bf16"),
        # a large model's shard
        _case("adamw flat", "adamw", "one", LARGEST, copy="bf16"),
        # the same three with states in 8 bits
        _case("adamw8 small", "adamw", "ragged", 65_549, 9, "aligned", state=8),
        _case("adamw8 resnet50", "adamw", "resnet50", RESNET50, 161, "packed", state=8),
        _case("adamw8 flat bf16", "adamw", "one", LARGEST, grad="bf16", copy="bf16", state=8),
        # the exchange's receiving end in 4 bits: a ResNet-18 with four workers, a ResNet-50 with eight
        _case("decode resnet18", "decode", "one", RESNET18, layout="packed", k=4, bucket=8192, s=4),
        _case("decode resnet50", "decode", "one", RESNET50, layout="packed", k=8, bucket=8192, s=4),
    ]


def draw(rng):
    do = rng.choice(["norm", "adamw", "adamw", "adamw8", "adamw8", "decode"])
    if do == "decode":
        k = rng.choice([1, 2, 3, 4, 5, 8])
        d = int(math.exp(rng.uniform(math.log(1 << 12), math.log(RESNET50 * 8 // max(k, 8)))))
        return _case(None, "decode", "one", d, layout="packed", k=k, bucket=rng.choice([256, 512, 768, 1024, 4096, 8192, 65536]), s=rng.randint(3, 6))
    count = 1 if rng.random() < 0.25 else int(math.exp(rng.uniform(0.0, math.log(600))))
    total = max(int(math.exp(rng.uniform(math.log(1 << 10), math.log(LARGEST)))), 2 * count)
    return _case(None, do[:5] if do != "norm" else do, "ragged" if count > 1 else "one", total, count,
                 rng.choice(["packed", "aligned"]), rng.choice(["f32", "f32", "bf16", "f16"]),
                 "" if do == "norm" else rng.choice(["", "", "bf16", "f16"]), 8 if do == "adamw8" else 32,
                 do != "norm" and rng.random() < 0.3)


def _conv(cin, cout, k):
    return [cout * cin * k * k, cout, cout]                 # a convolution, its normalisation's weight and bias


def _resnet(kind):
    sizes, cin = _conv(3, 64, 7), 64
    blocks, wide = ((2, 2, 2, 2), 1) if kind == "resnet18" else ((3, 4, 6, 3), 4)
    for stage, n in enumerate(blocks):
        width = 64 << stage
        for block in range(n):
            shape = [(cin, width, 3), (width, width, 3)] if wide == 1 else [(cin, width, 1), (width, width, 3), (width, 4 * width, 1)]
            sizes += [x for c in shape for x in _conv(*c)]
            if block == 0 and cin != wide * width:
                sizes += _conv(cin, wide * width, 1)
            cin = wide * width
    return sizes + [1000 * cin, 1000]


def _sizes(case):
    total, count = case["total"], case["count"]
    if case["sizes"] in ("resnet18", "resnet50"):
        return _resnet(case["sizes"])
    if count == 1:
        return [total]
    r = random.Random(total * 1009 + count)
    share = [math.exp(r.uniform(0.0, 8.0)) for _ in range(count)]
    sizes = [1 + int((total - count) * x / sum(share)) for x in share]
    sizes[-1] += total - sum(sizes)
    return sizes


class _State:
    pass


def _places(sizes, unit):
    """Where tensors of these sizes start when each starts at a multiple of `unit`, and the end."""
    at, starts = 0, []
    for n in sizes:
        starts.append(at)
        at += -(-n // unit) * unit
    return starts, at


def _quantized(x):
    """A state as it is kept in 8 bits, rounded to nearest here: codes of e4m3 and a scale per block."""
    x = x.view(-1, BLOCK)
    most = _most(x)
    return (x * (448.0 / most)[:, None]).to(torch.float8_e4m3fn).view(torch.uint8).reshape(-1), most / 448.0


def _most(x):
    """What the largest code stands for, for each row of x: its largest finite magnitude, and no less than 2^-100."""
    return torch.where(torch.isfinite(x), x.abs(), 0.0).amax(1).clamp(min=2.0 ** -100)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    st = _State()
    st.do, st.clip, st.state, st.table = case["do"], case["clip"], case["state"], None
    st.sizes = _sizes(case)
    st.starts, st.length = _places(st.sizes, 1 if case["layout"] == "packed" else 64)
    st.blocks, end = _places([-(-n // BLOCK) for n in st.sizes], 1)
    st.nblocks = end
    # matrices decay, biases and normalisation weights do not
    st.decays = [DECAY if n >= 4096 else 0.0 for n in st.sizes]
    st.control = torch.zeros(CONTROL_WORDS, dtype=torch.int64, device=dev)
    st.control[0] = 999                                     # steps taken
    st.control.view(torch.float32)[4] = 1.0                 # the learning rate's factor
    many = len(st.sizes) > 1

    def spread(per_tensor):                                 # one value per tensor, over the buffer
        if not many:
            return per_tensor[0]
        ends = st.starts[1:] + [st.length]
        gaps = torch.tensor([b - a for a, b in zip(st.starts, ends)], device=dev)
        return torch.repeat_interleave(torch.tensor(per_tensor, device=dev), gaps, output_size=st.length)

    r = random.Random(seed)
    scales = spread([10.0 ** r.uniform(-4.0, -1.5) for _ in st.sizes])
    inside = None                                           # 1 where a tensor is, 0 between two
    if case["layout"] != "packed" and st.length != sum(st.sizes):
        inside = torch.zeros(st.length, device=dev)
        for a, n in zip(st.starts, st.sizes):
            inside[a:a + n] = 1.0

    def normal():
        x = torch.randn(st.length, generator=gen, device=dev)
        return x if inside is None else x.mul_(inside)

    if st.do == "decode":
        st.d, st.bucket, st.s = case["total"], case["bucket"], case["s"]
        st.containers = [_container(normal().mul_(scales), st.bucket, st.s, gen) for _ in range(case["k"])]
    else:
        # heavy tails, as gradients have them
        st.g = normal().mul_(normal().abs_().add_(0.5)).mul_(scales).to(TYPES[case["grad"]])
    if st.do == "norm":
        return st
    st.w = normal().mul_(0.05)
    st.copy = st.w.to(TYPES[case["copy"]]) if case["copy"] else None
    m = normal().mul_(0.2).mul_(scales)
    v = normal().square_().add_(0.3).mul_(scales).mul_(scales)
    if inside is not None:
        v.mul_(inside)
    if st.state == 32:
        st.m, st.v = m, v
        return st
    st.scales = torch.empty(st.nblocks, 2, device=dev)
    codes = []
    for i, x in enumerate((m, v.sqrt_())):
        blocks = torch.zeros(st.nblocks * BLOCK, device=dev)
        for a, b, n in zip(st.starts, st.blocks, st.sizes):
            blocks[b * BLOCK:b * BLOCK + n] = x[a:a + n]
        c, st.scales[:, i] = _quantized(blocks)
        codes.append(c)
    st.m, st.v = codes
    return st


def _container(g, bucket, s, gen):
    """One worker's gradient in a container of 4-bit fields (sign, level index), as it is received."""
    d, dev = g.numel(), g.device
    nb = -(-d // bucket)
    x = torch.zeros(nb * bucket, device=dev)
    x[:d] = g
    x = x.view(nb, bucket)
    norm = x.double().square().sum(1).sqrt().float()
    y = (x.abs() / norm[:, None]).clamp_(max=1.0).mul_(2.0 ** s)
    e = torch.floor(torch.log2(y.clamp(min=1.0))).clamp_(max=s - 1)
    low = torch.where(y < 1.0, torch.zeros_like(y), e + 1)
    p = torch.where(y < 1.0, y, y * torch.exp2(-e) - 1.0)
    index = low + (torch.rand(y.shape, generator=gen, device=dev) < p)
    field = (index + 8.0 * ((x < 0) & (index > 0))).to(torch.int64).view(nb, bucket // 8, 8)
    word = (field << torch.arange(28, -1, -4, device=dev)).sum(2)
    record = torch.cat([norm.view(torch.int32).view(nb, 1).to(torch.int64) & 0xFFFFFFFF, word], 1).view(-1)
    last = d - (nb - 1) * bucket
    words = 16 + (nb - 1) * (1 + bucket // 8) + 1 + (last + 7) // 8
    bits = 32 * words
    nnz = int((index > 0).sum())
    low32 = 0xFFFFFFFF
    head = [0x3151554E, 1, d & low32, d >> 32, bucket, s, 1 << 16, 256, nb & low32, nb >> 32, bits & low32, bits >> 32,
            (4 * d) & low32, (4 * d) >> 32, nnz & low32, nnz >> 32]
    out = torch.zeros((words + 3) // 4 * 4, dtype=torch.int64, device=dev)
    out[:16] = torch.tensor(head, device=dev)
    out[16:words] = record[:words - 16]
    return torch.where(out >= 1 << 31, out - (1 << 32), out).to(torch.int32)


# ---- the plain forms ----

def _control(st):
    f = st.control.view(torch.float32)
    return {"step": st.control[0], "norm": f[2], "scale": f[3], "skip": st.control.view(torch.int32)[5]}


def _plain_norm(st):
    f = st.control.view(torch.float32)
    norm = st.g.float().square().sum(dtype=torch.float64).sqrt().float()
    fine = torch.isfinite(norm)
    f[2] = norm
    f[3] = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm))
    st.control.view(torch.int32)[5] = ~fine
    st.control[0] += fine.to(torch.int64)


def _corrections(st):
    """lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t), t, the gradients' factor and whether the step is taken."""
    if not st.clip:
        t = 1000
        return LR / (1.0 - BETA1 ** t), 1.0 / math.sqrt(1.0 - BETA2 ** t), t, 1.0, None
    f, t = st.control.view(torch.float32), st.control[0]
    lr = LR * f[4].double()
    first = (lr / (1.0 - torch.pow(BETA1, t.double()))).float()
    second = (1.0 / torch.sqrt(1.0 - torch.pow(BETA2, t.double()))).float()
    return first, second, t, f[3], st.control.view(torch.int32)[5] == 0


def _kept(st):
    """1 - lr * decay of each element."""
    if len(st.sizes) == 1:
        return 1.0 - LR * st.decays[0]
    dev = st.w.device
    spans = torch.tensor([b - a for a, b in zip(st.starts, st.starts[1:] + [st.length])], device=dev)
    kept = torch.tensor([1.0 - LR * x for x in st.decays], device=dev)
    return torch.repeat_interleave(kept, spans, output_size=st.length)


def _plain_step(st, g, m, v, root, first, second, taken):
    """The parameters' part of the step, with the new moments."""
    w = st.w * _kept(st) - (m * first) / (root * second + EPS)
    if taken is not None:
        w = torch.where(taken, w, st.w)
    st.w.copy_(w)
    if st.copy is not None:
        st.copy.copy_(w)


def _plain_adamw(st, g):
    first, second, _, scale, taken = _corrections(st)
    g = g * scale
    m = st.m * BETA1 + g * (1.0 - BETA1)
    v = st.v * BETA2 + (g * g) * (1.0 - BETA2)
    _plain_step(st, g, m, v, v.sqrt(), first, second, taken)
    if taken is not None:
        m, v = torch.where(taken, m, st.m), torch.where(taken, v, st.v)
    st.m.copy_(m)
    st.v.copy_(v)


LOW = 0xFFFFFFFF


def _philox(c0, c1, c2, c3, k0, k1, rounds):
    """Philox4x32 of the counter words (int64 tensors or numbers that hold 32 bits)."""
    if rounds == 0:
        return c0, c1, c2, c3
    a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
    return _philox(((b >> 32) & LOW) ^ c1 ^ k0, b & LOW, ((a >> 32) & LOW) ^ c3 ^ k1, a & LOW,
                   (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW, rounds - 1)


def _coded(x, most, random16):
    """448 x / most in e4m3, rounded up with the probability that keeps the mean; 0x7f where x is not finite."""
    y = x.abs() * (448.0 / most)[:, None]
    small = y < 2.0 ** -6
    bits = torch.where(small, y + 2.0 ** -6, y).view(torch.int32) + (random16 * 16 + 8).to(torch.int32)
    code = (bits >> 20) - torch.where(small, 968, 960)
    code = torch.where(torch.isfinite(x), code, 0x7F)
    return code + torch.where(torch.signbit(x), 128, 0)


def _plain_adamw8(st):
    dev, n = st.w.device, sum(st.sizes)
    first, second, t, scale, taken = _corrections(st)
    # the elements' places in the buffer and in the blocks
    if len(st.sizes) == 1:
        flat, block = slice(0, n), slice(0, n)
    else:
        sizes = torch.tensor(st.sizes, device=dev)
        before = torch.cumsum(sizes, 0) - sizes
        i = torch.arange(n, device=dev)
        flat = i + torch.repeat_interleave(torch.tensor(st.starts, device=dev) - before, sizes, output_size=n)
        block = i + torch.repeat_interleave(torch.tensor(st.blocks, device=dev) * BLOCK - before, sizes, output_size=n)
    g = torch.zeros(st.nblocks * BLOCK, device=dev)
    g[block] = st.g[flat].float()
    g = g * scale
    spans = torch.tensor([b - a for a, b in zip(st.blocks, st.blocks[1:] + [st.nblocks])], device=dev)
    tensor = torch.repeat_interleave(torch.arange(len(st.sizes), device=dev), spans, output_size=st.nblocks)
    inside = torch.arange(st.nblocks, device=dev) - torch.tensor(st.blocks, device=dev)[tensor]
    quad = (inside[:, None] * 64 + torch.arange(64, device=dev)).view(-1)
    words = _philox(quad & LOW, quad >> 32, t & LOW, torch.repeat_interleave(tensor, 64), SEED & LOW, SEED >> 32, 10)
    words = torch.stack(words, 1).view(-1, BLOCK)
    held = [(c.view(torch.float8_e4m3fn).float().view(-1, BLOCK) * st.scales[:, i:i + 1]).view(-1) for i, c in enumerate((st.m, st.v))]
    m = held[0] * BETA1 + g * (1.0 - BETA1)
    v = (held[1] * held[1]) * BETA2 + (g * g) * (1.0 - BETA2)
    root = v.sqrt()
    mf, rf = torch.zeros(st.length, device=dev), torch.zeros(st.length, device=dev)
    mf[flat], rf[flat] = m[block], root[block]
    _plain_step(st, g, mf, None, rf, first, second, taken)
    new = []
    for x, bits in ((m, words & 0xFFFF), (root, words >> 16)):
        x = x.view(-1, BLOCK)
        most = _most(x)
        new.append((_coded(x, most, bits), most / 448.0))
    new[1] = (torch.where((root.view(-1, BLOCK) > 0) & (new[1][0] == 0), 1, new[1][0]), new[1][1])
    for i, (old, (code, size)) in enumerate(zip((st.m, st.v), new)):
        code = code.to(torch.uint8).view(-1)
        if taken is not None:
            code, size = torch.where(taken, code, old), torch.where(taken, size, st.scales[:, i])
        old.copy_(code)
        st.scales[:, i] = size


def _plain_decode(st):
    """The mean of the decoded containers."""
    nb, words, dev = -(-st.d // st.bucket), 1 + st.bucket // 8, st.w.device
    body = torch.zeros(len(st.containers), nb * words, dtype=torch.int32, device=dev)
    every = torch.stack(st.containers)[:, 16:]
    n = min(every.shape[1], nb * words)
    body[:, :n] = every[:, :n]
    body = body.view(len(st.containers), nb, words)
    norm = body[:, :, :1].contiguous().view(torch.float32)
    field = (body[:, :, 1:, None] >> torch.arange(28, -1, -4, device=dev, dtype=torch.int32)) & 15
    level = torch.tensor([0.0] + [2.0 ** (j - 1 - st.s) for j in range(1, 8)], device=dev)
    value = torch.cat([level, -level])[field.view(len(st.containers), nb, -1)] * norm
    return value.view(len(st.containers), -1).sum(0)[:st.d] / len(st.containers)


# ---- a pass ----

def _table(st):
    """The list of tensors as the package takes it: made once and kept, as a training program keeps it."""
    from paper_1908_06077_b200 import nuq

    def parts(x):
        return None if x is None else [x[a:a + n] for a, n in zip(st.starts, st.sizes)]

    if st.do == "norm":
        return nuq.tensors(parts(st.g))
    if st.state == 32:
        return nuq.tensors(parts(st.g), parts(st.w), parts(st.m), parts(st.v), copy=parts(st.copy), weight_decay=st.decays)
    ends = [b + -(-n // BLOCK) for b, n in zip(st.blocks, st.sizes)]
    m, v = [[x[b * BLOCK:b * BLOCK + n] for b, n in zip(st.blocks, st.sizes)] for x in (st.m, st.v)]
    return nuq.tensors(parts(st.g), parts(st.w), m, v, scales=[st.scales[b:e] for b, e in zip(st.blocks, ends)],
                       copy=parts(st.copy), weight_decay=st.decays)


def _own(st):
    from paper_1908_06077_b200 import nuq
    if st.do == "decode":
        nuq.decode_adamw(st.containers, st.d, st.bucket, st.s, st.w, st.m, st.v, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS,
                         weight_decay=st.decays[0], step=1000, likely=nuq.MODE_FIXED)
        return
    if st.table is None:
        st.table = _table(st)
    if st.do == "norm" or st.clip:
        nuq.grad_norm(st.table, st.control, max_norm=MAX_NORM)
    if st.do == "adamw":
        when = {"control": st.control} if st.clip else {"step": 1000}
        nuq.adamw(st.table, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, seed=SEED, **when)


def run(st):
    if own:
        _own(st)
    elif st.do == "decode":
        _plain_adamw(st, _plain_decode(st))
    else:
        if st.do == "norm" or st.clip:
            _plain_norm(st)
        if st.do == "adamw" and st.state == 32:
            _plain_adamw(st, st.g.float())
        elif st.do == "adamw":
            _plain_adamw8(st)
    out = {}
    if st.do == "norm" or st.clip:
        out.update(_control(st))
    if st.do != "norm":
        out["w"] = st.w
        if st.copy is not None:
            out["copy"] = st.copy
        if st.state == 32:
            out.update(m=st.m, v=st.v)
        else:                                               # codes as the numbers they are, relative to their block's scale
            out.update(m=st.m.view(torch.float8_e4m3fn), v=st.v.view(torch.float8_e4m3fn), scales=st.scales)
    return out


def _container_bytes(case):
    return 64.0 + 4.0 * math.ceil(case["total"] / case["bucket"]) + case["total"] / 2


def work(case):
    n = float(case["total"])
    grad = n * (4 if case["grad"] == "f32" else 2)
    if case["do"] == "norm":
        return {"bytes": grad, "flops": 2 * n}
    copy = 2 * n if case["copy"] else 0.0
    if case["do"] == "decode":
        return {"bytes": case["k"] * _container_bytes(case) + 24 * n, "flops": (2.0 * case["k"] + 15) * n}
    step = (24 * n if case["state"] == 32 else 12 * n + 16 * n / BLOCK) + copy
    clip = 1 if case["clip"] else 0                         # (the norm has to be known before the first parameter moves)
    return {"bytes": grad * (1 + clip) + step, "flops": (15.0 if case["state"] == 32 else 60.0) * n + 2 * n * clip}


# ---- the definition in 64 bits ----

def _nearest_below(x):
    """x >= 0 as a multiple of e4m3's spacing there: the multiple below, the part above it, the spacing."""
    e = torch.floor(torch.log2(x.clamp(min=2.0 ** -6)))
    e = torch.where(torch.exp2(e) > x.clamp(min=2.0 ** -6), e - 1, e)
    spacing = torch.exp2(e - 3)
    q = x / spacing
    return torch.floor(q), q - torch.floor(q), spacing


def _random_words(n, step, tensor, dev):
    """The four output words of each counter, for a tensor of n elements."""
    q = torch.arange(-(-n // 4), device=dev)
    x = [q & LOW, q >> 32, torch.full_like(q, step & LOW), torch.full_like(q, tensor)]
    key = [SEED & LOW, SEED >> 32]
    for _ in range(10):
        products = [x[0] * 0xD2511F53, x[2] * 0xCD9E8D57]
        high, low = [(p >> 32) & LOW for p in products], [p & LOW for p in products]
        x = [high[1] ^ x[1] ^ key[0], low[1], high[0] ^ x[3] ^ key[1], low[0]]
        key = [(key[0] + 0x9E3779B9) & LOW, (key[1] + 0xBB67AE85) & LOW]
    return torch.stack(x, 1).view(-1)[:n]


def exact(case, seed):
    st = prepare(case, seed)
    dev = st.control.device
    out, step, factor = {}, 1000, 1.0
    if st.do == "decode":
        i = torch.arange(st.d, device=dev)
        bucket, j = i // st.bucket, i % st.bucket
        record = 16 + bucket * (1 + st.bucket // 8)         # the word with the bucket's norm
        byte = 4 * (record + 1 + j // 8) + 3 - j % 8 // 2   # (words are little endian, fields start at the top)
        total = torch.zeros(st.d, dtype=torch.float64, device=dev)
        for c in st.containers:
            field = c.view(torch.uint8)[byte].int() >> 4 * (1 - j % 2).int()
            index, sign = field & 7, 1 - 2 * (field >> 3 & 1)
            size = torch.where(index > 0, 2.0 ** (index.double() - 1 - st.s), 0.0)
            total += sign * size * c[record].view(torch.float32).double()
        g = total / len(st.containers)
    else:
        g = st.g.double()
    if st.do == "norm" or st.clip:
        norm = float(torch.linalg.vector_norm(g))
        factor = min(1.0, MAX_NORM / norm) if norm else 1.0
        out.update(step=torch.tensor(1000), norm=torch.tensor(norm, dtype=torch.float64),
                   scale=torch.tensor(factor, dtype=torch.float64), skip=torch.tensor(0, dtype=torch.int32))
    if st.do == "norm":
        return out
    g = g * factor
    lr, second = LR / (1.0 - BETA1 ** step), math.sqrt(1.0 - BETA2 ** step)
    w = st.w.double()
    if st.state == 32:
        m, v = BETA1 * st.m.double() + (1.0 - BETA1) * g, BETA2 * st.v.double() + (1.0 - BETA2) * g * g
        out.update(m=m, v=v)
        for a, n, decay in zip(st.starts, st.sizes, st.decays):
            p = slice(a, a + n)
            w[p] -= LR * decay * w[p] + lr * m[p] / (torch.sqrt(v[p]) / second + EPS)
    else:
        codes = [x.view(torch.float8_e4m3fn).double() for x in (st.m, st.v)]
        scales = st.scales.double()
        for i, (a, b, n, decay) in enumerate(zip(st.starts, st.blocks, st.sizes, st.decays)):
            p, q = slice(a, a + n), slice(b * BLOCK, b * BLOCK + n)
            blocks = torch.arange(n, device=dev) // BLOCK + b
            held = [codes[j][q] * scales[blocks, j] for j in (0, 1)]
            m, v = BETA1 * held[0] + (1.0 - BETA1) * g[p], BETA2 * held[1] ** 2 + (1.0 - BETA2) * g[p] ** 2
            w[p] -= LR * decay * w[p] + lr * m / (torch.sqrt(v) / second + EPS)
            word = _random_words(n, step, i, dev)
            for j, (x, bits) in enumerate(((m, word & 0xFFFF), (torch.sqrt(v), word >> 16))):
                most = torch.zeros(-(-n // BLOCK) * BLOCK, dtype=torch.float64, device=dev)
                most[:n] = x.abs()
                scale = most.view(-1, BLOCK).amax(1).clamp(min=2.0 ** -100) / 448.0
                size = scale[torch.arange(n, device=dev) // BLOCK]
                whole, rest, spacing = _nearest_below(x.abs() / size)
                up = rest * 2.0 ** 20 + (bits * 16 + 8).double() >= 2.0 ** 20
                code = (whole + up) * spacing
                if j == 1:
                    code = torch.where((code == 0) & (x > 0), 2.0 ** -9, code)
                codes[j][q] = torch.where(x < 0, -code, code)
                scales[b:b + scale.numel(), j] = scale
        out.update(m=codes[0], v=codes[1], scales=scales)
    out["w"] = w
    if st.copy is not None:
        out["copy"] = w
    return out
