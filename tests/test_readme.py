"""The README's example is run as it stands there."""
import os

import pytest

from gpu_util import require_cuda

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example(word):
    """the README's first code block that has `word` in it"""
    with open(os.path.join(ROOT, "README.md")) as f:
        return next(block for block in f.read().split("```")[1::2] if word in block)


@pytest.mark.gpu
def test_the_example_of_a_clipped_step_follows_new_gradients():
    """the example's loop on three exchanges of different gradients, against calls that make everything anew in every step"""
    torch, nuq = require_cuda()
    shapes, K, bucket, s = [(64, 33), (33,), (7, 5, 3), (1,)], 2, 256, 4
    sizes = [torch.Size(x).numel() for x in shapes]
    d = sum(sizes)
    gen = torch.Generator(device="cuda").manual_seed(3)
    start = [torch.randn(x, generator=gen, device="cuda") for x in shapes]
    exchanges = [[nuq.encode((10.0 ** -i) * torch.randn(d, generator=gen, device="cuda"), bucket, s, seed=k, offset=i)[0] for k in range(K)] for i in range(3)]
    names = {"torch": torch, "nuq": nuq, "exchanges": exchanges, "sizes": sizes, "weights": [x.clone() for x in start], "d": d, "bucket": bucket, "s": s, "K": K}
    exec(_example("nuq.tensors("), names)
    weights = [x.clone() for x in start]
    m, v = ([torch.zeros(n, dtype=torch.uint8, device="cuda") for n in sizes] for _ in range(2))
    scales = [torch.zeros(2 * -(-n // nuq.STATE_BLOCK), device="cuda") for n in sizes]
    control = nuq.step_control()
    for containers in exchanges:
        total = nuq.decode_accumulate(containers, d, bucket, s)
        tensors = nuq.tensors(torch.split(total, sizes), weights, m, v, scales=scales, weight_decay=[0.05 if w.dim() > 1 else 0.0 for w in weights])
        nuq.grad_norm(tensors, control, max_norm=1.0, scale=1.0 / K)
        nuq.adamw(tensors, lr=1e-3, seed=7, control=control)
    assert nuq.last_status() == 0 and control[0].item() == 3
    assert torch.equal(names["control"][:3], control[:3])
    assert all(torch.equal(a, b) for a, b in zip(names["weights"], weights))
