"""Clipped gradients on the GPU are rounded once, from fp64 to their type: products that lie next to the
middle between two numbers of bf16, nearer than fp32 can tell, go to the side on which they lie."""
import math
import random

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
PAIRS = 2500  # of (3, 4): their norm is 5 * 50


def rounded(v):
    """A positive float64 tensor's nearest numbers of bf16, of two as near the even one."""
    bits = (v.float().view(torch.int32) >> 16).to(torch.int64)  # by truncation, or one further
    near = torch.stack([(bits + k).clamp(min=0) for k in (-1, 0, 1, 2)])
    values = (near << 16).to(torch.int32).view(torch.float32).double()
    off = (values - v).abs()
    odd = torch.where(off == off.min(0).values, near & 1, 2)
    return values.gather(0, odd.argmin(0)[None])[0]


def next_to_a_middle(scale, seed):
    """(max_norm in fp32, the clipped 3 and 4 times scale): one of them so near a middle that by way of fp32 it
    goes to the wrong side."""
    rng = random.Random(seed)
    pair, norm = torch.tensor([3.0, 4.0], dtype=torch.float64) * scale, 250.0 * scale
    for _ in range(5000):
        g = float(pair[rng.choice((0, 1))])
        step = max(2.0 ** (math.floor(math.log2(g)) - 8), 2.0 ** -133)  # of bf16 between g / 2 and g / 4, or of its smallest numbers
        middle = (rng.randrange(40 if step == 2.0 ** -133 else 128, 256) + 0.5) * step
        most = float(torch.tensor(middle / g * norm, dtype=torch.float64).float())
        product = pair * min(1.0, most / norm)
        if most < norm and not torch.equal(product.float().to(BF16).double(), rounded(product)):
            return most, rounded(product)
    raise AssertionError("no such maximum")


@pytest.mark.parametrize("scale", [1.0, 2.0 ** 100, 2.0 ** -120, 2.0 ** -126])
@pytest.mark.parametrize("seed", range(4))
def test_products_next_to_a_middle(seed, scale):
    from paper_2411_17866_amd import ops
    most, want = next_to_a_middle(scale, seed)
    want = want.repeat(PAIRS)
    g = (torch.tensor([3.0, 4.0], dtype=torch.float64) * scale).to(BF16).repeat(PAIRS)
    room = torch.zeros(2 * PAIRS + 1, device="cuda", dtype=BF16)
    for sign in (1, -1):
        for t in (g.cuda() * sign, room[1:].copy_(g * sign), (g.view(100, 50).cuda() * sign)):
            norm = ops.GradClip([t], eps=0.0)([t], most)
            assert float(norm[0]) == 250.0 * scale
            assert torch.equal(t.double().cpu().flatten(), want * sign)
