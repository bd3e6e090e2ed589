"""The slopes of the linear layer's activations on the GPU, relative to their own size: far below 0
they fall to nothing, as the formulas' do, and far above they are 1.

With one token that has a gradient of ones, dbias is dz in fp32: the slopes themselves.  Bounds count
roundings of half a step, U = 2^-24.  The argument u of an exponential is off by up to 5 U |u| (three
roundings, two more for exp2's), and so is the exponential, relative to itself; 24 U are the rest (exp and
erfc by up to 2 steps each, the reciprocal, the products and sums).  erfc's argument is off by 2 U, erfc by
2 U z^2 therefore.  In bf16 erfc is a polynomial's, 2^-19.  Exponentials below the normal numbers keep fp32's last
digit (2^-149), and are 0 where exp2 is the hardware's (bf16).  All this is relative to the slope's two terms, which meet
with opposite signs around -1."""
import math

import pytest

torch = pytest.importorskip("torch")

import block_oracle as O  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
FAR = (1e4, 1e12, 1e30, math.inf)


def slopes(name, z, dtype):
    """(the slopes, how far they may be off), float64."""
    least = 2.0 ** -126 if dtype == BF16 else 2.0 ** -147
    if name == "gelu":
        share, bell = 0.5 * torch.erfc(-z / math.sqrt(2)), torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
        along = torch.where(bell > 0, z * bell, 0.0)
        off = (3 * z * z).clamp(max=1e6) + 24 + (2.0 ** 5 if dtype == BF16 else 0)
        rate = torch.ones_like(z)
    else:
        c = 2 * math.sqrt(2 / math.pi)
        u = z if name == "silu" else c * (z + 0.044715 * z ** 3)
        rate = torch.ones_like(z) if name == "silu" else c * (1 + 3 * 0.044715 * z * z)
        share = torch.sigmoid(u)
        bell = share * torch.sigmoid(-u)
        along = torch.where(bell > 0, z * rate * bell, 0.0)
        off = (5 * u.abs()).clamp(max=1e6) + 24
    size = 1 + (z.abs() * rate).clamp(max=1e5)
    return share + along, off * O.U * (share + along.abs()) + least * size


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("name", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("tokens", [1, 40, 150])
def test_slopes_far_from_zero(tokens, name, dtype):
    from paper_2411_17866_amd import ops
    z = torch.cat([torch.linspace(-220, 220, 4001), torch.linspace(-16, 16, 3001), torch.tensor([s * v for v in FAR for s in (-1, 1)])])
    z = z.cuda().to(dtype)
    wide = z.numel()
    rows = torch.zeros(tokens, wide, device="cuda", dtype=dtype)
    rows[tokens // 2] = z
    dy = torch.zeros_like(rows)
    dy[tokens // 2] = 1
    plan = ops.Linear(tokens, 8, wide, dtype=dtype, act=name)
    got = plan.backward(dy, z=rows, wanted=("dbias",))["dbias"].double()
    want, bound = slopes(name, z.double(), dtype)
    assert torch.isfinite(want).all() and torch.isfinite(got).all()
    off = (got - want).abs() - bound
    worst = int(off.argmax())
    assert float(off[worst]) <= 0, (float(z[worst]), float(got[worst]), float(want[worst]), float(bound[worst]))
    far = z.abs() >= 1e4
    assert torch.equal(got[far], (z[far] > 0).double())
