"""The linear layer, the norms and clipping at sizes, strides and alignments drawn from fixed
seeds, with nothing but NaN between and behind the rows; against 64-bit values within a
priori bounds."""
import math
import random

import pytest

torch = pytest.importorskip("torch")

import block_oracle as O  # noqa: E402
import test_gpu_clip as clip  # noqa: E402
import test_gpu_linear as linear  # noqa: E402
import test_gpu_norm as norm  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


class Drawn:
    def __init__(self, seed):
        self.rng = random.Random(seed)
        self.views = []

    def size(self, least, most):
        return int(round(math.exp(self.rng.uniform(math.log(least), math.log(most)))))

    def even(self):
        return self.rng.random() < 0.5

    def view(self, t):
        """t with rows apart, from any element on."""
        pad, skip = self.rng.choice((0, 1, 3, 8, 16, 32, 64)), self.rng.choice((0, 0, 1, 2, 4, 8))
        big = torch.full((t.shape[0] * (t.shape[1] + pad) + 64,), float("nan"), device="cuda", dtype=t.dtype)
        v = torch.as_strided(big[skip:], t.shape, (t.shape[1] + pad, 1))
        v.copy_(t)
        self.views.append((v, big))
        return v

    def check_gaps(self):
        for v, big in self.views:
            rest = torch.ones_like(big, dtype=torch.bool)
            torch.as_strided(rest, v.shape, v.stride(), v.storage_offset()).fill_(False)
            assert torch.isnan(big[rest]).all()


@pytest.mark.parametrize("seed", range(60))
def test_linear(seed):
    d = Drawn(seed)
    dtype, dw = d.rng.choice(((F32, F32), (BF16, BF16), (BF16, F32)))
    tokens = d.rng.randint(1, 140) if d.even() else d.size(1, 1500)
    dim, wide = d.size(1, 3000), d.size(1, 2000)
    if d.even():
        dim, wide = (dim + 31) // 32 * 32, (wide + 31) // 32 * 32
    name = d.rng.choice(O.ACTS)
    i = linear._inputs(tokens, dim, wide, dtype, seed=seed)
    for k in ("x", "w", "residual", "dy", "z"):
        i[k] = d.view(i[k])
    y, dx = d.view(torch.zeros_like(i["dy"])), d.view(torch.zeros_like(i["x"]))
    linear._forward(i, name, bias=d.even(), residual=d.even(), y=y)
    linear._backward(i, name, dw_dtype=dw, dx=dx, dw=d.view(torch.zeros(wide, dim, device="cuda", dtype=dw)))
    d.check_gaps()


@pytest.mark.parametrize("seed", range(30))
def test_norms(seed):
    d = Drawn(100 + seed)
    dtype, kind, post = d.rng.choice((F32, BF16)), d.rng.choice(("layer", "rms", "none")), d.rng.choice(("layer", "rms", "none"))
    i = norm._inputs(d.size(1, 400), d.size(1, 8192), dtype, seed=seed)
    for k in ("h", "f", "dy", "ds"):
        i[k] = d.view(i[k])
    outs = {k: d.view(torch.zeros_like(i["h"])) for k in (("s", "y") if kind != "none" else ("s",))}
    norm._run(i, kind, post, without=("gate",) if d.even() else (), forward=outs,
              backward={k: d.view(torch.zeros_like(i["h"])) for k in ("dh", "df")})
    d.check_gaps()


@pytest.mark.parametrize("seed", range(20))
def test_clipping(seed):
    d = Drawn(200 + seed)
    tensors, groups = [], []
    for _ in range(d.rng.randint(1, 70)):
        t = clip._tensors([(d.size(1, 300), d.size(1, 3000))], [d.rng.choice((F32, BF16))], seed=len(tensors))[0]
        tensors.append(d.view(t) if d.even() else t)
        groups.append(d.rng.randint(0, 3))
    clip._check(tensors, groups, d.rng.choice((0.5, 1.0, 100.0, 1e9)))
    d.check_gaps()
