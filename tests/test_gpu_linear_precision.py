"""The linear layer's gradients on the GPU against differences of its own forward pass, each along the
gradient itself, so that none that is too small, too large or turned passes; and fp32 products of few
tokens, which take their operands' bits, against bounds without the halves' share."""
import math

import pytest

torch = pytest.importorskip("torch")

import block_oracle as O  # noqa: E402

pytestmark = pytest.mark.gpu

F32 = torch.float32


def _inputs(tokens, dim, wide, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, sigma=1.0):
        return torch.empty(shape, device="cuda").normal_(0, sigma, generator=gen)

    return dict(x=normal(tokens, dim), w=normal(wide, dim, sigma=dim ** -0.5), bias=normal(wide, sigma=0.5),
                dy=normal(tokens, wide) * torch.exp(normal(tokens, 1)), z=normal(tokens, wide, sigma=1.5))


def _along(i, key, v):
    """How z moves with i[key] along v, float64."""
    if key == "bias":
        return v.expand(i["x"].shape[0], -1)
    return v @ i["w"].double().t() if key == "x" else i["x"].double() @ v.t()


@pytest.mark.parametrize("name", O.ACTS)
@pytest.mark.parametrize("tokens", [40, 100, 150])
def test_gradients_against_differences_along_themselves(tokens, name):
    """With v along the gradient, of such a size that z moves by 1 on average, (L(+h v) - L(-h v)) / 2 h is
    |gradient| |v|.  It is off by h^2 / 6 of the third derivative (no activation's is above 1 anywhere; the places'
    own rounding moves their middle by 2^-24, which is less than h^2 / 100 of it), by the forward pass's errors
    over h, and the gradient by its own, each within its bound.  Together that is below 3% of the value, so a
    gradient that is 0, or 4% too small, does not pass."""
    from paper_2411_17866_amd import ops
    dim, wide, h = 40, 50, 2.0 ** -6
    i = _inputs(tokens, dim, wide, seed=13)
    if name == "relu":  # away from the kink, over which a difference is no derivative
        i["bias"] = torch.where(torch.arange(wide, device="cuda") % 2 == 0, 9.0, -9.0)
    plan = ops.Linear(tokens, dim, wide, act=name)
    z = plan(i["x"], i["w"], bias=i["bias"], z=torch.empty_like(i["z"]))["z"]
    out = plan.backward(i["dy"], i["x"], i["w"], z=z if name != "none" else None)
    e = O.linear_backward(i["dy"], i["x"], i["w"], z, name)
    bounds = O.linear_backward_bounds(e, i["dy"], i["x"], i["w"], name, F32)
    dy = i["dy"].double()
    for key, grad in (("x", "dx"), ("w", "dw"), ("bias", "dbias")):
        g = out[grad].double()
        v = g / g.norm()
        v = (v / _along(i, key, v).square().mean().sqrt()).float().double()
        # The places as fp32 has them, and the step between them.
        up, down = ((i[key].double() + sign * h * v).float() for sign in (1, -1))
        v = (up.double() - down.double()) / (2 * h)
        moved = _along(i, key, v)

        def total(place):
            at = dict({k: i[k] for k in ("x", "w", "bias")}, **{key: place})
            off = O.linear_bounds(at["x"], at["w"], at["bias"], None, name, tokens <= 128)["y"]
            return float((plan(**at)["y"].double() * dy).sum()), float((dy.abs() * off).sum())

        (above, off_above), (below, off_below) = total(up), total(down)
        want, got = (above - below) / (2 * h), float((g * v).sum())
        bend = 0.0 if name in ("none", "relu") else h * h / 6 * float((dy.abs() * moved.abs() ** 3).sum())
        tolerance = (off_above + off_below) / (2 * h) + bend + float((bounds[grad] * v.abs()).sum())
        assert tolerance < 0.03 * got, (key, tolerance, got)
        assert abs(got - want) <= tolerance, (key, got, want, tolerance)
        for wrong in (0.0, 0.96 * got, 1.04 * got):
            assert abs(wrong - want) > tolerance, key


@pytest.mark.parametrize("name", ["none", "gelu", "silu"])
@pytest.mark.parametrize("size", [(65, 64, 64), (66, 33, 129), (90, 1600, 48), (100, 96, 300), (127, 129, 130), (128, 128, 128), (128, 700, 2100)], ids=str)
def test_products_of_up_to_128_tokens_take_their_operands_bits(size, name):
    from paper_2411_17866_amd import ops
    i = _inputs(*size, seed=sum(size))
    out = ops.Linear(*size, act=name)(i["x"], i["w"], bias=i["bias"])
    e = O.linear(i["x"], i["w"], i["bias"], None, name)
    O.check(out, e, O.linear_bounds(i["x"], i["w"], i["bias"], None, name, True), list(out))


@pytest.mark.parametrize("tokens", [1, 17, 33, 64, 65, 100, 128])
def test_entries_far_below_their_rows_largest_count(tokens):
    """x's rows hold 2^45 and entries of 1, which meet 0 and entries of 1 in w: all that is left in y is a sum of
    what an operand of 22 bits would have lost.  In the gradients (up to 64 tokens) dz's rows do the same, and w's."""
    from paper_2411_17866_amd import ops
    dim, wide = 96, 80
    i = _inputs(tokens, dim, wide, seed=3)
    i["x"][:, 5] = 2.0 ** 45
    i["w"][:, 5] = 0
    plan = ops.Linear(tokens, dim, wide)
    y = plan(i["x"], i["w"])["y"]
    O.check_norm(y, O.linear(i["x"], i["w"])["y"], O.norm_bound(dim, F32), "y")
    if tokens > 64:
        return
    i = _inputs(tokens, dim, wide, seed=4)
    i["dy"][:, 7] = 2.0 ** 45
    i["w"][7] = 0
    dx = plan.backward(i["dy"], i["x"], i["w"], wanted=("dx",))["dx"]
    O.check_norm(dx, O.linear_backward(i["dy"], i["x"], i["w"])["dx"], O.norm_bound(wide, F32), "dx")
    i["x"][:, 3] = 2.0 ** 45  # (other columns of dw do not see it)
    dw = plan.backward(i["dy"], i["x"], i["w"], wanted=("dw",))["dw"]
    want = O.linear_backward(i["dy"], i["x"], i["w"])["dw"]
    rest = [torch.arange(n, device="cuda") != k for n, k in ((wide, 7), (dim, 3))]
    O.check_norm(dw[rest[0]][:, rest[1]], want[rest[0]][:, rest[1]], O.norm_bound(tokens, F32), "dw")


def test_third_derivatives_stay_below_one():
    """What the differences' tolerance takes for granted."""
    z = torch.linspace(-12, 12, 24001, dtype=torch.float64)
    for name in ("gelu", "gelu_tanh", "silu"):
        slope = O.act(name, z)[1]
        h = float(z[1] - z[0])
        assert float(((slope[2:] - 2 * slope[1:-1] + slope[:-2]) / h ** 2).abs().max()) < 1 - math.sqrt(h)
