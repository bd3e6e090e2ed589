"""dsm_linear and dsm_linear_backward on the GPU against 64-bit values, within a priori
bounds (block_oracle), over types, activations, sizes around every tile and step,
layouts and magnitudes; against differences; streams, graphs, refusals."""
import threading

import pytest

torch = pytest.importorskip("torch")

import block_oracle as O  # noqa: E402
from paper_2411_17866_amd import dsm  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
FEW = 64


def _ops():
    from paper_2411_17866_amd import ops
    return ops


def _inputs(tokens, dim, wide, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, sigma=1.0):
        return torch.empty(shape, device="cuda").normal_(0, sigma, generator=gen)

    return dict(x=normal(tokens, dim).to(dtype), w=normal(wide, dim, sigma=dim ** -0.5).to(dtype),
                bias=normal(wide, sigma=0.5), residual=normal(tokens, wide).to(dtype),
                dy=(normal(tokens, wide) * torch.exp(normal(tokens, 1))).to(dtype), z=normal(tokens, wide, sigma=1.5).to(dtype))


def _forward(i, name="none", bias=True, residual=True, **given):
    tokens, dim = i["x"].shape
    plan = _ops().Linear(tokens, dim, i["w"].shape[0], dtype=i["x"].dtype, act=name)
    b, r = (i["bias"] if bias else None), (i["residual"] if residual else None)
    out = plan(i["x"], i["w"], bias=b, residual=r, **given)
    e = O.linear(i["x"], i["w"], b, r, name)
    bounds = O.linear_bounds(i["x"], i["w"], b, r, name, tokens <= FEW)
    O.check(out, e, bounds, list(out))
    return out


def _backward(i, name="none", dw_dtype=None, **given):
    tokens, dim = i["x"].shape
    dtype = i["x"].dtype
    plan = _ops().Linear(tokens, dim, i["w"].shape[0], dtype=dtype, act=name, dw_dtype=dw_dtype)
    out = plan.backward(i["dy"], i["x"], i["w"], z=i["z"] if name != "none" else None, **given)
    e = O.linear_backward(i["dy"], i["x"], i["w"], i["z"], name)
    O.check(out, e, O.linear_backward_bounds(e, i["dy"], i["x"], i["w"], name, dw_dtype or dtype), list(out))
    return out


# One, odd sizes, and around runs of k (32, 64), fragments (16), few tokens (64), tiles (64, 128, 256).
SIZES = [(1, 1, 1), (1, 7, 3), (1, 768, 1000), (2, 64, 17), (3, 65, 16), (7, 31, 129), (15, 128, 33), (16, 100, 48), (17, 63, 64),
         (31, 257, 100), (33, 96, 255), (48, 1000, 15), (63, 64, 65), (50, 6400, 40), (3, 4097, 20), (64, 192, 31), (65, 64, 64), (66, 1, 9), (80, 72, 136),
         (127, 129, 130), (128, 128, 128), (129, 320, 384), (192, 64, 257), (255, 33, 65), (256, 256, 256), (257, 264, 520),
         (300, 1600, 48), (500, 24, 2000), (513, 512, 513), (1025, 40, 72)]


@TYPES
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward(size, dtype):
    k = sum(size)
    _forward(_inputs(*size, dtype, seed=k), O.ACTS[k % 5], bias=k % 4 != 0, residual=k % 3 != 0)


@TYPES
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_backward(size, dtype):
    k = sum(size)
    _backward(_inputs(*size, dtype, seed=k), O.ACTS[(k + 2) % 5], dw_dtype=F32 if k % 2 else None)


@TYPES
@pytest.mark.parametrize("name", O.ACTS)
@pytest.mark.parametrize("tokens", [5, 70])
def test_activations(tokens, name, dtype):
    i = _inputs(tokens, 40, 100, dtype, seed=3)
    # From far below to far above 0, and 0 itself.
    i["z"] = (torch.linspace(-60, 60, tokens * 100, device="cuda").view(tokens, 100) ** 3 / 1000).to(dtype)
    i["z"][0, :3] = torch.tensor([0.0, -0.0, 1e30], device="cuda", dtype=dtype)
    i["w"] *= 4
    out = _forward(i, name, residual=False)
    if name != "none":
        assert "z" in out
    _backward(i, name)


# Many entries: what roundings that are independent add up to.
LONG = [(2048, 1024, 1024), (4093, 1600, 640), (1024, 4100, 700), (70, 6400, 1600), (64, 6400, 1601), (8192, 72, 80), (700, 300, 9000)]


@TYPES
@pytest.mark.parametrize("size", LONG, ids=str)
def test_long_sums(size, dtype):
    tokens, dim, wide = size
    i = _inputs(*size, dtype, seed=7)
    plan = _ops().Linear(*size, dtype=dtype, act="gelu")
    y = plan(i["x"], i["w"], bias=i["bias"])["y"]
    e = O.linear(i["x"], i["w"], i["bias"], None, "gelu")
    O.check_norm(y, e["y"], O.norm_bound(dim, dtype), "y")
    out = plan.backward(i["dy"], i["x"], i["w"], z=i["z"])
    e = O.linear_backward(i["dy"], i["x"], i["w"], i["z"], "gelu")
    for name, terms in (("dx", wide), ("dw", tokens)):
        O.check_norm(out[name], e[name], O.norm_bound(terms, dtype, 2), name)
    O.check_norm(out["dbias"], e["dbias"], O.norm_bound(tokens, F32), "dbias")
    if dtype == BF16:  # dz as two halves: of 16 bits
        plan = _ops().Linear(*size, dtype=dtype, act="gelu", dw_dtype=F32)
        dw = plan.backward(i["dy"], i["x"], i["w"], z=i["z"], wanted=("dw",))["dw"]
        O.check_norm(dw, e["dw"], O.norm_bound(2 * tokens, F32) + 2.0 ** -16, "dw in fp32")


@TYPES
@pytest.mark.parametrize("tokens", [3, 64, 130, 192])
def test_strided_and_misaligned_views(tokens, dtype):
    dim, wide = 64, 192
    i = _inputs(tokens, dim, wide, dtype, seed=5)
    for pad, skip in ((8, 0), (3, 1), (64, 8)):
        def view(t):
            big = torch.full((t.shape[0] * (t.shape[1] + pad) + 16,), float("nan"), device="cuda", dtype=t.dtype)
            v = torch.as_strided(big[skip:], t.shape, (t.shape[1] + pad, 1))
            v.copy_(t)
            return v, big

        seen = {k: view(t) for k, t in i.items() if k != "bias"}
        j = dict({k: v for k, (v, _) in seen.items()}, bias=i["bias"])
        outs = {k: view(torch.zeros_like(i[like])) for k, like in (("y", "dy"), ("dx", "x"), ("dw", "w"))}
        _forward(j, "silu", y=outs["y"][0])
        _backward(j, "silu", dx=outs["dx"][0], dw=outs["dw"][0])
        _backward(j, "none")
        for v, big in list(seen.values()) + list(outs.values()):
            rest = torch.ones_like(big, dtype=torch.bool)
            torch.as_strided(rest[skip:], v.shape, v.stride()).fill_(False)
            assert torch.isnan(big[rest]).all()  # nothing between the rows was written


@TYPES
@pytest.mark.parametrize("tokens,dim,wide", [(66, 32, 40), (100, 96, 130), (114, 352, 17), (128, 160, 64), (100, 2528, 200), (40, 96, 64), (200, 96, 64)])
def test_rows_that_end_with_half_a_step(tokens, dim, wide, dtype):
    """Rows of 32 columns past the steps of 64, with nothing but NaN behind them."""
    i = _inputs(tokens, dim, wide, dtype, seed=6)
    big = {k: torch.full((i[k].shape[0], dim + 32), float("nan"), device="cuda", dtype=dtype) for k in "xw"}
    for k, t in big.items():
        t[:, :dim] = i[k]
        i[k] = t[:, :dim]
    _forward(i, "relu")
    _backward(i, "relu")
    _forward(dict(i, w=i["w"].contiguous()), bias=False)
    _forward(dict(i, x=i["x"].contiguous()), residual=False)


@TYPES
@pytest.mark.parametrize("tokens", [4, 200])
def test_onto_the_residual_in_place(tokens, dtype):
    i = _inputs(tokens, 96, 136, dtype, seed=6)
    apart = _forward(i)["y"]
    plan = _ops().Linear(tokens, 96, 136, dtype=dtype)
    r = i["residual"].clone()
    out = plan(i["x"], i["w"], bias=i["bias"], residual=r, y=r)
    assert out["y"] is r and torch.equal(r, apart)


@TYPES
def test_some_of_the_gradients(dtype):
    i = _inputs(200, 96, 136, dtype, seed=8)
    plan = _ops().Linear(200, 96, 136, dtype=dtype, act="relu")
    whole = plan.backward(i["dy"], i["x"], i["w"], z=i["z"])
    for wanted in (("dx",), ("dw",), ("dbias",), ("dx", "dbias"), ()):
        some = plan.backward(i["dy"], i["x"] if "dw" in wanted else None, i["w"] if "dx" in wanted else None, z=i["z"],
                             wanted=wanted)
        assert sorted(some) == sorted(wanted)
        for k in wanted:
            assert torch.equal(some[k], whole[k])


@TYPES
def test_no_tokens(dtype):
    plan = _ops().Linear(0, 40, 24, dtype=dtype, act="gelu")
    x, w = torch.empty(0, 40, device="cuda", dtype=dtype), torch.ones(24, 40, device="cuda", dtype=dtype)
    y = torch.empty(0, 24, device="cuda", dtype=dtype)
    assert plan(x, w)["y"].shape == (0, 24)
    out = plan.backward(y, x, w, z=y, dw=torch.full_like(w, 7), dbias=torch.full((24,), 7.0, device="cuda"))
    assert not out["dw"].any() and not out["dbias"].any() and out["dx"].shape == (0, 40)


def test_rows_of_very_different_sizes():
    """fp32 rows take powers of two of their own: each keeps its digits."""
    i = _inputs(200, 100, 140, F32, seed=9)
    size = torch.pow(2.0, torch.linspace(-90, 30, 200, device="cuda"))[:, None]
    i["x"] *= size
    i["w"] *= torch.pow(2.0, torch.linspace(20, -30, 140, device="cuda"))[:, None]
    i["residual"] *= 0
    i["bias"] *= 0
    out = _forward(i, "none")
    want = O.linear(i["x"], i["w"])["y"]
    for rows in (slice(0, 20), slice(90, 110), slice(180, 200)):
        O.check_norm(out["y"][rows, :20], want[rows, :20], O.norm_bound(100, F32), "large rows of w")
        O.check_norm(out["y"][rows, 120:], want[rows, 120:], O.norm_bound(100, F32), "small rows of w")
    # Tokens whose gradients are small meet their own rows in dx, and w as a whole.
    i = _inputs(200, 100, 140, F32, seed=10)
    i["dy"] *= size
    i["x"] /= size  # so that every token counts in dw
    got = _backward(i, "none")
    e = O.linear_backward(i["dy"], i["x"], i["w"])
    for rows in (slice(0, 20), slice(90, 110), slice(180, 200)):
        O.check_norm(got["dx"][rows], e["dx"][rows], O.norm_bound(140, F32), "dx")
    O.check_norm(got["dw"], e["dw"], O.norm_bound(200, F32), "dw")


@TYPES
@pytest.mark.parametrize("tokens", [20, 150])
def test_zeros(tokens, dtype):
    i = _inputs(tokens, 70, 90, dtype, seed=11)
    i["x"][3] = 0
    i["w"][5] = 0
    i["dy"][7] = 0
    i["x"] *= 1e5 if dtype == F32 else 1
    _forward(i)
    _backward(i)
    i["dy"].zero_()
    out = _backward(i)
    assert all(not v.any() for v in out.values())
    i["w"].zero_()
    i["x"].zero_()
    _forward(i)
    _backward(i)


@TYPES
@pytest.mark.parametrize("tokens", [5, 40, 100, 200])
def test_operands_below_the_normal_numbers(tokens, dtype):
    """Operands of 2^-130 and large ones make ordinary products: none of them is taken as 0."""
    i = _inputs(tokens, 70, 90, dtype, seed=11)
    i["x"] = (i["x"].double() * 2.0 ** -130).to(dtype)
    i["w"] = (i["w"].double() * 2.0 ** 60).to(dtype)
    plan = _ops().Linear(tokens, 70, 90, dtype=dtype)
    y = plan(i["x"], i["w"])["y"]
    e = O.linear(i["x"], i["w"], None, None)
    O.check_norm(y, e["y"], O.norm_bound(70, dtype), "y")
    i["dy"] = (i["dy"].double() * 2.0 ** 80).to(dtype)
    dw = plan.backward(i["dy"], i["x"], i["w"], wanted=("dw",))["dw"]
    e = O.linear_backward(i["dy"], i["x"], i["w"])
    O.check_norm(dw, e["dw"], O.norm_bound(tokens, dtype), "dw")
    i["dy"] = (i["dy"].double() * 2.0 ** -210).to(dtype)
    dx = plan.backward(i["dy"], i["x"], i["w"], wanted=("dx",))["dx"]
    e = O.linear_backward(i["dy"], i["x"], i["w"])
    O.check_norm(dx, e["dx"], O.norm_bound(90, dtype), "dx")


@TYPES
@pytest.mark.parametrize("tokens", [20, 150])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_non_finite_values_reach_what_depends_on_them_alone(tokens, bad, dtype):
    i = _inputs(tokens, 70, 90, dtype, seed=12)
    i["x"][3, 4] = bad
    i["w"][5, 6] = bad
    plan = _ops().Linear(tokens, 70, 90, dtype=dtype)
    y = plan(i["x"], i["w"], bias=i["bias"])["y"]
    hit = torch.zeros_like(y, dtype=torch.bool)
    hit[3] = True
    hit[:, 5] = True
    assert (torch.isfinite(y) == ~hit).all()
    i = _inputs(tokens, 70, 90, dtype, seed=12)
    i["dy"][3, 4] = bad
    out = plan.backward(i["dy"], i["x"], i["w"])
    assert (torch.isfinite(out["dx"]).all(1) == (torch.arange(tokens, device="cuda") != 3)).all()
    assert (torch.isfinite(out["dw"]).all(1) == (torch.arange(90, device="cuda") != 4)).all()
    assert (torch.isfinite(out["dbias"]) == (torch.arange(90, device="cuda") != 4)).all()


@pytest.mark.parametrize("name", O.ACTS)
def test_gradients_against_differences(name):
    i = _inputs(150, 40, 50, F32, seed=13)
    plan = _ops().Linear(150, 40, 50, act=name)
    if name == "relu":  # away from the kink, over which a difference is no derivative
        i["bias"] = torch.where(torch.arange(50, device="cuda") % 2 == 0, 9.0, -9.0)
    z = plan(i["x"], i["w"], bias=i["bias"], z=torch.empty_like(i["z"]))["z"]
    out = plan.backward(i["dy"], i["x"], i["w"], z=z if name != "none" else None)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for key, grad in (("x", "dx"), ("w", "dw"), ("bias", "dbias")):
        v = torch.empty_like(i[key]).normal_(0, 1, generator=gen)
        step = 2.0 ** -6

        def total(sign):
            y = plan(**{k: i[k] + (sign * step * v if k == key else 0) for k in ("x", "w", "bias")})["y"]
            return float((y.double() * i["dy"].double()).sum())

        want = (total(1) - total(-1)) / (2 * step)
        got = float((out[grad].double() * v.double()).sum())
        # The third derivative's term, step^2 |v x|^3 / 6 a row at most, and y's roundings over the step.
        scale = float(i["dy"].double().norm() * (v.double().norm() * (6 if key != "bias" else 1)))
        assert abs(got - want) <= 2e-3 * scale, (key, got, want)


@TYPES
@pytest.mark.parametrize("size", [(1, 768, 1600), (33, 200, 100), (300, 257, 1000), (2000, 64, 80)], ids=str)
def test_reruns_give_the_same_bits(size, dtype):
    i = _inputs(*size, dtype, seed=14)
    plan = _ops().Linear(*size, dtype=dtype, act="gelu_tanh")

    def run():
        out = plan(i["x"], i["w"], bias=i["bias"], residual=i["residual"])
        return dict(out, **plan.backward(i["dy"], i["x"], i["w"], z=i["z"]))

    first = run()
    plan.workspace.fill_(255)
    again = run()
    assert all(torch.equal(first[k], again[k]) for k in first)


@TYPES
@pytest.mark.parametrize("tokens", [1, 200])
def test_graphs_replay(tokens, dtype):
    """Captured beside an eager autograd graph of the same tensors; replayed with eager work between."""
    dim, wide = 96, 136
    i = _inputs(tokens, dim, wide, dtype, seed=15)
    plan = _ops().Linear(tokens, dim, wide, dtype=dtype, act="silu")
    leaf = i["w"].detach().requires_grad_()
    alive = (i["x"].float().clone() @ leaf.float().t()).square().mean()

    def run(out=None):
        given = {} if out is None else dict(y=out["y"], z=out["z"])
        f = plan(i["x"], i["w"], bias=i["bias"], residual=i["residual"], **given)
        given = {} if out is None else {k: out[k] for k in ("dx", "dw", "dbias")}
        return dict(f, **plan.backward(i["dy"], i["x"], i["w"], z=f["z"], **given))

    out = run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out)
    for seed in (20, 21, 22):
        for k, t in _inputs(tokens, dim, wide, dtype, seed=seed).items():
            i[k].copy_(t)
        want = {k: t.clone() for k, t in run().items()}
        for t in out.values():
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[k]) for k in want)
    alive.backward()
    assert torch.isfinite(leaf.grad).all()


def test_streams_and_threads():
    i = _inputs(200, 96, 136, BF16, seed=16)
    plan = _ops().Linear(200, 96, 136, dtype=BF16, act="gelu")

    def run():
        f = plan(i["x"], i["w"], bias=i["bias"])
        return dict(f, **plan.backward(i["dy"], i["x"], i["w"], z=i["z"]))

    want = run()
    torch.cuda.synchronize()
    bad = []

    def work():
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got = run()
                stream.synchronize()
                bad.extend(k for k in want if not torch.equal(got[k], want[k]))

    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_refusals():
    ops = _ops()
    i = _inputs(70, 40, 24, BF16)
    plan = ops.Linear(70, 40, 24, dtype=BF16, act="relu")
    for make in (lambda: ops.Linear(70, 40, 24, dtype=torch.float16), lambda: ops.Linear(70, 40, 24, act="tanh"),
                 lambda: ops.Linear(70, 40, 24, dw_dtype=BF16), lambda: ops.Linear(70, 0, 24),
                 lambda: ops.Linear(70, 40, 24, device="cpu")):
        with pytest.raises((ValueError, dsm.DsmError)):
            make()
    for call in (lambda: plan(i["x"].float(), i["w"]), lambda: plan(i["x"][:, :39], i["w"]), lambda: plan(i["x"].cpu(), i["w"]),
                 lambda: plan(i["x"], i["w"].t().contiguous().t()), lambda: plan(i["x"], i["w"], bias=i["bias"].to(BF16)),
                 lambda: plan(i["x"], i["w"], y=torch.empty(70, 24, device="cuda")),
                 lambda: plan(i["x"], i["w"], residual=i["residual"][:1].expand(70, 24)),
                 lambda: plan.backward(i["dy"], i["x"], i["w"]), lambda: plan.backward(i["dy"], None, i["w"], z=i["z"]),
                 lambda: plan.backward(i["dy"], i["x"], i["w"], z=i["z"], dx=i["x"]),
                 lambda: plan.backward(i["dy"], i["x"], i["w"], z=i["z"], wanted=("dz",)),
                 lambda: plan.backward(i["dy"], i["x"], i["w"], z=i["z"], dw=i["w"].clone(), wanted=("dx",)),
                 lambda: ops.Linear(70, 40, 24, dtype=BF16, grads=False).backward(i["dy"], i["x"], i["w"])):
        with pytest.raises((ValueError, dsm.DsmError)):
            call()
