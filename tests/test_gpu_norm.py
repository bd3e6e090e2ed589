"""dsm_residual_norm and its gradients on the GPU against 64-bit values, within a priori
bounds (block_oracle), over types, kinds of norms, widths, layouts; against
differences; in place, streams, graphs, refusals."""
import itertools
import threading

import pytest

torch = pytest.importorskip("torch")

import block_oracle as O  # noqa: E402
from paper_2411_17866_amd import dsm  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
VECTORS = ("weight", "bias", "gate", "post_weight", "post_bias")


def _ops():
    from paper_2411_17866_amd import ops
    return ops


def _inputs(tokens, dim, dtype, seed=0, mean=0.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, sigma=1.0, mean=0.0):
        return torch.empty(shape, device="cuda").normal_(mean, sigma, generator=gen)

    rows = {k: normal(tokens, dim, mean=mean if k in "hf" else 0.0).to(dtype) for k in ("h", "f", "dy", "ds")}
    return dict(rows, **{k: normal(dim, mean=0.3) for k in VECTORS})


def _given(i, norm, post, branch=True, without=()):
    return {k: i[k] for k in VECTORS if k not in without and (branch or k in ("weight", "bias")) and
            (norm != "none" or k not in ("weight", "bias")) and (post != "none" or not k.startswith("post"))}


def _run(i, norm="layer", post="none", branch=True, scale=0.7, without=(), eps=1e-5, post_eps=1e-3, ds=True, forward={}, backward={}):
    tokens, dim = i["h"].shape
    plan = _ops().ResidualNorm(tokens, dim, dtype=i["h"].dtype, norm=norm, post=post, eps=eps, post_eps=post_eps)
    vectors, kinds = _given(i, norm, post, branch, without), dict(norm=norm, post=post, eps=eps, post_eps=post_eps)
    f = i["f"] if branch else None
    scale = scale if branch else 1.0
    e = O.residual_norm(i["h"], f, scale=scale, **vectors, **kinds)
    s_in, f_in = i["h"].clone(), None if f is None else f.clone()
    out = plan(i["h"], f=f, scale=scale, **vectors, **forward)
    names = (["s"] if branch else []) + (["y"] if norm != "none" else [])
    assert sorted(out) == sorted(names)
    O.check(out, e, {n: e[n + "_bound"] for n in names}, names)
    ds = i["ds"] if ds or norm == "none" else None
    dy = i["dy"] if norm != "none" else None
    e = O.residual_norm_backward(dy, s_in, f_in, ds, scale=scale, **vectors, **kinds)
    got = plan.backward(dy, s_in, f=f_in, ds=ds, scale=scale, **vectors, **backward)
    names = [n for n in e if not n.endswith("_bound")]
    assert sorted(got) == sorted(names)
    O.check(got, e, {n: e[n + "_bound"] for n in names}, names)
    return dict(out, **got)


# Widths around 8 columns a lane and 1 to 16 waves; tokens around the rows of a work-group.
SIZES = [(1, 1), (1, 2), (1, 1600), (2, 7), (3, 8), (2, 9), (5, 63), (4, 511), (3, 512), (6, 513), (5, 1030), (7, 768), (9, 1000), (3, 1024), (2, 1025),
         (11, 1601), (4, 2048), (3, 2049), (5, 4096), (3, 4097), (2, 6400), (3, 8191), (2, 8192), (1, 8185), (333, 100), (1000, 48)]


@TYPES
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_sizes(size, dtype):
    k = sum(size)
    _run(_inputs(*size, dtype, seed=k), norm=("layer", "rms")[k % 2], post=("none", "layer", "rms")[k % 3],
         without=("gate",) if k % 4 == 0 else ())


@TYPES
@pytest.mark.parametrize("norm,post", itertools.product(("none", "layer", "rms"), repeat=2))
def test_kinds(norm, post, dtype):
    i = _inputs(37, 300, dtype, seed=1)
    _run(i, norm, post)
    _run(i, norm, post, without=VECTORS, ds=False)
    _run(i, norm, post, without=("bias", "post_weight", "gate"))
    if post == "none" and norm != "none":
        _run(i, norm, branch=False)
        _run(i, norm, branch=False, ds=False, without=("bias",))


@TYPES
@pytest.mark.parametrize("tokens,dim", [(5000, 96), (4097, 1280), (700, 5000)])
def test_many_rows(tokens, dim, dtype):
    """More rows than the work-groups take in one turn."""
    _run(_inputs(tokens, dim, dtype, seed=2), norm="layer", post="rms")


@TYPES
def test_a_mean_far_from_zero(dtype):
    _run(_inputs(50, 700, dtype, seed=3, mean=100.0), norm="layer", post="layer")


@TYPES
@pytest.mark.parametrize("dim", [64, 333])
def test_strided_views(dim, dtype):
    i = _inputs(40, dim, dtype, seed=4)
    want = _run(i, "layer", "rms")
    for pad, skip in ((8, 0), (3, 1)):
        def view(t):
            big = torch.full((40 * (dim + pad) + 16,), float("nan"), device="cuda", dtype=dtype)
            v = torch.as_strided(big[skip:], t.shape, (dim + pad, 1))
            v.copy_(t)
            return v, big

        seen = {k: view(i[k]) for k in ("h", "f", "dy", "ds")}
        outs = {k: view(i["h"]) for k in ("s", "y", "dh", "df")}
        j = dict(i, **{k: v for k, (v, _) in seen.items()})
        got = _run(j, "layer", "rms", forward={k: outs[k][0] for k in ("s", "y")}, backward={k: outs[k][0] for k in ("dh", "df")})
        assert all(torch.equal(got[k], want[k]) for k in want)
        for v, big in list(seen.values()) + list(outs.values()):
            rest = torch.ones_like(big, dtype=torch.bool)
            torch.as_strided(rest[skip:], v.shape, v.stride()).fill_(False)
            assert torch.isnan(big[rest]).all()


@TYPES
@pytest.mark.parametrize("post", ["none", "layer"])
@pytest.mark.parametrize("dim", [200, 203, 513, 1029])  # rows that end within a lane's columns, and in a wave's first lane
def test_in_place(dim, post, dtype):
    i = _inputs(77, dim, dtype, seed=5)
    want = _run(i, "layer", post)
    vectors = _given(i, "layer", post)
    plan = _ops().ResidualNorm(77, dim, dtype=dtype, norm="layer", post=post, post_eps=1e-3)
    for s_at, y_at in (("h", "f"), ("f", "h")):
        rows = {k: i[k].clone() for k in ("h", "f")}
        out = plan(rows["h"], f=rows["f"], scale=0.7, s=rows[s_at], y=rows[y_at], **vectors)
        assert out["s"] is rows[s_at] and torch.equal(out["s"], want["s"]) and torch.equal(out["y"], want["y"])
    for dh_at, df_at in (("dy", "ds"), ("ds", "dy"), ("ds", "f")):
        rows = {k: i[k].clone() for k in ("h", "f", "dy", "ds")}
        out = plan.backward(rows["dy"], rows["h"], f=rows["f"], ds=rows["ds"], scale=0.7, dh=rows[dh_at], df=rows[df_at], **vectors)
        assert all(torch.equal(out[k], want[k]) for k in out)


@TYPES
def test_no_tokens(dtype):
    plan = _ops().ResidualNorm(0, 100, dtype=dtype, post="rms")
    e = torch.empty(0, 100, device="cuda", dtype=dtype)
    v = torch.ones(100, device="cuda")
    assert plan(e, f=e, weight=v)["y"].shape == (0, 100)
    out = plan.backward(e, e, f=e, weight=v, bias=v, gate=v, post_weight=v, dgate=torch.full((100,), 7.0, device="cuda"))
    assert all(not out[k].any() for k in ("dweight", "dbias", "dgate", "dpost_weight"))


@TYPES
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_non_finite_rows_stay_their_own(bad, dtype):
    i = _inputs(9, 100, dtype, seed=6)
    i["h"][4, 50] = bad
    plan = _ops().ResidualNorm(9, 100, dtype=dtype)
    out = plan(i["h"], f=i["f"], weight=i["weight"], bias=i["bias"])
    got = plan.backward(i["dy"], i["h"], f=i["f"], ds=i["ds"], weight=i["weight"], bias=i["bias"])
    other = torch.arange(9, device="cuda") != 4
    for t in (out["s"], out["y"], got["dh"]):
        assert (torch.isfinite(t).all(1) == other).all()
    assert torch.isfinite(got["dbias"]).all() and not torch.isfinite(got["dweight"]).all()


def test_rows_that_are_constant_or_zero():
    i = _inputs(6, 100, F32, seed=7)
    i["h"][2] = 0
    i["f"][2] = 0
    i["h"][4] = 3.0
    i["f"][4] = 0
    _run(i, "layer", "none")
    i["f"][2] = 0
    _run(i, "rms", "rms", eps=1e-3)


def test_gradients_against_differences():
    i = _inputs(20, 60, F32, seed=8)
    plan = _ops().ResidualNorm(20, 60, norm="layer", post="rms")
    args = {k: i[k] for k in ("h", "f", *VECTORS)}
    s = plan(**args, scale=0.5)["s"]
    out = plan.backward(i["dy"], s, f=i["f"], ds=i["ds"], scale=0.5, **{k: i[k] for k in VECTORS})
    gen = torch.Generator(device="cuda").manual_seed(1)
    for key in args:
        v = torch.empty_like(args[key]).normal_(0, 1, generator=gen)
        step = 2.0 ** -7

        def total(sign):
            o = plan(**{k: t + (sign * step * v if k == key else 0) for k, t in args.items()}, scale=0.5)
            return float((o["y"].double() * i["dy"].double()).sum() + (o["s"].double() * i["ds"].double()).sum())

        want = (total(1) - total(-1)) / (2 * step)
        got = float((out["d" + key].double() * v.double()).sum())
        # step^2 times the third derivative (some units), and 1200 roundings of 2^-23 over the step.
        scale = float((i["dy"].double().norm() + i["ds"].double().norm()) * v.double().norm())
        assert abs(got - want) <= 1e-3 * scale, (key, got, want)


@TYPES
def test_graphs_replay(dtype):
    i = _inputs(300, 200, dtype, seed=9)
    plan = _ops().ResidualNorm(300, 200, dtype=dtype, norm="layer", post="rms")
    vectors = _given(i, "layer", "rms")
    leaf = i["weight"].detach().requires_grad_()
    alive = (i["h"].float().clone() * leaf).square().mean()

    def run(out=None):
        pick = (lambda *names: {}) if out is None else (lambda *names: {k: out[k] for k in names})
        f = plan(i["h"], f=i["f"], **vectors, **pick("s", "y"))
        return dict(f, **plan.backward(i["dy"], f["s"], f=i["f"], ds=i["ds"], **vectors,
                                       **pick("dh", "df", *("d" + k for k in vectors))))

    out = run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out)
    for seed in (20, 21, 22):
        for k, t in _inputs(300, 200, dtype, seed=seed).items():
            i[k].copy_(t)
        want = {k: t.clone() for k, t in run().items()}
        for t in out.values():
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[k]) for k in want)
    alive.backward()


def test_streams_and_threads():
    i = _inputs(500, 300, BF16, seed=10)
    plan = _ops().ResidualNorm(500, 300, dtype=BF16, norm="layer", post="rms")
    vectors = _given(i, "layer", "rms")
    want = plan.backward(i["dy"], i["h"], f=i["f"], ds=i["ds"], **vectors)
    torch.cuda.synchronize()
    bad = []

    def work():
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got = plan.backward(i["dy"], i["h"], f=i["f"], ds=i["ds"], **vectors)
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
    i = _inputs(5, 40, F32)
    plan = ops.ResidualNorm(5, 40, norm="layer")
    none = ops.ResidualNorm(5, 40, norm="none", post="rms")
    for make in (lambda: ops.ResidualNorm(5, 8193), lambda: ops.ResidualNorm(5, 40, norm="batch"), lambda: ops.ResidualNorm(-1, 40),
                 lambda: ops.ResidualNorm(5, 40, eps=-1.0), lambda: ops.ResidualNorm(5, 40, eps=float("nan"))):
        with pytest.raises((ValueError, dsm.DsmError)):
            make()
    for call in (lambda: plan(i["h"].to(BF16)), lambda: plan(i["h"], gate=i["gate"]), lambda: plan(i["h"], f=i["f"], post_weight=i["gate"]),
                 lambda: plan(i["h"], weight=i["weight"][:39]), lambda: plan(i["h"], weight=i["weight"].to(BF16)),
                 lambda: plan(i["h"], s=i["f"]), lambda: none(i["h"]), lambda: none(i["h"], f=i["f"], weight=i["weight"]),
                 lambda: plan(i["h"], f=i["f"], s=i["ds"], y=i["ds"]), lambda: plan(i["h"], f=i["f"], scale=float("inf")),
                 lambda: plan.backward(None, i["h"]), lambda: none.backward(i["dy"], i["h"], f=i["f"], ds=i["ds"]),
                 lambda: none.backward(None, None, f=i["f"]), lambda: plan.backward(i["dy"], i["h"], dgate=i["gate"]),
                 lambda: plan.backward(i["dy"], i["h"], f=i["f"], dh=i["ds"], df=i["ds"]),
                 lambda: ops.ResidualNorm(5, 40, grads=False).backward(i["dy"], i["h"])):
        with pytest.raises((ValueError, dsm.DsmError)):
            call()
