"""The 64-bit values of the blocks' operators (block_oracle) against torch's own
derivatives in float64, on the CPU, and mistakes planted in copies of them, which their
bounds have to notice."""
import inspect

import pytest

torch = pytest.importorskip("torch")

import block_oracle as O  # noqa: E402


def _gen(seed=0):
    return torch.Generator().manual_seed(seed)


def _normal(*shape, seed=0):
    return torch.randn(*shape, generator=_gen(seed), dtype=torch.float64)


@pytest.mark.parametrize("name", O.ACTS)
def test_linear_gradients_are_those_of_its_values(name):
    x, w, b = (_normal(*s, seed=i).requires_grad_() for i, s in enumerate([(5, 7), (6, 7), (6,)]))
    dy = _normal(5, 6, seed=9)
    e = O.linear(x, w, b, None, name)
    e["y"].backward(dy)
    got = O.linear_backward(dy, x.detach(), w.detach(), e["z"].detach(), name)
    for grad, name_ in ((x.grad, "dx"), (w.grad, "dw"), (b.grad, "dbias")):
        assert torch.allclose(grad, got[name_], rtol=1e-10, atol=1e-12)


@pytest.mark.parametrize("post", ["none", "layer", "rms"])
@pytest.mark.parametrize("norm", ["none", "layer", "rms"])
def test_norm_gradients_are_those_of_its_values(norm, post):
    T, D = 4, 9
    rows = {n: _normal(T, D, seed=i).requires_grad_() for i, n in enumerate(("h", "f"))}
    vectors = {n: _normal(D, seed=20 + i).requires_grad_() for i, n in
               enumerate(("weight", "bias", "gate", "post_weight", "post_bias"))}
    kinds = dict(norm=norm, post=post, scale=0.7)

    def forward(h, f):  # without the bounds, whose types are torch's
        p = f
        if post != "none":
            p = O.standard(post, f, 1e-5)[0] * vectors["post_weight"] + vectors["post_bias"]
        s = h + 0.7 * vectors["gate"] * p
        return s, None if norm == "none" else O.standard(norm, s, 1e-5)[0] * vectors["weight"] + vectors["bias"]

    s, y = forward(**rows)
    dy, ds = _normal(T, D, seed=40), _normal(T, D, seed=41)
    total = (s * ds).sum() + (0 if y is None else (y * dy).sum())
    total.backward()
    given = {n: v.detach() for n, v in vectors.items()
             if (norm != "none" or n not in ("weight", "bias")) and (post != "none" or not n.startswith("post"))}
    O.HALF[torch.float64] = 2.0 ** -53
    try:
        got = O.residual_norm_backward(None if norm == "none" else dy, s.detach(), rows["f"].detach(), ds, **given, **kinds)
        e = O.residual_norm(rows["h"].detach(), rows["f"].detach(), **given, **kinds)
    finally:
        del O.HALF[torch.float64]
    assert torch.allclose(e["s"], s.detach()) and (y is None or torch.allclose(e["y"], y.detach()))
    assert torch.allclose(got["dh"], rows["h"].grad, rtol=1e-9, atol=1e-11)
    assert torch.allclose(got["df"], rows["f"].grad, rtol=1e-9, atol=1e-11)
    for n in given:
        assert torch.allclose(got["d" + n], vectors[n].grad, rtol=1e-9, atol=1e-11), n


def test_clip_values():
    ts = [_normal(3, 4), _normal(5, seed=1), _normal(2, seed=2)]
    norms, out = O.clip(ts, [0, 1, 0], 1.0)
    whole = torch.cat([ts[0].flatten(), ts[2]]).norm()
    assert abs(norms[0] - float(whole)) < 1e-12 and abs(norms[1] - float(ts[1].norm())) < 1e-12
    assert torch.allclose(out[0], ts[0] / (whole + 1e-6)) and torch.allclose(out[1], ts[1] / (ts[1].norm() + 1e-6))
    assert O.clip(ts, [0, 0, 0], 1e9)[1][1].equal(ts[1])


# (function, what, instead): each has to leave the true values' bounds.
PLANTED = [("back", "(d * hat).mean(1, keepdim=True)", "0 * d"),
           ("back", "d - d.mean(1, keepdim=True) if", "d if"),
           ("standard", "v.square().mean", "1.001 * v.square().mean"),
           ("act", "1 + 3 * b * z * z", "1 + b * z * z"),
           ("act", "share + z * share * torch.sigmoid(-z)", "share + z * share")]


@pytest.mark.parametrize("planted", PLANTED, ids=lambda p: p[1][:24])
def test_planted_mistakes_leave_the_bounds(planted):
    function, what, instead = planted
    source = inspect.getsource(O)
    assert what in inspect.getsource(getattr(O, function))
    wrong = {}
    exec(compile(source.replace(what, instead), "planted", "exec"), wrong)
    T, D = 6, 80
    dy, s, f, ds = (_normal(T, D, seed=i).float() for i in range(4))
    w, z = _normal(D, D, seed=5).float(), _normal(T, D, seed=6).float()
    missed = True
    for kinds in (dict(norm="layer", post="rms"), dict(norm="rms", post="layer")):
        true, false = (m.residual_norm_backward(dy, s, f, ds, weight=w[0], **kinds) if m is O else
                       m["residual_norm_backward"](dy, s, f, ds, weight=w[0], **kinds) for m in (O, wrong))
        missed = missed and all(((true[n] - false[n]).abs() <= true[n + "_bound"]).all() for n in ("dh", "df", "dweight"))
    for name in O.ACTS:
        true, false = O.linear_backward(dy, s, w, z, name), wrong["linear_backward"](dy, s, w, z, name)
        bounds = O.linear_backward_bounds(true, dy, s, w, name, torch.float32)
        missed = missed and all(((true[n] - false[n]).abs() <= bounds[n]).all() for n in ("dx", "dw", "dbias"))
    assert not missed
