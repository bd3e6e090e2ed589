"""dsm_linear_ce on the GPU against 64-bit values, within a priori bounds
(ops_oracle), over types, sizes around every tile and step, layouts, masks and
non-finite inputs; its gradients against differences; reruns, streams, graphs."""
import pytest

torch = pytest.importorskip("torch")

import ops_oracle as O  # noqa: E402
from paper_2411_17866_amd import dsm  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _ops():
    from paper_2411_17866_amd import ops
    return ops


def _problem(tokens, dim, vocab, dtype, seed=0, ignored=0.2, spread=1.0, lean=4.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.empty(tokens, dim, device="cuda").normal_(0, 1, generator=gen)
    w = torch.empty(vocab, dim, device="cuda").normal_(0, spread / dim ** 0.5, generator=gen)
    t = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen)
    h += lean * torch.rand(tokens, 1, device="cuda", generator=gen) * w[t] / w[t].square().sum(1, keepdim=True)
    t[torch.rand(tokens, device="cuda", generator=gen) < ignored] = -100
    weight = torch.rand(tokens, device="cuda", generator=gen)
    return h.to(dtype), w.to(dtype), t, weight


def _carried(dtype, tokens, grads):
    """What operands and G carry (relative), by the types and tokens at which the
    library changes its form; the loosest where a neighbouring form would do too."""
    if dtype == BF16:
        return 0.0, O.U_HALF if tokens > 128 else O.U_BF16_HALVES
    return (0.0, 0.0) if tokens <= 64 else (O.U_HALVES, O.U_HALVES)


def _check(out, e, bounds, names):
    for name in names:
        got, want = out[name].double(), e[name]
        assert got.shape == want.shape
        assert torch.isfinite(got).all(), name
        far = (got - want).abs() - bounds[name]
        assert (far <= 0).all(), f"{name}: {int((far > 0).sum())} of {far.numel()} outside, by {float(far.max()):.3g}"


def _run_and_check(h, w, t, weight, mean, grads):
    ops = _ops()
    tokens, dim = h.shape
    plan = ops.LinearCE(tokens, dim, w.shape[0], dtype=h.dtype, grads=grads)
    lse = torch.empty(tokens, device="cuda")
    out = plan(h, w, t, weight=weight, mean=mean, lse=lse)
    e = O.linear_ce(h, w, t, weight=weight, mean=mean)
    bounds = O.linear_ce_bounds(e, h.dtype, *_carried(h.dtype, tokens, grads))
    _check(out, e, bounds, ("total", "loss") + (("dh", "dw") if grads else ()))
    valid = e["valid"]
    assert ((lse.double() - e["lse"]).abs()[valid] <= bounds["loss"][valid]).all()
    return out


# Around the tiles (32, 64, 128, 256 tokens; 128, 256 words) and the steps of k (32,
# 64), sizes of one, odd sizes, and the changes of form at 64 and 128 tokens.
SIZES = [(1, 1, 1), (1, 1, 2), (1, 64, 1), (2, 5, 3), (1, 768, 1000), (5, 100, 257), (31, 64, 128), (32, 96, 129),
         (33, 33, 127), (63, 128, 255), (64, 65, 256), (65, 64, 257), (100, 321, 1009), (127, 128, 130),
         (128, 31, 500), (129, 200, 384), (255, 64, 129), (256, 100, 1000), (257, 320, 385), (300, 1, 77),
         (511, 72, 640), (513, 128, 1025), (700, 36, 130), (1030, 192, 2000), (2100, 64, 9000)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_values_and_gradients(size, dtype):
    tokens, dim, vocab = size
    h, w, t, weight = _problem(*size, dtype, seed=tokens + dim)
    _run_and_check(h, w, t, weight if tokens % 2 else None, tokens % 3 == 0, True)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES[::2], ids=str)
def test_losses_alone(size, dtype):
    h, w, t, weight = _problem(*size, dtype, seed=size[0])
    _run_and_check(h, w, t, weight, size[0] % 2 == 0, False)


@pytest.mark.parametrize("times", [1, 2])  # G in one piece of at most 1 GiB, and in two
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_several_pieces_of_the_vocabulary(dtype, times):
    tokens, dim, vocab = times * (4200 if dtype == BF16 else 2100), 64, 70001
    h, w, t, weight = _problem(tokens, dim, vocab, dtype, seed=3)
    ops = _ops()
    out = ops.LinearCE(tokens, dim, vocab, dtype=dtype)(h, w, t, weight=weight)
    rows = torch.arange(0, tokens, 97, device="cuda")
    words = torch.cat([torch.arange(0, vocab, 1511, device="cuda"), torch.arange(vocab - 300, vocab, device="cuda")])
    e = O.linear_ce(h[rows], w, t[rows], weight=weight[rows], mean=False)
    n = int(((t >= 0) & (t < vocab)).sum())
    u_op, u_g = _carried(dtype, tokens, True)
    e["dh"], e["g"], e["c"] = e["dh"] / n, e["g"] / n, e["c"] / n
    bounds = O.linear_ce_bounds(e, dtype, u_op, u_g)
    _check({"loss": out["loss"][rows], "dh": out["dh"][rows]}, e, bounds, ("loss", "dh"))
    # dw of some words, over all tokens: the bound of a sum of T terms of G h.
    lse = torch.cat([torch.logsumexp(h[i:i + 256].double() @ w.double().t(), 1) for i in range(0, tokens, 256)])
    valid = (t >= 0) & (t < vocab)
    c = torch.where(valid, weight.double() / n, 0.0)
    g = torch.exp(h.double() @ w[words].double().t() - lse[:, None]) - (t[:, None] == words[None, :]).double()
    g *= c[:, None]
    want = g.t() @ h.double()
    size = (g.abs() + c[:, None] * 2.0 ** -9).t() @ h.double().abs()
    far = (out["dw"][words].double() - want).abs()
    assert (far <= (2 * u_g + 2 * u_op + tokens * 2.0 ** -23 + 1e-5) * size + O.U_OUT[dtype] * want.abs()).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("tokens", [3, 70, 600])
def test_strided_and_misaligned_views(tokens, dtype):
    dim, vocab = 64, 300
    h, w, t, weight = _problem(tokens, dim, vocab, dtype, seed=5)
    for pad, skip in ((8, 0), (3, 1), (72, 8)):
        def view(x):
            big = torch.full((x.shape[0], dim + pad), float("nan"), device="cuda", dtype=dtype).flatten()
            big = torch.cat([big, big.new_full((16,), float("nan"))])[skip:]
            v = torch.as_strided(big, x.shape, (dim + pad, 1))
            v.copy_(x)
            return v, big

        (hv, _), (wv, _), (dh, dh_all), (dw, dw_all) = view(h), view(w), view(h), view(w)
        plan = _ops().LinearCE(tokens, dim, vocab, dtype=dtype)
        out = plan(hv, wv, t, weight=weight, dh=dh, dw=dw)
        assert out["dh"] is dh and out["dw"] is dw
        e = O.linear_ce(h, w, t, weight=weight)
        bounds = O.linear_ce_bounds(e, dtype, *_carried(dtype, tokens, True))
        _check(out, e, bounds, ("total", "loss", "dh", "dw"))
        # Nothing between the rows was written.
        for x, whole in ((h, dh_all), (w, dw_all)):
            rest = torch.ones_like(whole, dtype=torch.bool)
            torch.as_strided(rest, x.shape, (dim + pad, 1)).fill_(False)
            assert torch.isnan(whole[rest]).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("tokens", [4, 90, 600])
def test_tokens_left_out_touch_nothing(tokens, dtype):
    dim, vocab = 96, 200
    h, w, t, weight = _problem(tokens, dim, vocab, dtype, seed=6, ignored=0.0)
    out_of = torch.tensor([-1, vocab, -100, 2 ** 40, -2 ** 62], device="cuda")
    for k in range(0, tokens, 3):
        t[k] = out_of[(k // 3) % len(out_of)]
    clean = _ops().LinearCE(tokens, dim, vocab, dtype=dtype)(h, w, t, weight=weight)
    clean = {k: v.clone() for k, v in clean.items()}
    dirty_h, dirty_w = h.clone(), weight.clone()
    dirty_h[::3] = float("nan")
    dirty_h[::6, 0] = float("inf")
    dirty_w[::3] = float("nan")
    for grads in (True, False):
        out = _ops().LinearCE(tokens, dim, vocab, dtype=dtype, grads=grads)(dirty_h, w, t, weight=dirty_w)
        for name in out:
            if grads:
                assert torch.equal(out[name], clean[name]), name
            else:
                assert torch.isfinite(out[name]).all()
    assert (clean["loss"][::3] == 0).all() and (clean["dh"][::3] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("tokens", [0, 1, 40, 300, 600])
def test_no_token_left(tokens, dtype):
    dim, vocab = 72, 150
    h, w, t, weight = _problem(tokens, dim, vocab, dtype, seed=7)
    t.fill_(-1)
    plan = _ops().LinearCE(tokens, dim, vocab, dtype=dtype)
    dw = torch.full((vocab, dim), float("nan"), device="cuda", dtype=dtype)
    out = plan(h, w, t, weight=weight, dw=dw)
    assert float(out["total"]) == 0
    for name in ("loss", "dh", "dw"):
        assert (out[name] == 0).all(), name


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("tokens", [5, 200, 600])
def test_a_token_of_nan_spoils_its_own_loss_and_dw(tokens, dtype):
    dim, vocab = 64, 300
    h, w, t, _ = _problem(tokens, dim, vocab, dtype, seed=8, ignored=0.0)
    clean = {k: v.clone() for k, v in _ops().LinearCE(tokens, dim, vocab, dtype=dtype)(h, w, t).items()}
    h[2, 3] = float("nan")
    out = _ops().LinearCE(tokens, dim, vocab, dtype=dtype)(h, w, t)
    keep = torch.arange(tokens, device="cuda") != 2
    assert torch.isnan(out["loss"][2]) and torch.isnan(out["total"]) and torch.isnan(out["dw"]).all()
    assert torch.equal(out["loss"][keep], clean["loss"][keep])
    assert torch.isnan(out["dh"][2]).all() and torch.equal(out["dh"][keep], clean["dh"][keep])


@pytest.mark.parametrize("tokens", [3, 100, 600])
@pytest.mark.parametrize("scale", [1e30, 1e-30])
def test_magnitudes_far_from_one(tokens, scale):
    """h and w at opposite ends of fp32's range: the logits are ordinary."""
    h, w, t, weight = _problem(tokens, 100, 130, F32, seed=9)
    _run_and_check(h * scale, w / scale, t, weight, True, True)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_large_and_equal_logits(dtype):
    tokens, dim, vocab = 130, 64, 500
    h, w, t, _ = _problem(tokens, dim, vocab, dtype, seed=10)
    _run_and_check(h * 200, w, t, None, False, True)      # logits of some hundreds
    _run_and_check(torch.zeros_like(h), w, t, None, False, True)
    _run_and_check(h, torch.zeros_like(w), t, None, True, True)


@pytest.mark.parametrize("tokens", [6, 100])
def test_gradients_against_differences(tokens):
    """Along random directions, from the losses alone: the step's error is the third
    derivative's (bounded by 1 here) times its square, and the losses' own errors over
    it."""
    dim, vocab = 24, 60
    h, w, t, weight = _problem(tokens, dim, vocab, F32, seed=11)
    out = _ops().LinearCE(tokens, dim, vocab)(h, w, t, weight=weight)
    gen = torch.Generator(device="cuda").manual_seed(1)
    plan = _ops().LinearCE(tokens, dim, vocab, grads=False)
    step = 2e-2
    bound = float(O.linear_ce_bounds(O.linear_ce(h, w, t, weight=weight), F32, O.U_HALVES, O.U_HALVES)["total"])
    for x, grad in ((h, out["dh"]), (w, out["dw"])):
        d = torch.empty_like(x).normal_(0, 1, generator=gen)
        d /= d.norm()
        ends = []
        for s in (step, -step):
            y = x + s * d
            ends.append(float(plan(y if x is h else h, y if x is w else w, t, weight=weight)["total"]))
        slope = float((grad.double() * d.double()).sum())
        size = float(h.double().norm()) + float(w.double().norm()) + 1
        assert abs((ends[0] - ends[1]) / (2 * step) - slope) <= bound / step + step ** 2 * size


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("tokens", [10, 100, 700])
def test_reruns_streams_and_graphs_give_the_same_bits(tokens, dtype):
    dim, vocab = 192, 1500
    h, w, t, weight = _problem(tokens, dim, vocab, dtype, seed=12)
    plan = _ops().LinearCE(tokens, dim, vocab, dtype=dtype)
    first = {k: v.clone() for k, v in plan(h, w, t, weight=weight).items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = plan(h, w, t, weight=weight)
    torch.cuda.current_stream().wait_stream(side)
    third = plan(h, w, t, weight=weight)
    torch.cuda.synchronize()
    for name in first:
        assert torch.equal(first[name], again[name]) and torch.equal(first[name], third[name]), name
    # A graph, replayed with other work and new inputs between the replays.
    h2, w2, t2, weight2 = _problem(tokens, dim, vocab, dtype, seed=13)
    second = {k: v.clone() for k, v in plan(h2, w2, t2, weight=weight2).items()}
    hs, ws, ts, cs = h.clone(), w.clone(), t.clone(), weight.clone()
    outs = dict(dh=torch.empty_like(h), dw=torch.empty_like(w), loss=torch.empty(tokens, device="cuda"),
                total=torch.empty((), device="cuda"))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan(hs, ws, ts, weight=cs, **outs)
    for k in range(4):
        want, src = ((first, (h, w, t, weight)) if k % 2 == 0 else (second, (h2, w2, t2, weight2)))
        for dst, s in zip((hs, ws, ts, cs), src):
            dst.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(outs[name], want[name]), (k, name)
        (torch.randn(64, 64, device="cuda") @ torch.randn(64, 64, device="cuda")).sum()


def test_two_plans_on_two_streams():
    a, b = (_problem(300, 128, 700, BF16, seed=s) for s in (14, 15))
    plans = [_ops().LinearCE(300, 128, 700, dtype=BF16) for _ in range(2)]
    want = [{k: v.clone() for k, v in p(x[0], x[1], x[2]).items()} for p, x in zip(plans, (a, b))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for p, x, s in zip(plans, (a, b), streams):
            with torch.cuda.stream(s):
                got.append(p(x[0], x[1], x[2]))
        torch.cuda.synchronize()
        for g, e in zip(got, want):
            assert all(torch.equal(g[n], e[n]) for n in e)


def test_refusals_of_the_helper():
    ops = _ops()
    h, w, t, weight = _problem(8, 16, 20, F32)
    plan = ops.LinearCE(8, 16, 20)
    for bad in (lambda: plan(h[:7], w, t), lambda: plan(h, w[:, :8], t), lambda: plan(h.double(), w, t),
                lambda: plan(h, w.bfloat16(), t), lambda: plan(h, w, t.int()), lambda: plan(h.cpu(), w, t),
                lambda: plan(h.t().contiguous().t(), w, t), lambda: plan(h, w, t, weight=weight.double()),
                lambda: plan(h[:1].expand(8, 16), w, t),
                lambda: plan(h, w, torch.stack([t, t], 1)[:, 0]),
                lambda: ops.LinearCE(8, 16, 20, grads=False)(h, w, t, dh=torch.empty_like(h)),
                lambda: ops.LinearCE(8, 16, 20, dtype=torch.float16)):
        with pytest.raises(ValueError):
            bad()
    for sizes in ((-1, 16, 20), (8, 0, 20), (8, 16, 0), (2 ** 21, 16, 20)):
        with pytest.raises(dsm.DsmError) as e:
            ops.LinearCE(*sizes)
        assert e.value.status == dsm.DSM_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_rows_far_from_what_a_part_of_the_vocabulary_tells(dtype):
    """Many tokens of a large vocabulary: single words that hold nearly all of a row's
    sum, in every tile of the vocabulary in turn, beside even rows, tokens left out
    and rows whose logits are all equal."""
    tokens, dim, vocab = (4100 if dtype == BF16 else 2050), 64, 30011
    h, w, t, weight = _problem(tokens, dim, vocab, dtype, seed=11)
    peaked = torch.arange(0, tokens, 2, device="cuda")
    word = (peaked * 251 + 13) % vocab
    # The word's logit is 40 |w_v| above what its neighbours have.
    unit = torch.nn.functional.normalize(w[word].float(), dim=1)
    h[peaked] = (unit * 40.0).to(dtype)
    t[peaked[::3]] = word[::3]
    h[5::16] = 0
    ops = _ops()
    out = ops.LinearCE(tokens, dim, vocab, dtype=dtype)(h, w, t, weight=weight)
    e = O.linear_ce(h, w, t, weight=weight, mean=True)
    bounds = O.linear_ce_bounds(e, dtype, *_carried(dtype, tokens, True))
    # Of c_t, an entry of G below 2^-34 may vanish; and G may be rounded twice.
    u_g = _carried(dtype, tokens, True)[1]
    bounds["dh"] += 2.0 ** -34 * e["c"][:, None] * e["w"].abs().sum(0) + u_g * (e["g"].abs() @ e["w"].abs())
    c_h = e["c"][:, None] * e["h"].abs()
    bounds["dw"] += 2.0 ** -34 * c_h.sum(0) + u_g * (e["g"].abs().t().contiguous() @ e["h"].abs())
    _check(out, e, bounds, ("total", "loss", "dh", "dw"))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_non_finite_among_many_tokens(dtype):
    """NaN in a token that is left out reaches nothing; in a token that counts, its
    dh and all of dw, and no other token's dh."""
    tokens, dim, vocab = (4100 if dtype == BF16 else 2050), 64, 30011
    h, w, t, weight = _problem(tokens, dim, vocab, dtype, seed=12, ignored=0.0)
    ops = _ops()
    plan = ops.LinearCE(tokens, dim, vocab, dtype=dtype)
    t[777] = -1
    clean = plan(h, w, t, weight=weight)
    h[777, 5] = float("nan")
    h[777, 6] = float("inf")
    out = plan(h, w, t, weight=weight)
    for name in ("total", "loss", "dh", "dw"):
        assert torch.equal(clean[name], out[name]), name
    h[1234, 7] = float("nan")
    out = plan(h, w, t, weight=weight)
    others = torch.arange(tokens, device="cuda") != 1234
    assert torch.isnan(out["total"]) and torch.isnan(out["loss"][1234]) and torch.isnan(out["dh"][1234]).all()
    assert torch.equal(out["dh"][others], clean["dh"][others])
    assert torch.equal(out["loss"][others], clean["loss"][others])
    assert torch.isnan(out["dw"]).all()
