"""dsm_grad_clip on the GPU against 64-bit values: lists of tensors of both types, odd
sizes and rows apart, groups, arenas in every layout, magnitudes, non-finite entries;
streams, graphs, refusals."""
import math
import threading

import pytest

torch = pytest.importorskip("torch")

import block_oracle as O  # noqa: E402
from paper_2411_17866_amd import arena, dsm  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _ops():
    from paper_2411_17866_amd import ops
    return ops


def _tensors(shapes, dtypes, seed=0, sigma=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.empty(s, device="cuda").normal_(0, sigma, generator=gen).to(d) for s, d in zip(shapes, dtypes)]


def _check(tensors, groups, max_norm, eps=1e-6, norm_bound=4 * O.U):
    """Runs a plan and holds norms (fp64 sums, one rounding) and tensors (the factor's rounding, the product's, the type's)
    to their values."""
    norms, want = O.clip(tensors, groups, math.inf if max_norm is None else max_norm, eps)
    before = [t.clone() for t in tensors]
    plan = _ops().GradClip(tensors, groups=groups, eps=eps)
    got = plan(tensors, max_norm).tolist()
    for a, b in zip(got, norms):
        assert abs(a - b) <= norm_bound * b
    for t, b, w, g in zip(tensors, before, want, groups):
        if max_norm is None or norms[g] + eps < max_norm * (1 - 1e-6):
            assert torch.equal(t, b)  # as it was, to the bit
        else:
            half = O.HALF[t.dtype]
            assert ((t.double() - w).abs() <= (half + 4 * O.U) * w.abs() + 2.0 ** -149).all()
    return got


SIZES = [(1,), (7,), (8,), (9,), (2047,), (2048,), (16383,), (16384,), (16385,), (40000,), (33, 500), (3, 5, 7), (0,), (1, 1), (100003,)]


@pytest.mark.parametrize("max_norm", [None, 0.5, 1e9, 0.0])
def test_lists(max_norm):
    types = [F32, BF16, BF16, F32]
    ts = _tensors(SIZES, [types[k % 4] for k in range(len(SIZES))], seed=1)
    _check(ts, [0] * len(ts), max_norm)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_single_tensors(size, dtype):
    ts = _tensors([size], [dtype], seed=2)
    _check(ts, [0], 0.25)


def test_groups_in_any_order():
    ts = _tensors([(n,) for n in (5, 20000, 300, 17, 4000, 1)], [F32, BF16, F32, F32, BF16, F32], seed=3)
    got = _check(ts, [2, 0, 2, 0, 4, 2], 3.0)
    assert len(got) == 5 and got[1] == 0.0 and got[3] == 0.0  # groups without tensors
    ts = _tensors([(64,)] * 300, [F32] * 300, seed=4)  # more groups than the joined launch takes, several tables
    _check(ts, [k % 200 for k in range(300)], 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_rows_apart_and_misaligned(dtype):
    for rows, cols, pad, skip in ((300, 100, 4, 0), (300, 104, 8, 8), (70, 513, 3, 1), (5, 20000, 16, 3), (3, 16384, 8, 0), (2, 40007, 9, 5),
                                  (4096, 1, 7, 1), (1, 50, 0, 1)):
        big = torch.full((rows * (cols + pad) + 16,), float("nan"), device="cuda", dtype=dtype)
        v = torch.as_strided(big[skip:], (rows, cols), (cols + pad, 1))
        v.copy_(_tensors([(rows, cols)], [dtype], seed=5)[0])
        flat = _tensors([(999,)], [dtype], seed=6)[0][1:]
        _check([v, flat], [0, 0], 2.0)
        rest = torch.ones_like(big, dtype=torch.bool)
        torch.as_strided(rest[skip:], v.shape, v.stride()).fill_(False)
        assert torch.isnan(big[rest]).all()


def test_neighbours_in_memory():
    """Tensors that follow each other become one run; a gap, a type or a group ends it."""
    flat = _tensors([(100000,)], [F32], seed=7)[0]
    cuts = [0, 7, 64, 20000, 20000, 36385, 50000, 77777, 100000]
    ts = [flat[a:b] for a, b in zip(cuts, cuts[1:]) if (a, b) != (64, 20000)]
    keep = flat[64:20000].clone()
    _check(ts, [0, 0, 0, 0, 0, 1, 1], 1.5)
    assert torch.equal(flat[64:20000], keep)


@pytest.mark.parametrize("sigma", [1e-38, 1e-22, 1e18, 1e30])
def test_magnitudes(sigma):
    """Squares beyond fp32's range, both ways."""
    ts = _tensors([(5000,), (70, 11)], [F32, F32], seed=8, sigma=sigma)
    _check(ts, [0, 0], 1e-20 * sigma if sigma > 1 else sigma, eps=0.0)


def test_non_finite_groups_stay():
    for bad in (float("nan"), float("inf")):
        ts = _tensors([(500,), (20000,), (33,)], [F32, F32, BF16], seed=9)
        ts[1][777] = bad
        before = [t.clone() for t in ts]
        got = _ops().GradClip(ts, groups=[0, 0, 1])(ts, 0.1).tolist()
        assert not math.isfinite(got[0]) and math.isfinite(got[1])
        assert torch.equal(ts[0], before[0]) and torch.equal(ts[1].nan_to_num(7.0), before[1].nan_to_num(7.0))
        assert float(ts[2].float().norm()) < 0.11
    # A norm beyond fp32 is still a number: gradients are clipped by it.
    t = torch.full((40000,), 3e38, device="cuda")
    assert _ops().GradClip([t])([t], 2.0).tolist() == [float("inf")]
    assert abs(float(t.double().norm()) - 2.0) < 1e-5


def test_nothing():
    norm = _ops().GradClip([])([], 1.0)
    assert norm.tolist() == [0.0]
    t = torch.zeros(100, device="cuda")
    assert _ops().GradClip([t], eps=0.0)([t], 0.0).tolist() == [0.0] and not t.any()


@pytest.mark.parametrize("together", [False, True])
@pytest.mark.parametrize("layout", [dsm.DSM_REPLICAS_CONTIGUOUS, dsm.DSM_REPLICAS_BLOCKED, dsm.DSM_REPLICAS_STATE_BLOCKED])
@pytest.mark.parametrize("base", [dsm.DSM_BASE_ADAMW, dsm.DSM_BASE_SGD_MOMENTUM])
def test_arenas(layout, together, base):
    numel = [1, 65, 5000, 0, 16384, 40001, 3]
    ar = arena.Arenas(numel, 3, 2, base, replica_layout=layout)
    for name in ("x_rep", "s1_rep"):
        getattr(ar, name).fill_(3.0)
    g = torch.full((3, ar.arena_elems), 5.0, device="cuda")  # padding holds 5
    values = [_tensors([(n,) for n in numel], [F32] * len(numel), seed=20 + w) for w in range(3)]
    for w in range(3):
        for o, t in zip(ar.offsets, values[w]):
            g[w, int(o):int(o) + t.numel()] = t * (w + 1)
    ar.write_workers("g_rep", g)
    flat = [g[w, int(o):int(o) + n].clone() for w in range(3) for o, n in zip(ar.offsets, numel)]
    groups = [0 if together else w for w in range(3) for _ in numel]
    norms, want = O.clip(flat, groups, 150.0)
    got = _ops().ArenaClip(ar, together=together)(ar, 150.0).tolist()
    assert len(got) == len(norms) and all(abs(a - b) <= 4 * O.U * b for a, b in zip(got, norms))
    assert max(norms) > 150 and (together or min(norms) < max(norms))
    after = ar.workers("g_rep")
    for w in range(3):
        rest = torch.ones(ar.arena_elems, dtype=torch.bool, device="cuda")
        for k, (o, n) in enumerate(zip(ar.offsets, numel)):
            t = want[w * len(numel) + k]
            rest[int(o):int(o) + n] = False
            assert ((after[w, int(o):int(o) + n].double() - t).abs() <= 6 * O.U * t.abs()).all()
        assert (after[w][rest] == 5.0).all()
    assert (ar.workers("x_rep") == 3.0).all() and (ar.workers("s1_rep") == 3.0).all()


@pytest.mark.parametrize("size", [3000, 40_000_000])
def test_graphs_replay(size):
    gen = torch.Generator(device="cuda").manual_seed(1)
    t = torch.empty(size, device="cuda").normal_(0, 1, generator=gen)
    plan = _ops().GradClip([t])
    norm = plan([t], 2.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan([t], 2.0, norm=norm)
    for k in range(3):
        fresh = torch.empty(size, device="cuda").normal_(0, 10.0 ** -k, generator=gen)
        want = fresh.clone()
        want_norm = plan([want], 2.0)
        t.copy_(fresh)
        norm.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(t, want) and torch.equal(norm, want_norm)


def test_streams_and_threads():
    ts = _tensors([(30000,), (500, 33)], [F32, F32], seed=11)
    plan = _ops().GradClip(ts)
    other = [t.clone() for t in ts]
    want_norm = plan(other, 1.0)
    torch.cuda.synchronize()
    bad = []

    def work():
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                mine = [t.clone() for t in ts]
                norm = plan(mine, 1.0)
                stream.synchronize()
                if not (torch.equal(norm, want_norm) and all(torch.equal(a, b) for a, b in zip(mine, other))):
                    bad.append(1)

    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_refusals():
    ops = _ops()
    t = torch.ones(6, 8, device="cuda")
    plan = ops.GradClip([t])
    for call in (lambda: ops.GradClip([t], groups=[0, 1]), lambda: ops.GradClip([t], groups=[-1]), lambda: ops.GradClip([t.half()]),
                 lambda: ops.GradClip([t], groups=[256]), lambda: plan([t, t]), lambda: plan([t[:5]]), lambda: plan([t.to(BF16)]),
                 lambda: plan([t.cpu()]), lambda: plan([torch.ones(8, 6, device="cuda").t()]), lambda: plan([t[:1].expand(6, 8)]),
                 lambda: plan([t], -1.0), lambda: plan([t], float("nan")), lambda: plan([t], 1.0, norm=torch.empty(2, device="cuda")),
                 lambda: ops.GradClip([t], eps=-1.0)([t], 1.0)):
        with pytest.raises((ValueError, dsm.DsmError)):
            call()
    twice = ops.GradClip([t, t[:0], t[:0], t])
    with pytest.raises(ValueError, match="twice"):
        twice([t, t[:0], t[:0], t], 1.0)
    u = torch.ones(6, 8, device="cuda")
    assert twice([t, t[:0], t[:0], u], 1.0).tolist() == [pytest.approx(96 ** 0.5)] and torch.equal(t, u)
    ar = arena.Arenas([100], 2, 2, dsm.DSM_BASE_SGD_MOMENTUM)
    with pytest.raises(ValueError):
        ops.ArenaClip(ar)(arena.Arenas([101], 2, 2, dsm.DSM_BASE_SGD_MOMENTUM), 1.0)
