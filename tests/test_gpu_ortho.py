"""dsm_orthogonalize and dsm_ortho_step on the GPU against 64-bit values, over
types, shapes around every tile and path, layouts, scales and non-finite matrices;
the step's state; reruns, streams, graphs."""
import pytest

torch = pytest.importorskip("torch")

import ops_oracle as O  # noqa: E402
from paper_2411_17866_amd import dsm  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _ops():
    from paper_2411_17866_amd import ops
    return ops


def _update(count, rows, cols, dtype=F32, seed=0, scale=1e-3, rank=4):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.empty(shape, device="cuda").normal_(0, 1, generator=gen)

    strong = normal(count, rows, rank) @ normal(count, rank, cols)
    return (scale * (0.5 * strong + normal(count, rows, cols))).to(dtype)


def _check(got, u, steps=5, eps=1e-7, coeffs=None):
    want = O.orthogonalize(u, steps, eps, coeffs)
    bound = O.orthogonalize_bound(u, u.dtype, steps, eps, coeffs)
    got = got.double()
    assert torch.isfinite(got).all()
    off = (got - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1).clamp(min=1e-300)
    assert (off <= bound).all(), f"{off.tolist()} beyond {bound.tolist()}"


# Sizes of one; a single work-group (padded to 32); its limits; tiles of 64, 128 and
# 256 and their edges; odd sizes; tall and wide.
SHAPES = [(1, 1, 1), (1, 1, 7), (2, 7, 1), (1, 16, 16), (3, 33, 65), (1, 48, 64), (2, 64, 48), (1, 32, 500),
          (1, 500, 32), (1, 64, 320), (1, 96, 96), (1, 97, 128), (2, 130, 70), (1, 128, 128), (1, 200, 300),
          (3, 300, 200), (1, 257, 513), (1, 64, 1030), (1, 1030, 64), (2, 384, 384), (1, 640, 1000), (9, 256, 512),
          (5, 320, 1280), (12, 384, 1152), (1, 1100, 1100)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_against_64_bits(shape, dtype):
    u = _update(*shape, dtype, seed=sum(shape))
    out = _ops().Ortho(shape[1], shape[2], shape[0], dtype=dtype).orthogonalize(u)
    _check(out, u)


@pytest.mark.parametrize("shape", [(2, 40, 60), (2, 300, 140), (1, 513, 700)], ids=str)
@pytest.mark.parametrize("steps", [1, 2, 3, 9])
def test_iterations(shape, steps):
    for dtype in (F32, BF16):
        u = _update(*shape, dtype, seed=steps)
        out = _ops().Ortho(shape[1], shape[2], shape[0], dtype=dtype, steps=steps).orthogonalize(u)
        _check(out, u, steps=steps)


@pytest.mark.parametrize("shape", [(1, 40, 60), (2, 300, 140)], ids=str)
def test_other_coefficients(shape):
    for coeffs in ([[1.5, -0.5, 0.0]] * 4, [[3.4445, -4.775, 2.0315]] * 2 + [[1.875, -1.25, 0.375]] * 2,
                   [[1.0, 0.0, 0.0]], [[0.0, 0.0, 0.0]] * 2, [[-2.0, 0.5, 0.25]] * 2):
        u = _update(*shape, seed=len(coeffs))
        out = _ops().Ortho(shape[1], shape[2], shape[0], steps=len(coeffs), coeffs=coeffs).orthogonalize(u)
        if coeffs[0] == [0.0, 0.0, 0.0]:
            assert (out == 0).all()
        else:
            _check(out, u, steps=len(coeffs), coeffs=coeffs)


@pytest.mark.parametrize("shape", [(1, 64, 64), (1, 300, 500), (1, 600, 200)], ids=str)
def test_singular_values_come_near_one(shape):
    u = _update(*shape, seed=1, rank=1)
    s = torch.linalg.svdvals(u[0].double().cpu())
    t = torch.linalg.svdvals(_ops().Ortho(*shape[1:]).orthogonalize(u)[0].double().cpu())
    # Every singular value above 1/100 of the norm goes into [0.65, 1.25].
    n = int((s > 0.01 * s.norm()).sum())
    assert n > 0 and t[0] < 1.25 and t[n - 1] > 0.65


@pytest.mark.parametrize("shape", [(3, 48, 64), (3, 200, 130)], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_zero_and_non_finite_matrices_keep_to_themselves(shape, dtype):
    u = _update(*shape, dtype, seed=2)
    u[1] = 0
    ops = _ops()
    out = ops.Ortho(*shape[1:], shape[0], dtype=dtype).orthogonalize(u)
    assert (out[1] == 0).all()
    _check(out[::2], u[::2].contiguous())
    for value in (float("nan"), float("inf"), -float("inf")):
        bad = u.clone()
        bad[1, 3, 5] = value
        got = ops.Ortho(*shape[1:], shape[0], dtype=dtype).orthogonalize(bad)
        assert torch.isnan(got[1]).all()
        assert torch.equal(got[::2], out[::2])


@pytest.mark.parametrize("shape", [(2, 48, 64), (2, 300, 200)], ids=str)
@pytest.mark.parametrize("scale", [1e30, 1e-12, 1e-30])
def test_scales_whose_squares_leave_fp32(shape, scale):
    u = _update(*shape, seed=3) * scale
    _check(_ops().Ortho(*shape[1:], shape[0], eps=0.0).orthogonalize(u), u, eps=0.0)
    _check(_ops().Ortho(*shape[1:], shape[0]).orthogonalize(u), u)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 40, 52), (3, 200, 136), (2, 129, 300)], ids=str)
def test_views(shape, dtype):
    """Rows apart, matrices apart, side by side, misaligned, in place."""
    count, rows, cols = shape
    u = _update(*shape, dtype, seed=4)
    want = _ops().Ortho(rows, cols, count, dtype=dtype).orthogonalize(u)
    for row, each, skip in ((cols + 4, rows * (cols + 4) + 12, 4), (cols + 3, rows * (cols + 3) + 1, 1),
                            (count * cols, cols, 0), (count * (cols + 1), cols + 1, 3)):
        big = torch.full((skip + count * rows * (cols + 4) + 64 * count,), float("nan"), device="cuda", dtype=dtype)
        v = torch.as_strided(big, shape, (each, row, 1), skip)
        v.copy_(u)
        plan = _ops().Ortho(rows, cols, count, dtype=dtype)
        out = plan.orthogonalize(v)
        assert torch.equal(out, want)
        plan.orthogonalize(v, out=v)
        assert torch.equal(v, want)
        rest = torch.ones_like(big, dtype=torch.bool)
        torch.as_strided(rest, shape, (each, row, 1), skip).fill_(False)
        assert torch.isnan(big[rest]).all()


def test_more_matrices_than_one_set_of_launches_takes():
    for rows, cols in ((20, 24), (130, 70)):
        u = _update(150, rows, cols, seed=5)
        plan = _ops().Ortho(rows, cols, 150)
        out = plan.orthogonalize(u)
        one = _ops().Ortho(rows, cols, 1)
        for k in (0, 63, 64, 127, 128, 149):
            assert torch.equal(out[k], one.orthogonalize(u[k]))


@pytest.mark.parametrize("shape", [(2, 40, 60), (1, 64, 48), (2, 200, 300), (2, 300, 200), (1, 513, 260)], ids=str)
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("momentum", [True, False])
def test_step(shape, nesterov, momentum):
    x, m, g = (_update(*shape, seed=s) for s in (6, 7, 8))
    x *= 20
    x0, m0 = x.clone(), m.clone()
    plan = _ops().Ortho(*shape[1:], shape[0])
    hp = dict(lr=0.02, mu=0.95, scale=0.7, nesterov=nesterov)
    plan.step(x, m if momentum else None, g, wd=0.1, **hp)
    # The momentum and u in fp32, an operation at a time.
    mu, one = torch.tensor(0.95), torch.float32
    m1 = (mu.to("cuda", one) * m0 + g) if momentum else m0
    assert torch.equal(m, m1)
    u = g if not momentum else (g + mu.to("cuda", one) * m1 if nesterov else m1)
    o = O.orthogonalize(u)
    want = x0.double() - 0.02 * (0.7 * o + 0.1 * x0.double())
    bound = 0.02 * 0.7 * O.orthogonalize_bound(u, F32) * o.flatten(1).norm(dim=1)
    off = (x.double() - want).flatten(1).norm(dim=1)
    assert (off <= bound + 2.0 ** -22 * want.flatten(1).norm(dim=1)).all()
    # The direction, written over the gradient.
    m2, d = m0.clone(), g.clone()
    plan.direction(m2 if momentum else None, d, d, mu=0.95, scale=0.7, nesterov=nesterov)
    assert torch.equal(m2, m1)
    off = (d.double() - 0.7 * o).flatten(1).norm(dim=1)
    assert (off <= 0.7 * (O.orthogonalize_bound(u, F32) + 2.0 ** -22) * o.flatten(1).norm(dim=1)).all()


def test_arenas_and_offsets():
    """Matrices of two shapes inside the arenas, every worker's at once; the other
    tensors stay."""
    from paper_2411_17866_amd import arena
    shapes = [(40, 60), (7,), (40, 60), (130, 64), (33,)]
    numel = [s[0] * (s[1] if len(s) > 1 else 1) for s in shapes]
    ar = arena.Arenas(numel, 3, 2, dsm.DSM_BASE_SGD_MOMENTUM)
    gen = torch.Generator(device="cuda").manual_seed(9)
    ar.g_rep.normal_(0, 1e-3, generator=gen)
    before = ar.g_rep.clone()
    mom = torch.zeros_like(ar.g_rep)
    for shape, which in (((40, 60), (0, 2)), ((130, 64), (3,))):
        offsets = [int(ar.offsets[p]) + i * ar.arena_elems for i in range(3) for p in which]
        plan = _ops().Ortho(*shape, len(offsets), offsets=offsets)
        plan.direction(mom, ar.g_rep, ar.g_rep, mu=0.9, scale=1.0)
        for i in range(3):
            for p in which:
                o = int(ar.offsets[p])
                g = before[i, o:o + numel[p]].view(1, *shape)
                d = ar.g_rep[i, o:o + numel[p]].view(1, *shape)
                assert torch.equal(mom[i, o:o + numel[p]].view(1, *shape), g)
                one = _ops().Ortho(*shape).direction(None, g, torch.empty_like(g), mu=0.0)
                _check(d, g + torch.tensor(0.9, device="cuda") * g)
                _check(one, g)
    for i in range(3):
        for p in (1, 4):
            o = int(ar.offsets[p])
            assert torch.equal(ar.g_rep[i, o:o + numel[p]], before[i, o:o + numel[p]])
    ar.destroy()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 48, 64), (2, 300, 200), (1, 700, 640)], ids=str)
def test_reruns_streams_and_graphs_give_the_same_bits(shape, dtype):
    u, v = _update(*shape, dtype, seed=10), _update(*shape, dtype, seed=11)
    plan = _ops().Ortho(*shape[1:], shape[0], dtype=dtype)
    first, second = plan.orthogonalize(u), plan.orthogonalize(v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = plan.orthogonalize(u)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(plan.orthogonalize(u), first) and torch.equal(again, first)
    src, out = u.clone(), torch.empty_like(u)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.orthogonalize(src, out=out)
    for k in range(4):
        src.copy_(u if k % 2 == 0 else v)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first if k % 2 == 0 else second), k
        (torch.randn(64, 64, device="cuda") @ torch.randn(64, 64, device="cuda")).sum()


def test_empty_problems():
    for count, rows, cols in ((0, 5, 6), (3, 0, 6), (3, 5, 0)):
        u = torch.empty(count, rows, cols, device="cuda")
        plan = _ops().Ortho(rows, cols, count)
        assert plan.orthogonalize(u).shape == u.shape
        plan.step(u.clone(), u.clone(), u, lr=0.1, mu=0.9)


def test_refusals_of_the_helper():
    ops = _ops()
    u = _update(2, 8, 12)
    plan = ops.Ortho(8, 12, 2)
    for bad in (lambda: plan.orthogonalize(u[:1]), lambda: plan.orthogonalize(u.double()),
                lambda: plan.orthogonalize(u.cpu()), lambda: plan.orthogonalize(u[:, :, ::2].repeat(1, 1, 2)[:, :, ::2]),
                lambda: plan.orthogonalize(u.transpose(1, 2).contiguous().transpose(1, 2)),
                lambda: plan.orthogonalize(u[:1].expand(2, 8, 12)),
                lambda: plan.orthogonalize(u, out=torch.empty(2, 8, 13, device="cuda")[:, :, :12]),
                lambda: ops.Ortho(8, 12, 2, offsets=[0]), lambda: ops.Ortho(8, 12, 2, dtype=torch.float16),
                lambda: ops.Ortho(8, 12, 2, coeffs=[[1, 2, 3]]),
                lambda: ops.Ortho(8, 12, 2, offsets=[0, 96]).orthogonalize(u.flatten()[:150], out=u.flatten())):
        with pytest.raises(ValueError):
            bad()
    for call, status in ((lambda: ops.Ortho(8, 12, 2, steps=0), dsm.DSM_ERR_INVALID_ARG),
                         (lambda: ops.Ortho(8, 12, 2, steps=33), dsm.DSM_ERR_INVALID_ARG),
                         (lambda: ops.Ortho(2 ** 15, 2 ** 15), dsm.DSM_ERR_INVALID_ARG),
                         (lambda: ops.Ortho(8, 12, eps=-1.0), dsm.DSM_ERR_INVALID_ARG),
                         (lambda: ops.Ortho(8, 12, 2, steps=2, coeffs=[[1e3, 0, 0]] * 2), dsm.DSM_ERR_UNSUPPORTED),
                         (lambda: plan.step(u, None, u, lr=0.0, mu=0.9), dsm.DSM_ERR_INVALID_ARG),
                         (lambda: plan.step(u, u, u, lr=0.1, mu=1.5), dsm.DSM_ERR_INVALID_ARG),
                         (lambda: plan.step(u, u, u, lr=0.1, mu=0.5, wd=-1.0), dsm.DSM_ERR_INVALID_ARG)):
        with pytest.raises(dsm.DsmError) as e:
            call()
        assert e.value.status == status
