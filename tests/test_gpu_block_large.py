"""The blocks' operators over tensors of more than 2^32 elements (fp32: 2^31), by rows at
the ends, around the offsets that pass 32 bits and elsewhere, against 64-bit values; and
the sums over all of their tokens."""
import pytest

torch = pytest.importorskip("torch")

import block_oracle as O  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB of device memory")
    yield
    torch.cuda.empty_cache()


def _ops():
    from paper_2411_17866_amd import ops
    return ops


def _rows(tokens, cols):
    near = [p // cols + k for p in (2 ** 30, 2 ** 31, 2 ** 32) for k in (-1, 0, 1)]
    gen = torch.Generator().manual_seed(1)
    some = torch.randint(0, tokens, (64,), generator=gen).tolist()
    return torch.tensor(sorted({r for r in [*range(8), *range(tokens - 70, tokens), *near, *some] if 0 <= r < tokens}), device="cuda")


def _normal(*shape, dtype=F32, sigma=1.0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0, sigma, generator=gen)


@pytest.mark.parametrize("size,dtype,name,dw_dtype", [((2 ** 20, 48, 4100), BF16, "silu", F32), ((2 ** 20, 40, 2060), F32, "none", F32)],
                         ids=["bf16", "f32"])
def test_linear(size, dtype, name, dw_dtype):
    tokens, dim, wide = size
    plan = _ops().Linear(*size, dtype=dtype, act=name, dw_dtype=dw_dtype)
    x, w = _normal(tokens, dim, dtype=dtype, seed=1), _normal(wide, dim, dtype=dtype, sigma=dim ** -0.5, seed=2)
    bias, y = _normal(wide, seed=3), _normal(tokens, wide, dtype=dtype, seed=4)
    rows = _rows(tokens, wide)
    residual = y[rows]
    out = plan(x, w, bias=bias, residual=y, y=y)
    some = {k: v[rows] for k, v in out.items()}
    e = O.linear(x[rows], w, bias, residual, name)
    O.check(some, e, O.linear_bounds(x[rows], w, bias, residual, name, False), list(some))
    z = out.get("z")
    dy = y.normal_(0, 1)
    out = plan.backward(dy, x, w, z=z)
    some = out["dx"][rows]
    e = O.linear_backward(dy[rows], x[rows], w, None if z is None else z[rows], name)
    O.check({"dx": some}, e, O.linear_backward_bounds(e, dy[rows], x[rows], w, name, dw_dtype), ["dx"])
    dw, dbias = torch.zeros(wide, dim, dtype=torch.float64, device="cuda"), torch.zeros(wide, dtype=torch.float64, device="cuda")
    for t in range(0, tokens, 2 ** 16):
        part = slice(t, t + 2 ** 16)
        e = O.linear_backward(dy[part], x[part], w, None if z is None else z[part], name)
        dw += e["dw"]
        dbias += e["dbias"]
    # (bf16: dz as two halves, 16 bits; see the long sums of the linear layer's own tests.)
    O.check_norm(out["dw"], dw, O.norm_bound(2 * tokens, F32) + 2.0 ** -16 if dtype == BF16 else O.norm_bound(tokens, F32, 2), "dw")
    O.check_norm(out["dbias"], dbias, O.norm_bound(tokens, F32), "dbias")


def test_norms():
    tokens, dim = 2 ** 19 + 12, 8192
    kinds = dict(norm="layer", post="rms", eps=1e-5, post_eps=1e-3)
    plan = _ops().ResidualNorm(tokens, dim, dtype=BF16, **kinds)
    vectors = {k: _normal(dim, seed=n) + 0.3 for n, k in enumerate(("weight", "bias", "gate", "post_weight", "post_bias"))}
    h, f = _normal(tokens, dim, dtype=BF16, seed=11), _normal(tokens, dim, dtype=BF16, seed=12)
    rows = _rows(tokens, dim)
    e = O.residual_norm(h[rows], f[rows], scale=0.7, **vectors, **kinds)
    out = plan(h, f=f, scale=0.7, s=h, **vectors)
    O.check({k: v[rows] for k, v in out.items()}, e, {k: e[k + "_bound"] for k in out}, list(out))
    dy, ds, s = out["y"].normal_(0, 1), _normal(tokens, dim, dtype=BF16, seed=13), out["s"]
    e = O.residual_norm_backward(dy[rows], s[rows], f[rows], ds[rows], scale=0.7, **vectors, **kinds)
    sums = {"d" + k: torch.zeros(dim, dtype=torch.float64, device="cuda") for k in vectors}
    for t in range(0, tokens, 2 ** 15):
        part = slice(t, t + 2 ** 15)
        each = O.residual_norm_backward(dy[part], s[part], f[part], ds[part], scale=0.7, **vectors, **kinds)
        for k in sums:
            sums[k] += each[k]
        del each
    got = plan.backward(dy, s, f=f, ds=ds, scale=0.7, dh=ds, df=f, **vectors)
    O.check({k: got[k][rows] for k in ("dh", "df")}, e, {k: e[k + "_bound"] for k in ("dh", "df")}, ["dh", "df"])
    for k, want in sums.items():
        # Terms: a row's statistics are sums of 8 numbers a lane, 64 lanes and 16 waves, some 30 roundings each,
        # and few more: below 2^-16.
        O.check_norm(got[k], want, O.norm_bound(tokens, F32) + 2.0 ** -16, k)


def test_clipping():
    n = 2 ** 32 + 1003
    g, other = _normal(n, seed=21), _normal(1000, dtype=BF16, seed=22)
    plan = _ops().GradClip([g, other])
    places = [0, 2 ** 30 - 500, 2 ** 31 - 500, 2 ** 32 - 500, n - 1000]
    before = [g[p:p + 1000].double() for p in places]
    square = sum(float(g[t:t + 2 ** 28].double().square().sum()) for t in range(0, n, 2 ** 28)) + float(other.double().square().sum())
    norm = plan([g, other], 1.0)
    assert abs(float(norm[0]) - square ** 0.5) <= 1.01 * U * square ** 0.5
    factor = 1.0 / (square ** 0.5 + 1e-6)
    for p, b in zip(places, before):
        # One rounding to fp32 (a few below its normal numbers lose more: none here), and the sums' order in fp64.
        assert ((g[p:p + 1000].double() - b * factor).abs() <= 1.01 * U * (b * factor).abs()).all(), p
