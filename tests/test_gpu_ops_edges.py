"""The operators where plain arithmetic would not notice anything: magnitudes at the
ends of fp32, rows that are nearly sure of their target, launches past 2^32 threads,
non-finite words, zeros without eps."""
import math
import threading

import pytest

torch = pytest.importorskip("torch")

import ops_norms as N  # noqa: E402
import ops_oracle as O  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
DTYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
# Through every form: w read in place, tiles of 128, of 256, and with references; vocabularies
# that fit no tile.
SIZES = pytest.mark.parametrize("size", [(5, 64, 1001), (100, 64, 1001), (600, 64, 1001), (200, 72, 50257),
                                         (4100, 64, 30011)], ids=str)


def _ops():
    from paper_2411_17866_amd import ops
    return ops


def _normal(*shape, seed=0):
    return torch.empty(shape, device="cuda").normal_(0, 1, generator=torch.Generator(device="cuda").manual_seed(seed))


@DTYPES
@SIZES
def test_both_operands_tiny(size, dtype):
    """Logits of 1e-38 are equal ones: the loss is log(vocab), and the gradients are
    those of even rows."""
    tokens, dim, vocab = size
    h, w = (1e-20 * _normal(tokens, dim, seed=1)).to(dtype), (1e-18 * _normal(vocab, dim, seed=2)).to(dtype)
    t = torch.arange(tokens, device="cuda") * 7 % vocab
    for grads in (True, False):
        out = _ops().LinearCE(*size, dtype=dtype, grads=grads)(h, w, t, mean=False)
        assert (out["loss"] - math.log(vocab)).abs().max() <= 2.0 ** -21 * math.log(vocab)
        assert abs(float(out["total"]) / tokens - math.log(vocab)) <= 2.0 ** -21 * math.log(vocab)
        if grads:
            e = N.linear_ce(h, w, t, mean=False)
            assert N.off(out["dh"], e["dh"]) <= N.GRAD[dtype] and N.off(out["dw"], e["dw"]) <= N.GRAD[dtype]


def test_more_threads_than_a_launch_takes():
    """2^20 tokens by 2^19 words: 2^32 threads over the logits' tiles."""
    tokens, dim, vocab = 1 << 20, 8, 1 << 19
    h, w = _normal(tokens, dim, seed=5).to(BF16), _normal(vocab, dim, seed=6).to(BF16)
    t = torch.randint(0, vocab, (tokens,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(20))
    out = _ops().LinearCE(tokens, dim, vocab, dtype=BF16, grads=False)(h, w, t)
    rows = torch.cat([torch.arange(0, tokens, 16411, device="cuda"), torch.arange(tokens - 20, tokens, device="cuda")])
    e = N.linear_ce(h[rows], w, t[rows], grads=False)
    assert N.off(out["loss"][rows], e["loss"]) <= N.LOSS
    assert abs(float(out["total"]) - float(out["loss"].double().mean())) <= 1e-6 * float(out["total"])


@DTYPES
@pytest.mark.parametrize("dim", [64, 60])  # h read in place, and copied
@pytest.mark.parametrize("grads", [True, False])
@pytest.mark.parametrize("tokens", [5, 100, 600])
def test_lse_of_tokens_without_a_target(tokens, grads, dim, dtype):
    vocab = 300
    h, w = _normal(tokens, dim, seed=9).to(dtype), (dim ** -0.5 * _normal(vocab, dim, seed=10)).to(dtype)
    t = torch.randint(0, vocab, (tokens,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(20))
    t[::2] = -1
    lse = torch.full((tokens,), float("nan"), device="cuda")
    _ops().LinearCE(tokens, dim, vocab, dtype=dtype, grads=grads)(h, w, t, lse=lse)
    assert (lse[::2] == 0).all()
    want = torch.logsumexp(h[1::2].double() @ w.double().t().contiguous(), 1)
    assert (lse[1::2].double() - want).abs().max() <= 2.0 ** -18


@DTYPES
@SIZES
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_non_finite_words_leave_tokens_without_a_target_alone(size, dtype, value):
    tokens, dim, vocab = size
    h, w = _normal(tokens, dim, seed=7).to(dtype), (dim ** -0.5 * _normal(vocab, dim, seed=8)).to(dtype)
    t = torch.randint(0, vocab, (tokens,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(20))
    out_of = torch.arange(tokens, device="cuda") % 3 == 1
    t[out_of] = -1
    w[vocab // 2, 3] = value
    lse = torch.full((tokens,), float("nan"), device="cuda")
    out = _ops().LinearCE(*size, dtype=dtype)(h, w, t, lse=lse)
    for x in (out["dh"], out["loss"], lse):
        assert (x[out_of] == 0).all()
    # (A logit of -inf leaves its token a probability of 0 there: 0 * inf in one column, or
    # -inf where the word is its target.)
    assert not torch.isfinite(out["dh"][~out_of][:, 3]).any()
    if value != value:
        assert torch.isnan(out["dh"][~out_of]).all() and torch.isnan(out["total"])
    # No token that counts: nothing is left.
    t.fill_(vocab)
    out = _ops().LinearCE(*size, dtype=dtype)(h, w, t, lse=lse)
    for x in (out["dh"], out["dw"], out["loss"], out["total"], lse):
        assert (x == 0).all()


@pytest.mark.parametrize("size,dtype", [((4500, 64, 65001), F32), ((9000, 64, 65001), BF16)], ids=str)
def test_non_finite_words_of_a_later_piece(size, dtype):
    """Two pieces of the vocabulary; no token counts, then some."""
    tokens, dim, vocab = size
    h, w = _normal(tokens, dim, seed=7).to(dtype), (dim ** -0.5 * _normal(vocab, dim, seed=8)).to(dtype)
    w[vocab - 5, 3] = float("nan")
    t = torch.full((tokens,), -1, device="cuda")
    plan = _ops().LinearCE(*size, dtype=dtype)
    out = plan(h, w, t)
    for name, x in out.items():
        assert (x == 0).all(), name
    t[::2] = 11
    out = plan(h, w, t)
    assert (out["dh"][1::2] == 0).all() and torch.isnan(out["dh"][::2]).all()


@DTYPES
@SIZES
def test_rows_nearly_sure_of_their_target(size, dtype):
    """Losses from 1e-6 to 1e-2 keep their digits, and so do the gradients of such
    rows: what bounds both is the logits' own rounding."""
    tokens, dim, vocab = size
    w = torch.nn.functional.normalize(_normal(vocab, dim, seed=3), dim=1).to(dtype)
    # A third of the targets among the first words, which stand for frequent ones.
    t = torch.randint(0, vocab, (tokens,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))
    t[::3] %= 200
    # exp(others - target) sums to about vocab exp(a^2 / 2 dim - a).
    want = 10.0 ** torch.linspace(-6, -2, tokens, device="cuda")
    a = torch.full_like(want, 20.0)
    for _ in range(30):
        a = math.log(vocab) - want.log() + a * a / (2 * dim)
        a.clamp_(max=45.0)
    h = (a[:, None] * w[t].float()).to(dtype)
    e = N.linear_ce(h, w, t, mean=False)
    # Two logits of up to z (that of the target and those of the others that count), each a
    # sum of dim terms and of operands of 22 bits; three more roundings of z; log1p and exp.
    z = float(a.max())
    tol = 2 * z * (2.0 ** -24 * dim ** 0.5 + 2.0 ** -22) + 4 * z * 2.0 ** -24 + 2.0 ** -20
    for grads in (True, False):
        out = _ops().LinearCE(*size, dtype=dtype, grads=grads)(h, w, t, mean=False)
        rel = (out["loss"].double() - e["loss"]).abs() / e["loss"]
        assert (rel <= tol).all(), f"{float(rel.max()):.3g} beyond {tol:.3g}"
        if grads:
            # G's entries by the same; dh's rounding; and what G's 16-bit storage leaves out,
            # 2^-34 an entry, in random directions of w's unit rows.
            norm = e["dh"].norm(dim=1)
            dh = (out["dh"].double() - e["dh"]).norm(dim=1) / norm
            far = dh - (tol + N.GRAD[dtype] + 2.0 ** -34 * vocab ** 0.5 / norm)
            assert (far <= 0).all(), f"{int((far > 0).sum())} rows, by {float(far.max()):.3g}"


@DTYPES
@pytest.mark.parametrize("shape", [(3, 48, 64), (3, 200, 130), (3, 130, 200)], ids=str)
def test_zeros_without_eps(shape, dtype):
    u = (1e-3 * _normal(*shape, seed=11)).to(dtype)
    u[1] = 0
    plan = _ops().Ortho(*shape[1:], shape[0], dtype=dtype, eps=0.0)
    out = plan.orthogonalize(u)
    assert (out[1] == 0).all()
    want = O.orthogonalize(u[::2], eps=0.0)
    assert N.off(out[::2], want) <= (1e-5 if dtype == F32 else 4e-3)
    if dtype == F32:
        x = _normal(*shape, seed=12)
        x0 = x.clone()
        plan.step(x, None, u, lr=0.1, mu=0.0, wd=0.0)
        assert torch.equal(x[1], x0[1]) and torch.isfinite(x).all()


@pytest.mark.parametrize("shape", [(2, 200, 200), (2, 130, 70), (1, 400, 1600), (3, 900, 385), (12, 768, 768)], ids=str)
@pytest.mark.parametrize("noise", [1e-2, 1e-4])
def test_bf16_matrices_of_low_rank_cost_little_more_than_their_rounding(shape, noise):
    """Against 64 bits a bf16 result cannot be nearer than its rounding; what the
    iteration's own operands add has to stay below three quarters of that, which makes
    1.25 of it together.  Small singular values under a few large ones are multiplied by
    up to 485, and with them what storage puts there."""
    u = _normal(*shape[:2], 5, seed=13) @ _normal(shape[0], 5, shape[2], seed=14) + noise * _normal(*shape, seed=15)
    u = u.to(BF16)
    want = O.orthogonalize(u)
    out = _ops().Ortho(*shape[1:], shape[0], dtype=BF16).orthogonalize(u)
    assert N.off(out, want) <= 1.25 * N.off(want.to(BF16), want)


@pytest.mark.parametrize("shape", [(2, 200, 200), (2, 130, 70), (1, 400, 1600), (3, 900, 385), (12, 768, 768)], ids=str)
@pytest.mark.parametrize("spectrum", ["noise", "orthogonal", "power"])
def test_bf16_matrices_cost_little_more_than_their_rounding(shape, spectrum):
    """The same where all singular values end near 1: there a X and B X nearly cancel."""
    u = _normal(*shape, seed=16)
    if spectrum != "noise":
        left, _, right = torch.linalg.svd(u.double(), full_matrices=False)
        s = torch.arange(1, left.shape[2] + 1, device="cuda").double() ** (-1.0 if spectrum == "power" else 0.0)
        u = (left * s) @ right
    u = u.to(BF16)
    want = O.orthogonalize(u)
    out = _ops().Ortho(*shape[1:], shape[0], dtype=BF16).orthogonalize(u)
    assert N.off(out, want) <= 1.25 * N.off(want.to(BF16), want)


@pytest.mark.parametrize("streams", [False, True], ids=["one stream", "a stream each"])
def test_threads_share_a_plan(streams):
    """Four threads, each with its own inputs: the bits that one thread alone gets."""
    size = tokens, dim, vocab = 300, 128, 1500
    ce, orth = _ops().LinearCE(*size, dtype=BF16), _ops().Ortho(130, 200, 2)

    def inputs(k):
        t = torch.randint(0, vocab, (tokens,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(k))
        return _normal(tokens, dim, seed=k).to(BF16), (0.1 * _normal(vocab, dim, seed=k + 9)).to(BF16), t

    given = [inputs(k) for k in range(4)]
    us = [_normal(2, 130, 200, seed=30 + k) for k in range(4)]
    want = [{n: x.clone() for n, x in ce(*given[k]).items()} for k in range(4)]
    want_o = [orth.orthogonalize(u).clone() for u in us]
    torch.cuda.synchronize()
    bad = []

    def work(k):
        try:
            stream = torch.cuda.Stream() if streams else torch.cuda.current_stream()
            with torch.cuda.stream(stream):
                for _ in range(8):
                    out, o = ce(*given[k]), orth.orthogonalize(us[k])
                    stream.synchronize()
                    if not all(torch.equal(out[n], want[k][n]) for n in out) or not torch.equal(o, want_o[k]):
                        bad.append(k)
        except Exception as e:  # noqa: BLE001
            bad.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad, bad
