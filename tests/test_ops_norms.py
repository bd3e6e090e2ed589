"""The norm-wise checks of ops_norms.py on the CPU: plain fp32 arithmetic passes them, and
mistakes planted at a large vocabulary do not."""
import pytest
import torch

import ops_norms as N
import ops_oracle as O

TOKENS, DIM, VOCAB = 300, 64, 20011


@pytest.fixture(scope="module")
def problem():
    gen = torch.Generator().manual_seed(1)
    h = torch.randn(TOKENS, DIM, generator=gen)
    w = torch.randn(VOCAB, DIM, generator=gen) * DIM ** -0.5
    t = torch.randint(0, VOCAB, (TOKENS,), generator=gen)
    t[::10] = -1
    c = 0.5 + torch.rand(TOKENS, generator=gen)
    return h, w, t, c, N.linear_ce(h, w, t, c)


def _plain(h, w, t, c, dtype=torch.float32, g_as=None, words=slice(None), dh_words=slice(None), dw_scale=1.0):
    """fp32 arithmetic as the operator does it; `words` enter the statistics, `dh_words`
    the sums of dh; G is stored as g_as."""
    h, w = h.to(dtype).float(), w.to(dtype).float()
    valid = (t >= 0) & (t < VOCAB)
    at = t.clamp(min=0)
    z = h @ w.t()
    lse = torch.logsumexp(z[:, words], 1)
    loss = torch.where(valid, lse - z.gather(1, at[:, None])[:, 0], 0.0)
    share = torch.where(valid, c, 0.0) / valid.sum()
    p = torch.exp(z - lse[:, None]) * share[:, None] * dw_scale
    g = p.scatter_add(1, at[:, None], -share[:, None])
    if g_as is not None:
        g = g.to(g_as).float()
    return dict(loss=loss, total=(loss * share).sum(), dh=(g[:, dh_words] @ w[dh_words]).to(dtype),
                dw=(g.t() @ h).to(dtype))


def test_the_two_64_bit_forms_agree(problem):
    h, w, t, c, e = problem
    o = O.linear_ce(h, w, t, weight=c)
    for name in ("total", "loss", "dh", "dw"):
        torch.testing.assert_close(e[name], o[name], rtol=1e-11, atol=1e-15)


def test_losses_of_sure_rows_keep_their_digits():
    h = torch.tensor([[30.0, 0.0]], dtype=torch.float64)
    w = torch.tensor([[1.0, 0.0], [0.0, 1.0]], dtype=torch.float64)
    e = N.linear_ce(h, w, torch.tensor([0]))
    want = torch.log1p(torch.exp(torch.tensor(-30.0, dtype=torch.float64)))
    torch.testing.assert_close(e["loss"][0], want, rtol=1e-12, atol=0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_plain_arithmetic_passes(problem, dtype):
    h, w, t, c, _ = problem
    e = N.linear_ce(h.to(dtype), w.to(dtype), t, c)
    N.check_linear_ce(_plain(h, w, t, c, dtype), e, t, dtype)


@pytest.mark.parametrize("mistake", [
    dict(words=slice(256, None)),       # a tile of words left out of the statistics
    dict(words=slice(0, VOCAB - 43)),   # the last, partial tile
    dict(dh_words=slice(256, None)),    # a tile left out of dh
    dict(g_as=torch.bfloat16),          # G of 8 bits
    dict(dw_scale=0.0),                 # no softmax part in the gradients
    dict(dw_scale=1.001),
])
def test_planted_mistakes_fail(problem, mistake):
    h, w, t, c, e = problem
    with pytest.raises(AssertionError):
        N.check_linear_ce(_plain(h, w, t, c, **mistake), e, t, torch.float32)


def test_planted_mistakes_fail_in_bf16(problem):
    h, w, t, c, _ = problem
    e = N.linear_ce(h.bfloat16(), w.bfloat16(), t, c)
    for mistake in (dict(words=slice(256, None)), dict(dh_words=slice(256, None)), dict(dw_scale=0.0),
                    dict(dw_scale=1.01)):
        with pytest.raises(AssertionError):
            N.check_linear_ce(_plain(h, w, t, c, torch.bfloat16, **mistake), e, t, torch.bfloat16)
