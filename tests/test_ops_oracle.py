"""The 64-bit values that the operators' GPU tests compare with, checked on the CPU
against closed forms, torch's own cross entropy and differences; and that mistakes
planted in them show."""
import math

import pytest
import torch

import ops_oracle as O


def _problem(tokens=7, dim=5, vocab=11, seed=0):
    gen = torch.Generator().manual_seed(seed)
    h = torch.randn(tokens, dim, generator=gen, dtype=torch.float64)
    w = torch.randn(vocab, dim, generator=gen, dtype=torch.float64)
    t = torch.randint(0, vocab, (tokens,), generator=gen)
    t[::3] = -100
    return h, w, t, torch.rand(tokens, generator=gen, dtype=torch.float64)


@pytest.mark.parametrize("mean", [True, False])
def test_against_torch_cross_entropy(mean):
    h, w, t, _ = _problem()
    h.requires_grad_(), w.requires_grad_()
    e = torch.nn.functional.cross_entropy(h @ w.t(), t, ignore_index=-100,
                                          reduction="mean" if mean else "sum")
    e.backward()
    o = O.linear_ce(h.detach(), w.detach(), t, mean=mean)
    torch.testing.assert_close(o["total"], e.detach(), rtol=1e-13, atol=1e-13)
    torch.testing.assert_close(o["dh"], h.grad, rtol=1e-12, atol=1e-13)
    torch.testing.assert_close(o["dw"], w.grad, rtol=1e-12, atol=1e-13)


def test_weights_are_gradients_of_the_tokens_losses():
    h, w, t, c = _problem(seed=1)
    o = O.linear_ce(h, w, t, weight=c, mean=False)
    d = torch.randn(h.shape, generator=torch.Generator().manual_seed(2), dtype=torch.float64)
    step = 1e-6
    up = O.linear_ce(h + step * d, w, t, weight=c, mean=False)["total"]
    down = O.linear_ce(h - step * d, w, t, weight=c, mean=False)["total"]
    assert abs((up - down) / (2 * step) - (o["dh"] * d).sum()) < 1e-7


def test_one_word_has_no_loss_and_equal_logits_have_log_v():
    h, w, _, _ = _problem()
    one = O.linear_ce(h, w[:1], torch.zeros(7, dtype=torch.int64))
    assert one["loss"].abs().max() == 0 and one["dh"].abs().max() == 0
    flat = O.linear_ce(torch.zeros_like(h), w, torch.arange(7))
    torch.testing.assert_close(flat["loss"], torch.full((7,), math.log(11), dtype=torch.float64))


@pytest.mark.parametrize("shape", [(3, 5), (5, 3), (4, 4), (1, 6)])
def test_iteration_is_a_polynomial_of_the_singular_values(shape):
    u = torch.randn(2, *shape, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
    left, s, right = torch.linalg.svd(u / (u.flatten(1).norm(dim=1)[:, None, None] + 1e-7), full_matrices=False)
    a, b, c = O.COEFFS
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    torch.testing.assert_close(O.orthogonalize(u), left @ torch.diag_embed(s) @ right, rtol=1e-10, atol=1e-11)


def test_bounds_are_small_and_a_planted_mistake_passes_none():
    h, w, t, c = _problem(20, 16, 50, seed=4)
    e = O.linear_ce(h, w, t, weight=c)
    for dtype, u_op, u_g in ((torch.float32, O.U_HALVES, O.U_HALVES), (torch.bfloat16, 0.0, O.U_HALF)):
        bound = O.linear_ce_bounds(e, dtype, u_op, u_g)
        for name in ("loss", "dh", "dw"):
            rel = bound[name].norm() / e[name].norm()
            assert rel < (2e-3 if dtype == torch.float32 else 8e-2), (name, float(rel))
        # A left-out column of the vocabulary, a token counted twice, the one-hot
        # entry forgotten.
        wrong = O.linear_ce(h, w[:-1], torch.where(t == 49, -100, t), weight=c)
        assert ((wrong["loss"] - e["loss"]).abs() > bound["loss"])[e["valid"]].any()
        assert ((wrong["dh"] - e["dh"]).abs() > bound["dh"]).any()
        assert ((e["dw"] + e["g"][1][:, None] * h[1] - e["dw"]).abs() > bound["dw"]).any()
    u = torch.randn(1, 20, 30, generator=torch.Generator().manual_seed(5))
    for dtype in (torch.float32, torch.bfloat16):
        bound = float(O.orthogonalize_bound(u, dtype)[0])
        assert bound < (1e-4 if dtype == torch.float32 else 4e-2)
        exact, short = O.orthogonalize(u), O.orthogonalize(u, steps=4)
        assert (exact - short).norm() / exact.norm() > bound
        cut = u.clone()
        cut[:, :, -1] = 0
        assert (exact - O.orthogonalize(cut)).norm() / exact.norm() > bound
