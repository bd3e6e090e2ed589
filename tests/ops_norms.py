"""Norm-wise checks of the operators at sizes where the elementwise bounds of
ops_oracle, which grow with the vocabulary, would let a mistake pass.

Tolerances.  A logit is off by rounding: of fp32 sums of `dim` terms (random in sign,
2^-24 sqrt(dim) / 3 of the logit's size), and for fp32 many-token forms of operands of
22 bits.  At dim up to 1600 and logits of some units that is some 1e-6, the relative
error of a softmax entry; loss, a mean over the vocabulary's errors plus the target's
own, keeps that absolutely, against losses of about log(vocab).  Hence 2-norms relative
to the result's own: losses 2e-6, fp32 gradients 5e-6.  Rounding a gradient to bf16
costs 2^-9 / sqrt(3) of it or up to 1.5 times that (0.0011 to 0.0017, by where mantissas
lie), and G's 11 bits another 2^-12: 4e-3.
"""
import torch

LOSS, GRAD = 2e-6, {torch.float32: 5e-6, torch.bfloat16: 4e-3}


def linear_ce(h, w, target, weight=None, mean=True, grads=True, block=1 << 25):
    """total, loss, dh and dw in float64, some rows of logits at a time."""
    tokens, vocab = h.shape[0], w.shape[0]
    h, w = h.double(), w.double()
    valid = (target >= 0) & (target < vocab)
    c = valid.double() if weight is None else torch.where(valid, weight.double(), 0.0)
    if mean:
        c = c / max(int(valid.sum()), 1)
    wt = w.t().contiguous()
    out = dict(loss=torch.zeros(tokens, dtype=torch.float64, device=h.device), valid=valid)
    if grads:
        out.update(dh=torch.zeros_like(h), dw=torch.zeros_like(w))
    step = max(1, block // vocab)
    for lo in range(0, tokens, step):
        rows = torch.arange(lo, min(tokens, lo + step), device=h.device)[valid[lo:lo + step]]
        if not len(rows):
            continue
        z = h[rows] @ wt
        pick = torch.arange(len(rows), device=h.device)
        top = z.max(1, keepdim=True).values
        hit = z[pick, target[rows]]
        e = (z - top).exp_()
        size = e.sum(1)
        # log(1 + others / target): digits where the target is nearly sure.
        rest = size - e[pick, target[rows]]
        sure = (hit - top[:, 0]) > -1.0
        e[pick, target[rows]] = 0
        rest = torch.where(sure, e.sum(1), rest)
        out["loss"][rows] = torch.where(sure, torch.log1p(rest / (hit - top[:, 0]).exp()),
                                        size.log() + top[:, 0] - hit)
        if grads:
            e /= size[:, None]
            e[pick, target[rows]] = -rest / size
            e *= c[rows][:, None]
            out["dh"][rows] = e @ w
            out["dw"] += e.t().contiguous() @ h[rows]
    out["total"] = (out["loss"] * c).sum()
    return out


def off(got, want):
    return float((got.double() - want).norm() / want.norm().clamp(min=1e-300))


def check_linear_ce(out, e, target, dtype, grads=True, loss_tol=LOSS):
    """out against e: losses, their total, dh of the tokens that count, and dw of words
    that are targets and of words that are not, by itself."""
    vocab = e["dw"].shape[0] if grads else None
    assert (out["loss"][~e["valid"]] == 0).all()
    figures = {"loss": (off(out["loss"], e["loss"]), loss_tol),
               "total": (abs(float(out["total"]) - float(e["total"])) / abs(float(e["total"])), loss_tol)}
    if grads:
        hit = torch.zeros(vocab, dtype=torch.bool, device=target.device)
        hit[target[e["valid"]]] = True
        assert (out["dh"][~e["valid"]] == 0).all()
        figures["dh"] = (off(out["dh"], e["dh"]), GRAD[dtype])
        for name, rows in (("dw of targets", hit), ("dw of other words", ~hit)):
            if rows.any():
                figures[name] = (off(out["dw"][rows], e["dw"][rows]), GRAD[dtype])
    bad = {k: v for k, v in figures.items() if not v[0] <= v[1]}
    assert not bad, f"{bad} of {figures}"
