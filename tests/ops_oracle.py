"""64-bit values of the language-model operators, and how far a result may be
from them.

The values come from the operators' definitions, in float64 with torch's plain
operations on whichever device the inputs are; nothing here uses the library.

Bounds.  The cross entropy's are a priori and elementwise: an operand carries
`u_op` relative (0 for operands used as they are, and for bf16 numbers as scaled
fp16, which has their bits; 2^-21 for two fp16 halves with the lo lo products left
out), G `u_g` (2^-11 for one fp16, 2^-16 for two bf16 halves), a sum of K products adds at
most K 2^-23 of the sum of their magnitudes (whatever the order, additions may
truncate), and the rest follows the formulas.  The iteration's is measured on the
definition: every stored operand is perturbed by random relative errors of the
size that its storage may make, and the result may be four times as far off as
that puts it.
"""
import torch

COEFFS = (3.4445, -4.7750, 2.0315)
U_HALF, U_HALVES, U_BF16_HALVES = 2.0 ** -11, 2.0 ** -21, 2.0 ** -16
U_OUT = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}


def linear_ce(h, w, target, weight=None, mean=True):
    """total, loss, lse, dh, dw, and the G they come from."""
    h, w = h.double(), w.double()
    vocab = w.shape[0]
    valid = (target >= 0) & (target < vocab)
    h = torch.where(valid[:, None], h, torch.zeros_like(h))
    at = torch.where(valid, target, torch.zeros_like(target))[:, None]
    c = valid.double() if weight is None else torch.where(valid, weight.double(), 0.0)
    if mean:
        c = c / max(int(valid.sum()), 1)
    z = h @ w.t().contiguous()
    lse = torch.logsumexp(z, 1)
    loss = torch.where(valid, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    g = torch.exp(z - lse[:, None])
    g.scatter_add_(1, at, -torch.ones_like(g[:, :1]))
    g = torch.where(valid[:, None], g * c[:, None], torch.zeros_like(g))
    return dict(total=torch.where(valid, loss * c, 0.0).sum(), loss=loss, lse=lse, dh=g @ w,
                dw=g.t().contiguous() @ h, g=g, z=z, c=c, valid=valid, h=h, w=w)


def linear_ce_bounds(e, dtype, u_op, u_g):
    """Elementwise bounds for loss, total, dh and dw of linear_ce's values `e`:
    u_op of h and w in the logits and in the products of G, u_g of G."""
    h, w, c = e["h"].abs(), e["w"].abs(), e["c"].abs()
    dim, tokens, vocab = h.shape[1], h.shape[0], w.shape[0]
    # Logits: operands, the sum, the scaling.
    dz = (2 * u_op + dim * 2.0 ** -23) * (h @ w.t().contiguous()) + 2.0 ** -23 * e["z"].abs()
    worst = dz.max(1).values
    # lse: the worst logit, the sum of V exponentials, log2 and its rounding.
    d_lse = worst + vocab * 2.0 ** -23 + 2.0 ** -22 * (e["lse"].abs() + e["z"].abs().max(1).values + 1)
    d_loss = torch.where(e["valid"], d_lse + worst + 2.0 ** -22 * (e["lse"].abs() + 1), torch.zeros_like(worst))
    d_total = (c * d_loss).sum() + 2.0 ** -22 * e["loss"].abs().mul(c).sum()
    # G: the probability's argument and exponential, the subtraction, c, storage.
    p = torch.exp(e["z"] - e["lse"][:, None])
    d_arg = dz + d_lse[:, None] + 2.0 ** -22 * (e["z"].abs() + e["lse"].abs()[:, None] + 1)
    d_g = c[:, None] * p * torch.expm1(d_arg) + (2.0 ** -22 + u_g) * (e["g"].abs() + 2.0 ** -23 * c[:, None])
    # Entries of G below fp16's subnormals of the largest entry vanish.
    d_g = d_g + (2.0 ** -38) * c.max()
    d_dh = d_g @ w + (u_op + vocab * 2.0 ** -23) * (e["g"].abs() @ w)
    d_dw = d_g.t().contiguous() @ h + (u_op + tokens * 2.0 ** -23) * (e["g"].abs().t().contiguous() @ h)
    out = U_OUT[dtype]
    return dict(loss=d_loss, total=d_total, dh=d_dh + out * e["dh"].abs(), dw=d_dw + out * e["dw"].abs())


def orthogonalize(u, steps=5, eps=1e-7, coeffs=None, noise=None, generator=None):
    """The iteration on (count, rows, cols) in float64.  noise = (of X, A and B in
    the products, of X in a X): relative random errors of these sizes."""
    x = u.double()
    wide = x.shape[2] >= x.shape[1]
    x = x if wide else x.transpose(1, 2).contiguous()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + eps)

    def off(v, size):
        if noise is None:
            return v
        return v * (1 + size * (2 * torch.rand(v.shape, generator=generator, dtype=v.dtype, device=v.device) - 1))

    for k in range(steps):
        a, b, c = COEFFS if coeffs is None else (float(v) for v in coeffs[k])
        xq = off(x, noise[0]) if noise else x
        aq = torch.bmm(xq, xq.transpose(1, 2).contiguous())
        aq = off(aq, noise[0]) if noise else aq
        aq = 0.5 * (aq + aq.transpose(1, 2))
        bq = b * aq + c * torch.bmm(aq, aq)
        bq = off(bq, noise[0]) if noise else bq
        x = (a * off(x, noise[1]) if noise else a * x) + torch.bmm(bq, xq)
    return x if wide else x.transpose(1, 2).contiguous()


def orthogonalize_bound(u, dtype, steps=5, eps=1e-7, coeffs=None):
    """How far (2-norm over 2-norm of the result, per matrix) the library's result
    may be from orthogonalize(u)."""
    long = max(u.shape[1], u.shape[2])
    u_sum = long ** 0.5 * 2.0 ** -24
    noise = ((U_HALF if dtype == torch.bfloat16 else U_HALVES) + u_sum, U_HALVES + u_sum)
    gen = torch.Generator(device=u.device).manual_seed(7)
    exact = orthogonalize(u, steps, eps, coeffs)
    off = orthogonalize(u, steps, eps, coeffs, noise, gen)
    size = exact.flatten(1).norm(dim=1).clamp(min=1e-300)
    return 4 * (off - exact).flatten(1).norm(dim=1) / size + U_OUT[dtype]
