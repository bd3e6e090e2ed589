"""64-bit values of the operators of a model's blocks, and how far a result may be
from them.

Values come from the operators' definitions, in float64 with torch's plain operations
on whichever device the inputs are; nothing here uses the library.

Bounds are a priori.  U is half a step of fp32 (2^-24); a result's own rounding is half
a step of its type, HALF.  A sum of K products adds at most K 2^-23 of the sum of their
magnitudes (whatever the order; additions may truncate); operands as two fp16 halves
carry 2^-21 (the lo lo products left out included) and vanish below 2^-39 of the largest
one that shares their power of two.  Sums over a row of the norms run over 8 columns in a
lane, 6 exchanges and at most 16 waves, each a rounding.  A gradient through an
activation in bf16 carries one more rounding to bf16, dz's.

Since K 2^-23 is loose for long sums, whole results are also held to what roundings that
are independent add up to (norm_bound): partial sums of K random terms err by
2^-23 sqrt(K / 2) of the result.
"""
import math

import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
HALVES, VANISH = 2.0 ** -21, 2.0 ** -39
# exp2, reciprocal and erfc of the activations, relative to |z| or the slope.
ACT = 2.0 ** -19
ROW = 8 + 6 + 16 + 10  # roundings of a row's sum and what follows it


def act(name, z):
    """(the activation of z, its slope)."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if name == "gelu":
        share = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * share, share + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "silu":
        share = torch.sigmoid(z)
        return z * share, share + z * share * torch.sigmoid(-z)
    a, b = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(a * (z + b * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * b * z * z)


def linear(x, w, bias=None, residual=None, name="none"):
    """y and z."""
    z = x.double() @ w.double().t().contiguous()
    if bias is not None:
        z = z + bias.double()
    y = act(name, z)[0]
    return {"y": y if residual is None else y + residual.double(), "z": z}


def linear_bounds(x, w, bias, residual, name, few):
    """Elementwise, of y and z."""
    dtype = x.dtype
    x, w = x.double(), w.double()
    e = linear(x, w, bias, residual, name)
    sizes = x.abs() @ w.abs().t().contiguous()
    u = 0.0 if dtype == torch.bfloat16 or few else HALVES
    dz = (2 * u + (x.shape[1] + 2) * 2 * U) * sizes + 4 * U * e["z"].abs()
    if u:
        dz = dz + VANISH * (x.abs().amax(1)[:, None] * w.abs().sum(1) + x.abs().sum(1)[:, None] * w.abs().amax(1))
    dy = 1.13 * dz + 4 * U * e["y"].abs()  # (no slope is steeper)
    if name not in ("none", "relu"):
        dy = dy + ACT * e["z"].abs()
    if residual is not None:
        dy = dy + 2 * U * residual.double().abs()
    half = HALF[dtype]
    return {"y": dy * (1 + half) + half * e["y"].abs(), "z": dz * (1 + half) + half * e["z"].abs()}


def linear_backward(dy, x, w, z=None, name="none"):
    dz = dy.double()
    if name != "none":
        dz = dz * act(name, z.double())[1]
    return {"dz": dz, "dx": dz @ w.double(), "dw": dz.t().contiguous() @ x.double(), "dbias": dz.sum(0)}


def linear_backward_bounds(e, dy, x, w, name, dw_dtype):
    """Elementwise, of dx, dw and dbias of linear_backward's values e."""
    dtype = x.dtype
    x, w, dz, dy = x.double().abs(), w.double().abs(), e["dz"].abs(), dy.double().abs()
    u = 0.0 if dtype == torch.bfloat16 else HALVES
    d = torch.zeros_like(dz) if name == "none" else (0.0 if name == "relu" else ACT) * dy + 2 * U * dz
    rounded = name != "none" and dtype == torch.bfloat16
    halves = HALF[dtype] ** 2 if dw_dtype == torch.float32 else HALF[dtype]  # of a bf16 dz in dw: two of them
    dx = (d + (HALF[dtype] * (dz + d) if rounded else 0.0)) @ w + (2 * u + (w.shape[0] + 2) * 2 * U) * (dz @ w)
    dw = (d + (halves * (dz + d) if rounded else 0.0)).t().contiguous() @ x
    dw = dw + (2 * u + (x.shape[0] * (2 if rounded else 1) + 2) * 2 * U) * (dz.t().contiguous() @ x)
    if u:
        dx = dx + VANISH * (dz.amax(1)[:, None] * w.sum(0) + dz.sum(1)[:, None] * w.max())
        each = dz.amax(1) * x.amax(1)  # what a token's rows make together
        dw = dw + VANISH * ((dz.amax(1)[:, None] * x).sum(0)[None, :] + dz.shape[0] * each.max())
    db = d.sum(0) + (dz.shape[0] + 2) * 2 * U * dz.sum(0)
    return {"dx": dx + HALF[dtype] * (dx + e["dx"].abs()), "dw": dw + HALF[dw_dtype] * (dw + e["dw"].abs()), "dbias": db}


def norm_bound(terms, dtype, roundings=1):
    """Of the 2-norm of the error over that of the result, where a result of many entries is a sum of
    `terms` random terms: independent roundings of at most half a step, spread evenly."""
    return 2 * U * (2 + math.sqrt(terms / 2)) + HALF[dtype] * math.sqrt(roundings / 3) * 1.1


def check(out, values, bounds, names):
    for name in names:
        got, want = out[name].double(), values[name]
        assert got.shape == want.shape, name
        assert torch.isfinite(got).all(), name
        far = (got - want).abs() - bounds[name]
        assert (far <= 0).all(), f"{name}: {int((far > 0).sum())} of {far.numel()} outside, by {float(far.max()):.3g}"


def check_norm(got, want, bound, name):
    off = float((got.double() - want).norm() / want.norm())
    assert off <= bound, f"{name}: {off:.3g} > {bound:.3g}"


# ---- Norms ----

def standard(kind, v, eps):
    """(standardised v, 1 / its size)."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = 1 / torch.sqrt(v.square().mean(1, keepdim=True) + eps)
    return v * r, r


def back(kind, d, hat, r):
    d = d - hat * (d * hat).mean(1, keepdim=True)
    return r * (d - d.mean(1, keepdim=True) if kind == "layer" else d)


def _wide(t, otherwise, like):
    return torch.full_like(like[0], otherwise) if t is None else t.double()


def residual_norm(h, f=None, weight=None, bias=None, gate=None, scale=1.0, post_weight=None, post_bias=None,
                  norm="layer", post="none", eps=1e-5, post_eps=1e-5):
    """s, y, and p, and bounds of s and y, elementwise."""
    dtype, h = h.dtype, h.double()
    half = HALF[dtype]
    out, s, off = {}, h, torch.zeros_like(h)
    if f is not None:
        p, dp = f.double(), torch.zeros_like(h)
        if post != "none":
            pw, pb = _wide(post_weight, 1.0, h), _wide(post_bias, 0.0, h)
            size = p.abs().mean(1, keepdim=True)
            hat, r = standard(post, p, post_eps)
            p = hat * pw + pb
            dp = ROW * 2 * U * (hat.abs() * (1 + r * size) + r * size) * pw.abs() + 4 * U * (p.abs() + pb.abs())
        share = scale * _wide(gate, 1.0, h)
        s = h + share * p
        off = share.abs() * (dp + 4 * U * p.abs()) + 2 * U * (h.abs() + s.abs())
        out.update(s=s, p=p, s_bound=off + half * (s.abs() + off))
    if norm != "none":
        size = s.abs().mean(1, keepdim=True)
        hat, r = standard(norm, s, eps)
        w, b = _wide(weight, 1.0, h), _wide(bias, 0.0, h)
        y = hat * w + b
        # s is off by `off`, which hat follows (and, through mean and size, its neighbours').
        most = off.mean(1, keepdim=True)
        d = r * (off + most * (1 + hat.abs())) + ROW * 2 * U * (hat.abs() * (1 + r * size) + r * size)
        d = d * w.abs() + 4 * U * (y.abs() + b.abs())
        out.update(y=y, y_bound=d + half * (y.abs() + d))
    return out


def residual_norm_backward(dy, s, f=None, ds=None, weight=None, bias=None, gate=None, scale=1.0, post_weight=None,
                           post_bias=None, norm="layer", post="none", eps=1e-5, post_eps=1e-5):
    """The gradients, and their bounds under name + "_bound"."""
    like = s if s is not None else ds
    dtype, half = like.dtype, HALF[like.dtype]
    tokens = like.shape[0]
    out = {}

    def total(name, terms, off):
        out[name] = terms.sum(0)
        out[name + "_bound"] = off.sum(0) + (tokens + 2) * 2 * U * (terms.abs() + off).sum(0)

    def through(kind, e, e_off, v, r, hat):
        """The gradient through a norm of v, and its bound."""
        size = 1 + r * v.abs().mean(1, keepdim=True)  # what v's own size costs v - mean
        d = back(kind, e, hat, r)
        bulk = e.abs() + hat.abs() * (e * hat).abs().mean(1, keepdim=True) + e.abs().mean(1, keepdim=True)
        bulk = bulk + (e.abs().mean(1, keepdim=True) * (1 + hat.abs()))
        off = e_off + hat.abs() * (e_off * hat.abs()).mean(1, keepdim=True) + e_off.mean(1, keepdim=True)
        return d, r * (ROW * 4 * U * size * bulk + off)

    d = torch.zeros(like.shape, dtype=torch.float64, device=like.device)
    off = torch.zeros_like(d)
    if norm != "none":
        g, v = dy.double(), s.double()
        hat, r = standard(norm, v, eps)
        hat_off = ROW * 2 * U * (hat.abs() + 1) * (1 + r * v.abs().mean(1, keepdim=True))
        if weight is not None:
            total("dweight", g * hat, g.abs() * hat_off)
        if bias is not None:
            total("dbias", g, torch.zeros_like(g))
        e = g * _wide(weight, 1.0, v)
        d, off = through(norm, e, 2 * U * e.abs(), v, r, hat)
    if ds is not None:
        d = d + ds.double()
        off = off + 2 * U * (d.abs() + ds.double().abs())
    out["dh"], out["dh_bound"] = d, off + half * (d.abs() + off)
    if f is None:
        return out
    v = f.double()
    p, p_off = v, torch.zeros_like(v)
    pw = _wide(post_weight, 1.0, v)
    if post != "none":
        hat, r = standard(post, v, post_eps)
        hat_off = ROW * 2 * U * (hat.abs() + 1) * (1 + r * v.abs().mean(1, keepdim=True))
        p = hat * pw + _wide(post_bias, 0.0, v)
        p_off = hat_off * pw.abs() + 4 * U * p.abs() + 4 * U * _wide(post_bias, 0.0, v).abs()
    if gate is not None:
        total("dgate", scale * d * p, abs(scale) * (off * p.abs() + d.abs() * p_off + 4 * U * (d * p).abs()))
    share = scale * _wide(gate, 1.0, v)
    d, off = share * d, share.abs() * (off + 4 * U * d.abs())
    if post != "none":
        if post_weight is not None:
            total("dpost_weight", d * hat, off * hat.abs() + d.abs() * hat_off)
        if post_bias is not None:
            total("dpost_bias", d, off)
        e = d * pw
        d, off = through(post, e, off * pw.abs() + 2 * U * e.abs(), v, r, hat)
    out["df"], out["df_bound"] = d, off + half * (d.abs() + off)
    return out


# ---- Clipping ----

def clip(tensors, groups, max_norm, eps=1e-6):
    """(norms, clipped tensors)."""
    norms = [math.sqrt(sum(float(t.double().square().sum()) for t, g in zip(tensors, groups) if g == k))
             for k in range(max(groups, default=0) + 1)]
    factor = [min(1.0, max_norm / (n + eps)) if math.isfinite(n) and n + eps > 0 else 1.0 for n in norms]
    return norms, [t.double() * factor[g] for t, g in zip(tensors, groups)]
