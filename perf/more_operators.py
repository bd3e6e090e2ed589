"""Timed cases of the operators that a block of a language model trains and answers
with, up to the optimizer path: the linear layer with bias, activation and residual,
the norms around a block with its gate and residual scale, and the clipping of
gradients by their global norm.  Each with its gradients.

linear: z = x w^T + bias for x (tokens, dim) and w (wide, dim); y = act(z) +
residual.  Backward, z given: dz = dy act'(z); dx = dz w; dw = dz^T x; dbias = the
tokens' sum of dz.

norm: p = post(f); s = h + scale gate p; y = norm(s), or of h itself where there is
no f.  A norm is "layer", (v - mean) / sqrt(var + eps) weight + bias, "rms", v /
sqrt(mean of squares + eps) weight, or none.  Backward, from dy and from ds, the
gradient that s has from further on: dh, df and those of all vectors.

clip: for each group of tensors, norm = the 2-norm of all their entries and g <- g
min(1, max_norm / (norm + 1e-6)), in place.
"""
import math

import torch

own = False

VOCAB, CONTEXT = 50257, 1024
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS, CLIP_EPS = 1e-5, 1e-6
WIDTHS = (768, 1024, 1280, 1600)
TANH_A, TANH_B = math.sqrt(2 / math.pi), 0.044715


def _linear(name, way, tokens, dim, wide, dtype, act="none", residual=False, dw32=False):
    return dict(name=name, op="linear", way=way, tokens=tokens, dim=dim, wide=wide, dtype=dtype, act=act,
                residual=residual, dw32=dw32)


def _norm(name, way, tokens, dim, dtype, norm="layer", post="none", gate=False, scale=1.0, branch=True):
    return dict(name=name, op="norm", way=way, tokens=tokens, dim=dim, dtype=dtype, norm=norm, post=post, gate=gate,
                scale=scale, branch=branch)


def _clip(name, model, width, layers, workers, dtype, clipped=True):
    return dict(name=name, op="clip", model=model, width=width, layers=layers, workers=workers, dtype=dtype,
                clipped=clipped)


def listed():
    return [
        # One token's feed-forward input in the xl workload's layer: answering.
        _linear("one_token", "forward", 1, 1600, 6400, "bf16", act="gelu_tanh"),
        # Its output for 24 sequences that answer side by side, onto the residual.
        _linear("few_tokens", "forward", 24, 6400, 1600, "bf16", residual=True),
        # Eight contexts through the xl workload's feed-forward input.
        _linear("forward_xl", "forward", 8 * CONTEXT, 1600, 6400, "bf16", act="gelu_tanh"),
        # Its gradients, four contexts, a length that fits no tile.
        _linear("backward_xl", "backward", 4 * CONTEXT - 3, 1600, 6400, "bf16", act="gelu_tanh"),
        # The small workload's attention inputs, dw in the arenas' type.
        _linear("backward_small", "backward", 4 * CONTEXT, 768, 2304, "bf16", dw32=True),
        # A layer in fp32 as the arenas keep it, odd tokens.
        _linear("backward_f32", "backward", 2045, 1024, 4096, "f32", act="relu"),
        # One token's norm after the attention: answering.
        _norm("norm_one_token", "forward", 1, 1600, "bf16"),
        # Eight contexts between two blocks of the xl workload.
        _norm("norm_forward_xl", "forward", 8 * CONTEXT, 1600, "bf16"),
        # Their gradients, norms on both sides of the block and a gate.
        _norm("norm_backward_xl", "backward", 8 * CONTEXT, 1600, "bf16", norm="rms", post="rms", gate=True, scale=0.5),
        # An odd width in fp32.
        _norm("norm_ragged_f32", "backward", 333, 1001, "f32", post="layer", gate=True),
        # A probe model's gradients, odd shapes.
        _clip("clip_probe", "probe", 100, 2, 1, "bf16"),
        # Two workers' gradients of the small workload, a norm for each.
        _clip("clip_small", "gpt", 768, 12, 2, "f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("linear", "linear", "linear", "norm", "norm", "clip"))
    dtype = rng.choice(("f32", "bf16"))
    way = rng.choice(("forward", "backward"))
    if op == "linear":
        dim, wide = (rng.choice(WIDTHS + (2304, 4096, 4800, 5120, 6400, _log(rng, 16, 6400), _log(rng, 16, 6400)))
                     for _ in range(2))
        most = 8 * CONTEXT * 1600 * 6400 // (dim * wide * (2 if way == "backward" else 1))
        tokens = max(1, min(_log(rng, 1, 8 * CONTEXT), most))
        c = _linear("", way, tokens, dim, wide, dtype, act=rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu")),
                    residual=way == "forward" and rng.random() < 0.4,
                    dw32=way == "backward" and dtype == "bf16" and rng.random() < 0.5)
    elif op == "norm":
        branch = rng.random() < 0.8
        dim = rng.choice(WIDTHS + (_log(rng, 16, 6400), _log(rng, 16, 6400)))
        tokens = min(_log(rng, 1, 8 * CONTEXT), 8 * CONTEXT * 1600 // dim)
        c = _norm("", way, tokens, dim, dtype, norm=rng.choice(("layer", "rms")),
                  post=rng.choice(("none", "layer", "rms")) if branch else "none", gate=branch and rng.random() < 0.5,
                  scale=rng.choice((1.0, 0.5)) if branch else 1.0, branch=branch)
    else:
        model = rng.choice(("gpt", "probe"))
        width = _log(rng, 32, 768) if model == "gpt" else _log(rng, 17, 900)
        c = _clip("", model, width, _log(rng, 1, 12), rng.choice((1, 2)), dtype, clipped=rng.random() < 0.7)
    del c["name"]
    return c


def _shapes(case):
    """The shapes of a worker's tensors."""
    d = case["width"]
    if case["model"] == "probe":
        return [(1009, d)] + [s for _ in range(case["layers"]) for s in ((2 * d + 1, d), (2 * d + 1,), (d, 2 * d + 1), (d,))]
    layer = [(d,), (d,), (d, 3 * d), (3 * d,), (d, d), (d,), (d,), (d,), (d, 4 * d), (4 * d,), (4 * d, d), (d,)]
    return [(VOCAB, d), (CONTEXT, d)] + case["layers"] * layer + [(d,), (d,)]


def _ops():
    from paper_2411_17866_amd import ops
    return ops


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, sigma=1.0, mean=0.0):
        return torch.empty(shape, device="cuda").normal_(mean, sigma, generator=gen)

    s = dict(case=case)
    if case["op"] == "linear":
        T, D, N = case["tokens"], case["dim"], case["wide"]
        s.update(x=normal(T, D).to(dtype), w=normal(N, D, sigma=1.0 / math.sqrt(D)).to(dtype))
        if case["way"] == "forward":
            s.update(bias=normal(N, sigma=0.1), residual=normal(T, N).to(dtype) if case["residual"] else None)
        else:
            # Gradients of a mean loss; some tokens' are far smaller than others'.
            size = torch.exp(normal(T, 1)) * (1e-3 / T)
            s.update(dy=(normal(T, N) * size).to(dtype), z=normal(T, N).to(dtype) if case["act"] != "none" else None)
        if own:
            s["plan"] = _ops().Linear(T, D, N, dtype=dtype, act=case["act"], grads=case["way"] == "backward",
                                      dw_dtype=torch.float32 if case["dw32"] else dtype)
    elif case["op"] == "norm":
        T, D = case["tokens"], case["dim"]
        # A residual stream has a few channels that are much larger than the others.
        spread = 1.0 + 20.0 * (torch.rand(D, device="cuda", generator=gen) < 0.01).float()
        s.update(h=((normal(T, D) + 0.3) * spread).to(dtype), weight=normal(D, sigma=0.1, mean=1.0),
                 bias=normal(D, sigma=0.1) if case["norm"] == "layer" else None, f=None, gate=None, post_weight=None,
                 post_bias=None)
        if case["branch"]:
            s["f"] = (normal(T, D) * 2.0 + 0.1).to(dtype)
            if case["gate"]:
                s["gate"] = normal(D, sigma=0.3, mean=0.5)
            if case["post"] != "none":
                s["post_weight"] = normal(D, sigma=0.1, mean=1.0)
            if case["post"] == "layer":
                s["post_bias"] = normal(D, sigma=0.1)
        if case["way"] == "backward":
            s.update(dy=normal(T, D, sigma=1e-3).to(dtype), ds=normal(T, D, sigma=1e-3).to(dtype) if case["branch"] else None)
        if own:
            s["plan"] = _ops().ResidualNorm(T, D, dtype=dtype, norm=case["norm"], post=case["post"], eps=EPS,
                                            grads=case["way"] == "backward")
    else:
        shapes = _shapes(case)
        each = sum(math.prod(shape) for shape in shapes)
        flat = normal(case["workers"], each, sigma=1e-3)
        # A few rows of the embedding hold most of it; the workers differ.
        flat[:, :16 * case["width"]] *= 30.0
        flat *= torch.arange(1, case["workers"] + 1, device="cuda")[:, None]
        norm = flat.double().square().sum(1).sqrt()
        s["max_norm"] = float(norm.min()) * 0.37 if case["clipped"] else float(norm.max()) * 2.0
        flat = flat.to(dtype)
        tensors, groups = [], []
        for worker in range(case["workers"]):
            at = 0
            for shape in shapes:
                n = math.prod(shape)
                tensors.append(flat[worker, at:at + n].view(shape))
                groups.append(worker)
                at += n
        s.update(flat=flat, tensors=tensors, groups=groups)
        if own:
            s["plan"] = _ops().GradClip(tensors, groups=groups, eps=CLIP_EPS)
    return s


def _act(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(TANH_A * (z + TANH_B * z * z * z)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(TANH_A * (z + TANH_B * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * TANH_A * (1 + 3 * TANH_B * z * z)
    share = 1 / (1 + torch.exp(-z))
    return share * (1 + z * (1 - share))


def _plain_linear(s):
    case = s["case"]
    x, w = s["x"].float(), s["w"].float()
    dtype = s["x"].dtype
    if case["way"] == "forward":
        z = x @ w.t() + s["bias"]
        y = _act(case["act"], z)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(dtype)}
    dz = s["dy"].float()
    if case["act"] != "none":
        dz = dz * _slope(case["act"], s["z"].float())
    return {"dx": (dz @ w).to(dtype), "dw": (dz.t() @ x).to(torch.float32 if case["dw32"] else dtype), "dbias": dz.sum(0)}


def _hat(kind, v):
    """(v standardised, 1 / its size)."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)
    return v * r, r


def _hat_grad(kind, d, hat, r):
    d = d - hat * (d * hat).mean(1, keepdim=True)
    return r * (d - d.mean(1, keepdim=True) if kind == "layer" else d)


def _post(s, f):
    """(p, f standardised, 1 / its size)."""
    if s["case"]["post"] == "none":
        return f, None, None
    hat, r = _hat(s["case"]["post"], f)
    p = hat * s["post_weight"]
    return (p if s["post_bias"] is None else p + s["post_bias"]), hat, r


def _plain_norm(s):
    case, dtype = s["case"], s["h"].dtype
    scale = case["scale"]
    if case["way"] == "forward":
        out, v = {}, s["h"].float()
        if case["branch"]:
            p, _, _ = _post(s, s["f"].float())
            v = v + scale * (p if s["gate"] is None else p * s["gate"])
            out["s"] = v.to(dtype)
        y = _hat(case["norm"], v)[0] * s["weight"]
        out["y"] = (y if s["bias"] is None else y + s["bias"]).to(dtype)
        return out
    dy = s["dy"].float()
    hat, r = _hat(case["norm"], s["h"].float())
    out = {"dweight": (dy * hat).sum(0)}
    if s["bias"] is not None:
        out["dbias"] = dy.sum(0)
    d = _hat_grad(case["norm"], dy * s["weight"], hat, r)
    if not case["branch"]:
        out["dh"] = d.to(dtype)
        return out
    d = d + s["ds"].float()
    out["dh"] = d.to(dtype)
    p, hat, r = _post(s, s["f"].float())
    dp = scale * d
    if s["gate"] is not None:
        out["dgate"] = (dp * p).sum(0)
        dp = dp * s["gate"]
    if case["post"] != "none":
        out["dpost_weight"] = (dp * hat).sum(0)
        if s["post_bias"] is not None:
            out["dpost_bias"] = dp.sum(0)
        dp = _hat_grad(case["post"], dp * s["post_weight"], hat, r)
    out["df"] = dp.to(dtype)
    return out


def _plain_clip(s):
    squares = [torch.zeros((), device="cuda", dtype=torch.float64) for _ in range(s["case"]["workers"])]
    for t, group in zip(s["tensors"], s["groups"]):
        squares[group] += t.float().square().sum(dtype=torch.float64)
    norm = torch.stack(squares).sqrt()
    factor = (s["max_norm"] / (norm + CLIP_EPS)).clamp(max=1.0).float()
    for t, group in zip(s["tensors"], s["groups"]):
        t.copy_(t.float() * factor[group])
    return {"norm": norm.float(), "g": s["flat"]}


def run(s):
    case = s["case"]
    if case["op"] == "linear":
        if not own:
            return _plain_linear(s)
        if case["way"] == "forward":
            return s["plan"](s["x"], s["w"], bias=s["bias"], residual=s["residual"])
        return s["plan"].backward(s["dy"], s["x"], s["w"], z=s["z"])
    if case["op"] == "norm":
        if not own:
            return _plain_norm(s)
        vectors = dict(weight=s["weight"], bias=s["bias"], gate=s["gate"], scale=case["scale"],
                       post_weight=s["post_weight"], post_bias=s["post_bias"])
        if case["way"] == "forward":
            return s["plan"](s["h"], f=s["f"], **vectors)
        return s["plan"].backward(s["dy"], s["h"], f=s["f"], ds=s["ds"], **vectors)
    if not own:
        return _plain_clip(s)
    return {"norm": s["plan"](s["tensors"], s["max_norm"]), "g": s["flat"]}


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "linear":
        T, D, N = case["tokens"], case["dim"], case["wide"]
        if case["way"] == "forward":
            return {"bytes": size * (T * D + N * D + T * N * (2 if case["residual"] else 1)) + 4 * N, "flops": 2 * T * D * N}
        return {"bytes": size * (2 * T * D + N * D + T * N * (1 if case["act"] == "none" else 2)) +
                (4 if case["dw32"] else size) * N * D + 4 * N, "flops": 4 * T * D * N}
    if case["op"] == "norm":
        moved = (4 if case["branch"] else 2) if case["way"] == "forward" else (3 if not case["branch"] else 6)
        if case["way"] == "backward" and case["branch"] and case["post"] == "none" and not case["gate"]:
            moved = 5  # f is not wanted
        each = 10 if case["way"] == "forward" else 24
        return {"bytes": size * moved * case["tokens"] * case["dim"], "flops": each * case["tokens"] * case["dim"]}
    n = case["workers"] * sum(math.prod(shape) for shape in _shapes(case))
    return {"bytes": size * n * (2 if case["clipped"] else 1), "flops": n * (3 if case["clipped"] else 2)}


def _exact_act(name, z):
    """(the activation, its slope), from their integrals and logistic forms."""
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z)), torch.where(z > 0, 1.0, 0.0).to(z)
    if name == "gelu":
        share = 0.5 * torch.erfc(-z * math.sqrt(0.5))
        return z * share, share + z * torch.exp(-z * z / 2) * math.sqrt(0.5 / math.pi)
    if name in ("gelu_tanh", "silu"):
        at = 2 * TANH_A * (z + TANH_B * z ** 3) if name == "gelu_tanh" else z
        rate = 2 * TANH_A * (1 + 3 * TANH_B * z ** 2) if name == "gelu_tanh" else torch.ones_like(z)
        share = torch.sigmoid(at)
        return z * share, share + z * rate * share * torch.sigmoid(-at)
    return z, torch.ones_like(z)


def _exact_stats(kind, v):
    mean = v.sum(1, keepdim=True) / v.shape[1] if kind == "layer" else torch.zeros_like(v[:, :1])
    var = (v - mean).pow(2).sum(1, keepdim=True) / v.shape[1]
    return mean, (var + EPS).pow(-0.5)


def _exact_back(kind, v, mean, r, d):
    """The gradient of sum(d * (v - mean) r) by v."""
    n = v.shape[1]
    out = d * r - (v - mean) * r.pow(3) * ((d * (v - mean)).sum(1, keepdim=True) / n)
    return out - d.sum(1, keepdim=True) * r / n if kind == "layer" else out


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept

    def wide(name):
        return None if s.get(name) is None else s[name].double()

    if case["op"] == "linear":
        x, w = wide("x"), wide("w")
        if case["way"] == "forward":
            y = torch.addmm(wide("bias"), x, w.t().contiguous())
            y = _exact_act(case["act"], y)[0]
            return {"y": y if s["residual"] is None else y + wide("residual")}
        dz = wide("dy")
        if s["z"] is not None:
            dz = dz * _exact_act(case["act"], wide("z"))[1]
        return {"dx": torch.mm(dz, w), "dw": torch.mm(dz.t().contiguous(), x), "dbias": dz.sum(0)}
    if case["op"] == "clip":
        g = s["flat"].double()
        norm = torch.linalg.vector_norm(g, dim=1)
        return {"norm": norm, "g": g * torch.minimum(s["max_norm"] / (norm + CLIP_EPS), torch.ones_like(norm))[:, None]}
    h, f, scale = wide("h"), wide("f"), case["scale"]
    if f is not None:
        mean_f, r_f = _exact_stats(case["post"], f) if case["post"] != "none" else (0.0, 1.0)
        hat_f = (f - mean_f) * r_f
        p = hat_f if case["post"] == "none" else hat_f * wide("post_weight")
        p = p if s["post_bias"] is None else p + wide("post_bias")
        share = torch.full((case["dim"],), scale, dtype=torch.float64, device="cuda")
        share = share if s["gate"] is None else share * wide("gate")
    if case["way"] == "forward":
        out = {}
        if f is not None:
            h = h + share * p
            out["s"] = h
        mean, r = _exact_stats(case["norm"], h)
        out["y"] = (h - mean) * r * wide("weight") + (0.0 if s["bias"] is None else wide("bias"))
        return out
    dy = wide("dy")
    mean, r = _exact_stats(case["norm"], h)
    out = {"dweight": (dy * (h - mean) * r).sum(0)}
    if s["bias"] is not None:
        out["dbias"] = dy.sum(0)
    d = _exact_back(case["norm"], h, mean, r, dy * wide("weight"))
    if f is None:
        out["dh"] = d
        return out
    d = d + wide("ds")
    out["dh"] = d
    if s["gate"] is not None:
        out["dgate"] = (scale * d * p).sum(0)
    d = share * d
    if case["post"] != "none":
        out["dpost_weight"] = (d * hat_f).sum(0)
        if s["post_bias"] is not None:
            out["dpost_bias"] = d.sum(0)
        d = _exact_back(case["post"], f, mean_f, r_f, d * wide("post_weight"))
    out["df"] = d
    return out
