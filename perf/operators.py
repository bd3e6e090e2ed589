"""Timed cases of the language-model operators beside the optimizer path: the
output layer's cross entropy with its gradients, the orthogonalised update, and
the momentum step that applies it.

linear_ce: logits = h w^T for h (tokens, dim) and the output embedding w (vocab,
dim); per token the loss logsumexp(logits) - logits[target], 0 where the target
is outside [0, vocab) (padding); total = the weighted sum over the tokens, or
over the number of valid ones; with gradients, d total / dh and d total / dw.

orthogonalize: X = U / (||U||_F + 1e-7), five times X <- a X + (b A + c A A) X
with A = X X^T, on the shorter side.

ortho_step: m <- mu m + g; u = g + mu m (Nesterov) or m; x <- x - lr (s O(u) +
wd x), O as above, with m and x updated in place.
"""
import math

import torch

own = False

VOCAB, CONTEXT = 50257, 1024
COEFFS = (3.4445, -4.7750, 2.0315)
STEPS, EPS = 5, 1e-7
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
STEP = dict(lr=0.02, mu=0.95, wd=0.1)


def _ce(name, tokens, dim, vocab, dtype, grads, mean=True, weighted=False, ignored=0.0):
    return dict(name=name, op="linear_ce", tokens=tokens, dim=dim, vocab=vocab, dtype=dtype, grads=grads, mean=mean,
                weighted=weighted, ignored=ignored)


def _ortho(name, rows, cols, count, dtype):
    return dict(name=name, op="orthogonalize", rows=rows, cols=cols, count=count, dtype=dtype)


def _step(name, rows, cols, count, nesterov=True):
    return dict(name=name, op="ortho_step", rows=rows, cols=cols, count=count, dtype="f32", nesterov=nesterov)


def listed():
    return [
        # One token's loss: scoring a continuation token by token.
        _ce("score_one_token", 1, 768, VOCAB, "bf16", False),
        # One full context scored for its perplexity.
        _ce("score_context", CONTEXT, 1600, VOCAB, "bf16", False, ignored=0.02),
        # An odd-sized head of a byte- or character-level model, some padding
        # and a weight for each token, in the arenas' own type.
        _ce("train_ragged", 333, 100, 1009, "f32", True, mean=False, weighted=True, ignored=0.1),
        # A worker's batch on the small workload's head, eight contexts.
        _ce("train_small", 8 * CONTEXT, 768, VOCAB, "bf16", True, ignored=0.02),
        # The xl workload's head, four contexts, a length that fits no tile.
        _ce("train_xl", 4 * CONTEXT - 3, 1600, VOCAB, "bf16", True, weighted=True),
        # The small workload's head in fp32, as the arenas keep parameters.
        _ce("train_f32", 2 * CONTEXT, 768, VOCAB, "f32", True),
        # A single small matrix (a probe model's layer).
        _ortho("one_tiny_matrix", 64, 48, 1, "f32"),
        # The attention projections of the small workload's layers.
        _ortho("projections_bf16", 768, 768, 12, "bf16"),
        # Eight layers' feed-forward matrices of the xl workload, tall.
        _ortho("feed_forward_bf16", 6400, 1600, 8, "bf16"),
        # Matrices that fit no tile, in fp32.
        _ortho("ragged_f32", 333, 1001, 5, "f32"),
        # The small workload's attention inputs, every layer.
        _step("step_small", 768, 2304, 12),
        # Four feed-forward matrices of the large workload, tall, plain momentum.
        _step("step_large", 5120, 1280, 4, nesterov=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("linear_ce", "linear_ce", "orthogonalize", "ortho_step"))
    if op == "linear_ce":
        grads = rng.random() < 0.7
        dtype = rng.choice(("f32", "bf16"))
        dim = rng.choice((768, 1024, 1280, 1600, _log(rng, 64, 1600)))
        vocab = rng.choice((VOCAB, _log(rng, 256, VOCAB)))
        most = 8 * CONTEXT if dtype == "bf16" else 2 * CONTEXT
        tokens = min(_log(rng, 1, most), most * 768 * VOCAB // (dim * vocab))
        c = _ce("", tokens, dim, vocab, dtype, grads, mean=rng.random() < 0.5, weighted=rng.random() < 0.5,
                ignored=rng.choice((0.0, 0.02, 0.3)))
    else:
        short = rng.choice((768, 1024, 1280, 1600, _log(rng, 16, 1600)))
        long = int(short * rng.choice((1, 1, 3, 4, rng.uniform(1, 4))))
        count = max(1, min(_log(rng, 1, 12), int(4 * 1280 * 1280 * 5120 / (short * short * long))))
        rows, cols = (short, long) if rng.random() < 0.5 else (long, short)
        if op == "orthogonalize":
            c = _ortho("", rows, cols, count, rng.choice(("f32", "bf16")))
        else:
            c = _step("", rows, cols, count, nesterov=rng.random() < 0.5)
    del c["name"]
    return c


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))

    def normal(*shape, sigma=1.0):
        return torch.empty(shape, device="cuda").normal_(0.0, sigma, generator=gen)

    def update(sigma):
        # A gradient's spectrum: a few strong directions over noise.
        rank = min(16, case["rows"], case["cols"])
        strong = normal(case["count"], case["rows"], rank) @ normal(case["count"], rank, case["cols"])
        return sigma * (0.3 * strong + normal(case["count"], case["rows"], case["cols"]))

    dtype = DTYPES[case["dtype"]]
    if case["op"] == "linear_ce":
        T, D, V = case["tokens"], case["dim"], case["vocab"]
        w = normal(V, D, sigma=0.02)
        # Frequent tokens come first; a trained model leans towards the target.
        target = (V * torch.rand(T, device="cuda", generator=gen).pow(3)).long().clamp_(max=V - 1)
        lean = 10.0 * torch.rand(T, 1, device="cuda", generator=gen) / w[target].square().sum(1, keepdim=True)
        h = normal(T, D) + lean * w[target]
        target[torch.rand(T, device="cuda", generator=gen) < case["ignored"]] = -100
        weight = torch.rand(T, device="cuda", generator=gen) if case["weighted"] else None
        state = dict(case=case, h=h.to(dtype), w=w.to(dtype), target=target, weight=weight)
        if own:
            from paper_2411_17866_amd import ops
            state["plan"] = ops.LinearCE(T, D, V, dtype=dtype, grads=case["grads"])
        return state
    shape = (case["count"], case["rows"], case["cols"])
    if case["op"] == "orthogonalize":
        state = dict(case=case, u=update(1e-3).to(dtype))
    else:
        # Momentum of a run under way: the sum of many gradients.
        state = dict(case=case, g=update(1e-3), m=update(3e-3), x=normal(*shape, sigma=0.02))
    if own:
        from paper_2411_17866_amd import ops
        state["plan"] = ops.Ortho(case["rows"], case["cols"], case["count"], dtype=dtype)
    return state


def _scale(case):
    return 0.2 * math.sqrt(max(case["rows"], case["cols"]))


def _plain_ortho(u):
    a, b, c = COEFFS
    x = u.float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    x = _plain_iterate(x, a, b, c)
    return x.transpose(1, 2).contiguous() if tall else x


def _plain_iterate(x, a, b, c, left=STEPS):
    if left == 0:
        return x
    gram = torch.bmm(x, x.transpose(1, 2).contiguous())
    x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return _plain_iterate(x, a, b, c, left - 1)


def _plain_ce(s):
    case, target = s["case"], s["target"]
    h, w = s["h"].float(), s["w"].float()
    valid = (target >= 0) & (target < case["vocab"])
    at = torch.where(valid, target, torch.zeros_like(target)).unsqueeze(1)
    logits = h @ w.t()
    top = logits.max(1, keepdim=True).values
    p = (logits - top).exp_()
    norm = p.sum(1, keepdim=True)
    loss = torch.where(valid, (norm.log() + top - logits.gather(1, at)).squeeze(1), torch.zeros_like(top[:, 0]))
    each = valid.float() if s["weight"] is None else valid.float() * s["weight"]
    if case["mean"]:
        each = each / valid.sum().clamp(min=1)
    out = {"total": (loss * each).sum(), "loss": loss}
    if case["grads"]:
        p *= each.unsqueeze(1) / norm
        p.scatter_add_(1, at, -each.unsqueeze(1))
        out["dh"] = (p @ w).to(s["h"].dtype)
        out["dw"] = (p.t() @ h).to(s["w"].dtype)
    return out


def run(s):
    case = s["case"]
    if case["op"] == "linear_ce":
        if own:
            return s["plan"](s["h"], s["w"], s["target"], weight=s["weight"], mean=case["mean"])
        return _plain_ce(s)
    if case["op"] == "orthogonalize":
        return s["plan"].orthogonalize(s["u"]) if own else _plain_ortho(s["u"]).to(s["u"].dtype)
    hp = dict(STEP, scale=_scale(case), nesterov=case["nesterov"])
    if own:
        s["plan"].step(s["x"], s["m"], s["g"], **hp)
    else:
        s["m"].mul_(hp["mu"]).add_(s["g"])
        u = s["g"] + hp["mu"] * s["m"] if hp["nesterov"] else s["m"]
        s["x"].sub_(hp["lr"] * (hp["scale"] * _plain_ortho(u) + hp["wd"] * s["x"]))
    return {"x": s["x"], "m": s["m"]}


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "linear_ce":
        T, D, V = case["tokens"], case["dim"], case["vocab"]
        return {"bytes": (2 if case["grads"] else 1) * size * (T + V) * D + 16 * T,
                "flops": (6 if case["grads"] else 2) * T * V * D}
    short, long = sorted((case["rows"], case["cols"]))
    # A and A A are symmetric: half of each is enough.
    flops = STEPS * (3 * short * short * long + short ** 3)
    passes = 2 if case["op"] == "orthogonalize" else 5
    return {"bytes": passes * size * case["count"] * short * long, "flops": case["count"] * flops}


def _exact_ortho(u):
    # The definition as a polynomial of the singular values, evaluated with the
    # products grouped from the right.
    a, b, c = COEFFS
    x = u.double()
    flat = x.flatten(1)
    x = x / ((flat * flat).sum(1).sqrt() + EPS)[:, None, None]
    wide = x.shape[2] >= x.shape[1]
    x = x if wide else x.transpose(1, 2).contiguous()
    for _ in range(STEPS):
        xt = x.transpose(1, 2).contiguous()
        once = torch.bmm(torch.bmm(x, xt), x)
        twice = torch.bmm(torch.bmm(once, xt), x)
        x = a * x + b * once + c * twice
    return x if wide else x.transpose(1, 2).contiguous()


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if case["op"] == "orthogonalize":
        return _exact_ortho(s["u"])
    if case["op"] == "ortho_step":
        x, m, g = s["x"].double(), s["m"].double(), s["g"].double()
        m = STEP["mu"] * m + g
        u = g + STEP["mu"] * m if case["nesterov"] else m
        return {"x": x * (1 - STEP["lr"] * STEP["wd"]) - STEP["lr"] * _scale(case) * _exact_ortho(u), "m": m}
    h, w, target = s["h"].double(), s["w"].double(), s["target"]
    n_valid = int(((target >= 0) & (target < case["vocab"])).sum())
    loss = torch.zeros(case["tokens"], dtype=torch.float64, device="cuda")
    share = torch.zeros_like(loss)
    dh, dw = torch.zeros_like(h), torch.zeros_like(w)
    for lo in range(0, case["tokens"], 1024):
        t = target[lo:lo + 1024]
        rows = torch.nonzero((t >= 0) & (t < case["vocab"])).squeeze(1)
        if not len(rows):
            continue
        hot = t[rows]
        rows = rows + lo
        z = torch.mm(h[rows], w.t().contiguous())
        lse = torch.logsumexp(z, 1)
        pick = torch.arange(len(rows), device="cuda")
        loss[rows] = lse - z[pick, hot]
        share[rows] = 1.0 if s["weight"] is None else s["weight"][rows].double()
        if case["mean"]:
            share[rows] /= n_valid
        if case["grads"]:
            p = torch.exp(z - lse[:, None])
            p[pick, hot] -= 1.0
            p *= share[rows][:, None]
            dh[rows] = torch.mm(p, w)
            dw += torch.mm(p.t().contiguous(), h[rows])
    out = {"total": (loss * share).sum(), "loss": loss}
    if case["grads"]:
        out.update(dh=dh, dw=dw)
    return out
