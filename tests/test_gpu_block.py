"""The operators of a model's blocks as a training step uses them: embedding, norm,
feed-forward with residual, the output layer's cross entropy, the gradients back into the
workers' arenas, clipping there, a local step; against the same step in float64 with
torch's own derivatives."""
import pytest

torch = pytest.importorskip("torch")

from paper_2411_17866_amd import arena, dsm  # noqa: E402

pytestmark = pytest.mark.gpu

TOKENS, DIM, HIDDEN, VOCAB, WORKERS = 150, 72, 200, 501, 2
SHAPES = {"E": (VOCAB, DIM), "g1": (DIM,), "b1": (DIM,), "U": (HIDDEN, DIM), "u": (HIDDEN,), "V": (DIM, HIDDEN), "v": (DIM,),
          "gate": (DIM,), "gp": (DIM,), "g2": (DIM,), "W": (VOCAB, DIM)}
MAX, LR = 0.05, 0.1


def _norm(x, weight, bias=None, layer=True):
    if layer:
        x = x - x.mean(1, keepdim=True)
    y = x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt() * weight
    return y if bias is None else y + bias


def _reference(p, tokens, target):
    """The gradients of the mean loss, clipped, in float64."""
    p = {k: t.detach().double().requires_grad_() for k, t in p.items()}
    h = p["E"][tokens]
    z = _norm(h, p["g1"], p["b1"]) @ p["U"].t() + p["u"]
    f = torch.nn.functional.gelu(z, approximate="tanh") @ p["V"].t() + p["v"]
    s = h + 0.5 * p["gate"] * _norm(f, p["gp"], layer=False)
    logits = _norm(s, p["g2"], layer=False) @ p["W"].t()
    loss = torch.nn.functional.cross_entropy(logits, target)
    loss.backward()
    grads = {k: t.grad for k, t in p.items()}
    norm = torch.stack([g.square().sum() for g in grads.values()]).sum().sqrt()
    return float(loss), float(norm), {k: g * min(1.0, MAX / (float(norm) + 1e-6)) for k, g in grads.items()}


@pytest.mark.parametrize("layout", [dsm.DSM_REPLICAS_CONTIGUOUS, dsm.DSM_REPLICAS_STATE_BLOCKED])
def test_a_training_step(layout):
    from paper_2411_17866_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(0)
    names = list(SHAPES)
    numel = [torch.Size(s).numel() for s in SHAPES.values()]
    ar = arena.Arenas(numel, WORKERS, 2, dsm.DSM_BASE_SGD_MOMENTUM, replica_layout=layout)
    for n, o, k in zip(names, ar.offsets, numel):
        v = torch.empty(k, device="cuda").normal_(1.0 if n in ("g1", "gp", "g2", "gate") else 0.0, 0.2, generator=gen)
        ar.x[int(o):int(o) + k] = v
    ar.init()
    first = ops.ResidualNorm(TOKENS, DIM, norm="layer")
    last = ops.ResidualNorm(TOKENS, DIM, norm="rms", post="rms")
    up = ops.Linear(TOKENS, DIM, HIDDEN, act="gelu_tanh")
    down = ops.Linear(TOKENS, HIDDEN, DIM)
    loss = ops.LinearCE(TOKENS, DIM, VOCAB)
    clip = ops.ArenaClip(ar)
    packed = torch.zeros(WORKERS, ar.arena_elems, device="cuda")
    want, losses = [], []
    for worker in range(WORKERS):
        tokens = torch.randint(0, VOCAB, (TOKENS,), device="cuda", generator=gen)
        target = torch.randint(0, VOCAB, (TOKENS,), device="cuda", generator=gen)
        x = ar.worker("x_rep", worker)
        p, g = ({n: b[int(o):int(o) + k].view(SHAPES[n]) for n, o, k in zip(names, ar.offsets, numel)} for b in (x, packed[worker]))
        h = p["E"][tokens]
        a = first(h, weight=p["g1"], bias=p["b1"])["y"]
        mid = up(a, p["U"], bias=p["u"])
        f = down(mid["y"], p["V"], bias=p["v"])["y"]
        vectors = dict(gate=p["gate"], scale=0.5, post_weight=p["gp"], weight=p["g2"])
        out = last(h, f=f, **vectors)
        ce = loss(out["y"], p["W"], target, dw=g["W"])
        d = last.backward(ce["dh"], out["s"], f=f, dgate=g["gate"], dpost_weight=g["gp"], dweight=g["g2"], **vectors)
        dm = down.backward(d["df"], mid["y"], p["V"], dw=g["V"], dbias=g["v"])["dx"]
        da = up.backward(dm, a, p["U"], z=mid["z"], dw=g["U"], dbias=g["u"])["dx"]
        dh = first.backward(da, h, weight=p["g1"], bias=p["b1"], dweight=g["g1"], dbias=g["b1"])["dh"]
        g["E"].index_add_(0, tokens, dh + d["dh"])
        losses.append(float(ce["total"]))
        want.append(_reference(p, tokens, target))
    ar.write_workers("g_rep", packed)
    norms = clip(ar, MAX).tolist()
    before = ar.workers("x_rep").clone()
    dsm.dsm_local_step(ar.ctx, -1, 1, lr=LR, beta1=0.0)
    after, got = ar.workers("x_rep"), ar.workers("g_rep")
    for worker, (value, norm, grads) in enumerate(want):
        # fp32 chains of some hundred roundings.
        assert abs(losses[worker] - value) < 1e-5 * value and abs(norms[worker] - norm) < 1e-5 * norm and norm > MAX
        for n, o, k in zip(names, ar.offsets, numel):
            at = slice(int(o), int(o) + k)
            off = float((got[worker, at].double() - grads[n].flatten()).norm() / grads[n].norm())
            assert off < 1e-5, (n, off)
            step = before[worker, at] - LR * got[worker, at]
            assert torch.allclose(after[worker, at], step, rtol=1e-6, atol=1e-8)
    ar.destroy()
