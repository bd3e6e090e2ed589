"""Trains a small language model with the library's operators end to end: the output
layer's cross entropy and its gradients (ops.LinearCE), orthogonalised momentum as the
direction of the hidden matrices (ops.Ortho), and distributed sign momentum with local
steps over the whole parameter arena.

The model predicts a token from the two before it:  a = E[t-1] + F[t-2],
h = a + relu(a U^T) V^T, logits = h W^T.  Its data is a synthetic second-order Markov
chain.  Every worker has its own replica and stream of tokens; each local step takes

  * h and W through LinearCE, whose dw is written into the worker's gradient arena;
  * dh back through the hidden layer into the arena (plain torch products);
  * the hidden matrices' gradients through momentum and orthogonalisation, in the arena
    (every worker's in one call);
  * the local step of the arena with that direction (SGD, beta1 = 0);

and each round ends with the global sign-momentum step.

    python examples/train_small_lm.py [rounds]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2411_17866_amd import arena, dsm, ops  # noqa: E402

VOCAB, DIM, HIDDEN = 1009, 96, 200
WORKERS, LOCAL_STEPS, TOKENS = 2, 4, 700
SHAPES = {"E": (VOCAB, DIM), "F": (VOCAB, DIM), "U": (HIDDEN, DIM), "V": (DIM, HIDDEN), "W": (VOCAB, DIM)}
LR, MU, GAMMA = 0.3, 0.9, 2e-3
GLOBAL = dict(eta=0.8, beta1=0.95, beta2=0.98, lam=0.0)


def chain(generator):
    """Each pair of classes of tokens is followed by few tokens, most often one."""
    following = torch.randint(0, VOCAB, (8, 8, 4), device="cuda", generator=generator)
    share = torch.tensor([0.7, 0.15, 0.1, 0.05], device="cuda")

    def batch(count):
        two = torch.randint(0, VOCAB, (2, count), device="cuda", generator=generator)
        pick = torch.multinomial(share.expand(count, 4), 1, generator=generator)[:, 0]
        return two[0], two[1], following[two[0] % 8, two[1] % 8, pick]

    return batch


class Model:
    def __init__(self, seed=0):
        self.generator = torch.Generator(device="cuda").manual_seed(seed)
        self.names = list(SHAPES)
        self.numel = [a * b for a, b in SHAPES.values()]
        self.ar = arena.Arenas(self.numel, WORKERS, LOCAL_STEPS, dsm.DSM_BASE_SGD_MOMENTUM)
        self.ar.x.normal_(0.0, 0.05, generator=self.generator)
        self.ar.init()
        self.batch = chain(self.generator)
        self.loss = ops.LinearCE(TOKENS, DIM, VOCAB)
        # The hidden matrices of every worker, by their places in the gradient arena.
        self.momentum = torch.zeros_like(self.ar.g_rep)
        self.ortho = []
        for name in ("U", "V"):
            at = int(self.ar.offsets[self.names.index(name)])
            plan = ops.Ortho(*SHAPES[name], WORKERS,
                             offsets=[at + i * self.ar.arena_elems for i in range(WORKERS)])
            self.ortho.append((plan, 0.2 * max(SHAPES[name]) ** 0.5 * 0.1))
        self.step = 0

    def views(self, buffer, worker):
        return {n: buffer[worker, int(o):int(o) + k].view(SHAPES[n])
                for n, o, k in zip(self.names, self.ar.offsets, self.numel)}

    def gradients(self, worker, stale):
        """The worker's gradients, written into the arena; its mean loss."""
        source = self.ar.x.expand(WORKERS, -1) if stale else self.ar.x_rep
        p, g = self.views(source, worker), self.views(self.ar.g_rep, worker)
        last, before, target = self.batch(TOKENS)
        a = p["E"][last] + p["F"][before]
        z = a @ p["U"].t()
        h = a + z.relu() @ p["V"].t()
        out = self.loss(h, p["W"], target, dw=g["W"])
        dz = (out["dh"] @ p["V"]) * (z > 0)
        da = out["dh"] + dz @ p["U"]
        torch.mm(out["dh"].t(), z.relu(), out=g["V"])
        torch.mm(dz.t(), a, out=g["U"])
        for name, tokens in (("E", last), ("F", before)):
            g[name].zero_().index_add_(0, tokens, da)
            g[name].mul_(30.0)
        g["W"].mul_(30.0)
        return out["total"]

    def round(self, t):
        """One outer iteration; the mean loss of its local steps."""
        total = 0.0
        for k in range(LOCAL_STEPS):
            # After a global step without broadcast the replicas are x.
            losses = [self.gradients(i, stale=k == 0 and t > 0) for i in range(WORKERS)]
            total = total + torch.stack(losses).mean()
            for plan, scale in self.ortho:
                plan.direction(self.momentum, self.ar.g_rep, self.ar.g_rep, mu=MU, scale=scale)
            self.step += 1
            if k + 1 < LOCAL_STEPS:
                dsm.dsm_local_step(self.ar.ctx, -1, self.step, lr=LR, beta1=0.0)
            else:
                dsm.dsm_round_end(self.ar.ctx, self.step, dict(lr=LR, beta1=0.0), t, gamma=GAMMA,
                                  broadcast=False, **GLOBAL)
        return float(total) / LOCAL_STEPS


def train(rounds=60, seed=0):
    model = Model(seed)
    losses = [model.round(t) for t in range(rounds)]
    model.ar.destroy()
    return losses


if __name__ == "__main__":
    history = train(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
    for t in range(0, len(history), max(1, len(history) // 10)):
        print(f"round {t:4d}  loss {history[t]:.4f}", flush=True)
    print(f"round {len(history) - 1:4d}  loss {history[-1]:.4f}")
