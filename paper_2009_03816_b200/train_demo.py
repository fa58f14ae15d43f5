"""Workers that train a small language model, synchronised by PSO-PS or by averaging.

    python -m paper_2009_03816_b200.train_demo [--epochs 4] [--vocab 2048] ...

K workers start from the same weights and each see their own stream of tokens
drawn from one second-order source.  A worker's model predicts the next token
from the last two: h = tanh(e[x1] + e[x2] m), logits = h w^T, with the three
matrices e (vocab x dim), m (dim x dim) and w (vocab x dim).  Its fp32 weights
are its row of the swarm (three views of it); the model itself reads bf16
copies.  A local step is, all of it on the device:

  loss and gradients of the head   training.LinearXent (the logits are never kept)
  gradients of e and m             a few torch operations
  norm of all gradients            training.GradNorm
  AdamW with the clipping factor   training.AdamW, one launch, which also rewrites
                                   the bf16 copies

and every `step` iterations each worker's loss on a common held-out batch --
LinearXent's forward alone, written straight into the swarm's loss vector -- is
its fitness for one synchronisation (binding.Swarm: psops_sync, or psops_average
for the averaging baseline).  The result is one JSON object with the best and the
mean held-out loss after every synchronisation.
"""
from __future__ import annotations

import argparse
import json
from dataclasses import asdict, dataclass

import torch

from . import binding, training
from . import build as _build


@dataclass(frozen=True)
class TrainConfig:
    K: int = 4                   # workers = particles
    vocab: int = 2048
    dim: int = 256
    tokens: int = 1024           # of a worker's batch, and of the held-out batch
    epochs: int = 4
    iters_per_epoch: int = 40
    step: int = 10               # iterations between synchronisations (Algorithm 1)
    lr: float = 3e-3
    weight_decay: float = 0.01
    max_norm: float = 1.0
    state_bits: int = 8          # of AdamW's moments
    seed: int = 11
    m_max: float = 0.9           # Table II
    m_min: float = 0.3
    c1: float = 0.2
    c2: float = 0.9

    @property
    def N(self) -> int:
        return 2 * self.vocab * self.dim + self.dim * self.dim

    @property
    def ld(self) -> int:
        return (self.N + 1023) // 1024 * 1024

    @property
    def t_max(self) -> int:
        return self.epochs * self.iters_per_epoch


class Source:
    """Tokens of uneven frequency; seven in ten follow from the last token, two from the one before, one from neither."""

    def __init__(self, cfg: TrainConfig, device):
        self.gen = torch.Generator(device=device).manual_seed(cfg.seed)
        self.vocab, self.device = cfg.vocab, device
        self.after, self.later = (torch.randperm(cfg.vocab, device=device, generator=self.gen) for _ in range(2))

    def _draw(self, tokens):
        u = torch.rand(tokens, device=self.device, generator=self.gen)
        return (self.vocab * u ** 3).long().clamp(max=self.vocab - 1)

    def batch(self, tokens):
        """(last token, token before it, next token), `tokens` of each."""
        x1, x2, free = (self._draw(tokens) for _ in range(3))
        u = torch.rand(tokens, device=self.device, generator=self.gen)
        return x1, x2, torch.where(u < 0.7, self.after[x1], torch.where(u < 0.9, self.later[x2], free))


class Worker:
    """One particle's model: views of its row, their bf16 copies, gradients and optimiser."""

    def __init__(self, cfg: TrainConfig, row, xent):
        V, D = cfg.vocab, cfg.dim
        shapes = ((V, D), (D, D), (V, D))
        at, self.weights = 0, []
        for a, b in shapes:
            self.weights.append(row[at:at + a * b].view(a, b))
            at += a * b
        self.copies = [w.to(torch.bfloat16) for w in self.weights]
        self.grads = [torch.zeros_like(c) for c in self.copies]
        self.xent = xent
        self.opt = training.AdamW(self.weights, self.grads, bits=cfg.state_bits, copies=self.copies,
                                  weight_decay=[0.0, cfg.weight_decay, cfg.weight_decay])
        self.clip = training.GradNorm(self.grads)
        self.cfg = cfg

    def hidden(self, x1, x2):
        e, m, _ = self.copies
        return torch.tanh(e[x1].float() + (e[x2] @ m).float())

    def local_step(self, x1, x2, y, one):
        e, m, w = self.copies
        de, dm, dw = self.grads
        h = self.hidden(x1, x2)
        h16 = h.to(torch.bfloat16)
        _, rows, lse = self.xent.forward(h16, w, y)
        dh, _ = self.xent.backward(h16, w, y, lse, one, rows=rows, dw=dw)
        du = (dh.float() * (1.0 - h * h)).to(torch.bfloat16)
        torch.mm(e[x2].T, du, out=dm)
        de.zero_()
        de.index_put_((torch.cat([x1, x2]),), torch.cat([du, du @ m.T]), accumulate=True)
        _, factor = self.clip.norm(self.cfg.max_norm)
        self.opt.step(self.cfg.lr, factor)

    def loss_into(self, out, x1, x2, y):
        self.xent.forward(self.hidden(x1, x2).to(torch.bfloat16), self.copies[2], y, loss=out)

    def reread(self):
        """The row was rewritten by a synchronisation."""
        for c, w in zip(self.copies, self.weights):
            c.copy_(w)

    def close(self):
        self.opt.close()
        self.clip.close()


def run(method: str, cfg: TrainConfig = TrainConfig(), device="cuda:0") -> dict:
    assert method in ("pso", "pa")
    _build.build_library()
    device = torch.device(device)
    gen = torch.Generator(device=device).manual_seed(cfg.seed + 1)
    x = torch.zeros((cfg.K, cfg.ld), dtype=torch.float32, device=device)
    x[:, :cfg.N] = torch.empty(cfg.N, device=device).normal_(0.0, cfg.dim ** -0.5, generator=gen)
    v, p = torch.zeros_like(x), x.clone()
    swarm = binding.Swarm(x, v, p, N=cfg.N, m_max=cfg.m_max, m_min=cfg.m_min, t_max=cfg.t_max, c1=cfg.c1, c2=cfg.c2,
                          seed=cfg.seed)
    xent = training.LinearXent(cfg.tokens, cfg.dim, cfg.vocab, device=device)
    workers = [Worker(cfg, x[k], xent) for k in range(cfg.K)]
    source = Source(cfg, device)
    held_out = source.batch(cfg.tokens)
    one = torch.ones((), device=device)
    losses = torch.zeros(cfg.K, device=device)

    def fitness():
        for k, worker in enumerate(workers):
            worker.loss_into(losses[k], *held_out)
        return losses

    initial = float(fitness()[0])
    best, mean, chosen = [], [], []
    for it in range(1, cfg.t_max + 1):
        for worker in workers:
            worker.local_step(*source.batch(cfg.tokens), one)
        if it % cfg.step:
            continue
        if method == "pa":
            swarm.average()
        else:
            swarm.set_losses(fitness())
            swarm.sync(it, float(1 + (it - 1) // cfg.iters_per_epoch))       # lambda = epoch index (Table II)
            chosen.append(swarm.info()[0])
        for worker in workers:
            worker.reread()
        after = fitness()
        best.append(float(after.min()))
        mean.append(float(after.mean()))
    torch.cuda.synchronize(device)
    out = {"method": method, "initial_loss": initial, "best_loss": best, "mean_loss": mean, "steps": workers[0].opt.steps}
    if chosen:
        out["gbest"] = chosen
    for worker in workers:
        worker.close()
    xent.close()
    swarm.close()
    return out


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, default in asdict(TrainConfig()).items():
        ap.add_argument("--" + name.replace("_", "-").lower(), type=type(default), default=default)
    ap.add_argument("--device", default="cuda:0")
    args = vars(ap.parse_args(argv))
    device = args.pop("device")
    cfg = TrainConfig(**{k: args[k.lower()] for k in asdict(TrainConfig())})
    out = {"config": asdict(cfg), "parameters": cfg.N, "methods": {m: run(m, cfg, device) for m in ("pso", "pa")}}
    print(json.dumps(out))
    return out


if __name__ == "__main__":
    main()
