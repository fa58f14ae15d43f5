"""The example's transformer layer: attention, kept activations, head, clipping and AdamW together, inside Algorithm 1."""
import math

import pytest
import torch

import gpu_util
from paper_2009_03816_b200 import train_demo, training

pytestmark = pytest.mark.gpu
SMALL = dict(K=2, vocab=509, dim=64, tokens=512, epochs=1, iters_per_epoch=20, model="block", ff=200, heads=4, kv_heads=2)


@pytest.mark.parametrize("method", ["pso", "pa"])
def test_it_runs(method):
    gpu_util.ensure_library()
    cfg = train_demo.TrainConfig(**SMALL)
    out = train_demo.run(method, cfg)
    assert len(out["best_loss"]) == 2 and out["steps"] == 20
    assert all(math.isfinite(v) for v in out["best_loss"] + out["mean_loss"])
    assert abs(out["initial_loss"] - math.log(cfg.vocab)) < 1.5          # random weights predict next to nothing


def test_packed_sequences_are_the_source():
    gpu_util.ensure_library()
    cfg = train_demo.TrainConfig(**SMALL)
    source = train_demo.Source(cfg, "cuda:0")
    x, y = source.packed(cfg.tokens)
    assert sum(cfg.lengths) == cfg.tokens == x.numel() == y.numel() and 1 in cfg.lengths
    ends = torch.tensor(cfg.lengths).cumsum(0) - 1
    inside = torch.ones(cfg.tokens, dtype=torch.bool)
    inside[ends] = False
    inside = inside.cuda()
    assert torch.equal(y[inside], x[1:][inside[:-1]])                    # what follows in a sequence is the next token
    assert float((y == source.after[x]).float().mean()) > 0.5


def test_gradients_of_the_layer():
    """One step's gradients against the same model in 64 bits.  What is kept in 8 bits is off by half a step, 1/254 of
    a block's largest number, some 1 % of a typical one, independently for each; a dozen 16-bit roundings of 2^-9 come
    on top: 5 % of a gradient's norm is far outside both."""
    gpu_util.ensure_library()
    cfg = train_demo.TrainConfig(**SMALL)
    gen = torch.Generator(device="cuda").manual_seed(3)
    row = torch.empty(cfg.ld, device="cuda").normal_(0.0, 1.5 * cfg.dim ** -0.5, generator=gen)
    xent = training.LinearXent(cfg.tokens, cfg.dim, cfg.vocab)
    worker = train_demo.BlockWorker(cfg, row, xent)
    x, y = train_demo.Source(cfg, "cuda:0").packed(cfg.tokens)
    leaves = [c.detach().double().requires_grad_() for c in worker.copies]
    worker.opt.step = lambda *a: None                                    # the gradients alone
    worker.local_step(x, y, torch.ones((), device="cuda"))
    e, qkv, bias, out, up, down, w = leaves
    H, G, D = cfg.heads, cfg.kv_heads, cfg.dim // cfg.heads
    h = e[x]
    p = (h @ qkv).view(-1, H + 2 * G, D)
    first = training.distance_buckets(cfg.buckets, cfg.far)
    parts, at = [], 0
    for n in cfg.lengths:
        r = slice(at, at + n)
        at += n
        d = torch.arange(n, device="cuda")[:, None] - torch.arange(n, device="cuda")
        of = torch.bucketize(d.clamp(min=0), torch.tensor(first, device="cuda"), right=True) - 1
        heads = []
        for k in range(H):
            s = p[r, k] @ p[r, H + k // (H // G)].T / D ** 0.5 + bias[:, k][of]
            heads.append(torch.softmax(torch.where(d >= 0, s, -math.inf), -1) @ p[r, H + G + k // (H // G)])
        parts.append(torch.stack(heads, 1))
    h = h + torch.cat(parts).reshape(-1, cfg.dim) @ out
    a, b = (h @ up).chunk(2, -1)
    h = h + (a * torch.sigmoid(a) * b) @ down
    loss = torch.nn.functional.cross_entropy(h @ w.T, y)
    loss.backward()
    for name, got, leaf in zip(("e", "qkv", "bias", "out", "up", "down", "w"), worker.grads, leaves):
        off = float((got.double() - leaf.grad).norm() / leaf.grad.norm())
        assert off < 0.05, (name, off)
    worker.close()


def test_command_line(capsys):
    out = train_demo.main(["--model", "block", "--k", "2", "--vocab", "300", "--dim", "32", "--tokens", "128", "--epochs", "1",
                           "--iters-per-epoch", "10", "--heads", "2", "--kv-heads", "1"])
    assert out["config"]["model"] == "block" and out["parameters"] == train_demo.TrainConfig(**out["config"]).N
    assert '"methods"' in capsys.readouterr().out
