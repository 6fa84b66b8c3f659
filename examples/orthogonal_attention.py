"""Workers that train a small attention model with orthogonalised local steps.

m logical workers on one GPU learn to repeat the token of two places before.  In
every local step of a worker
  - queries and keys go through HeadNormRotary: their norm for each head and the
    position rotation in one pass, differentiated by autograd;
  - the projections' gradients become directions by Orthogonalizer: the SGD row's
    momentum, then Newton-Schulz products.  They go to SlowMo.local_step as the gradient
    (momentum 0 there; its coupled decay is then the decoupled one);
  - embeddings, norm weights and the head take Adam, in a SlowMo of their own.
Every tau steps the workers' replicas are averaged and the slow momentum is applied.  The directions'
momentum is this program's: it is kept over the outer step, each worker's own, whatever the buffer policy
of SlowMo does to Adam's buffers.

    python examples/orthogonal_attention.py [outer iterations]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1910_00643_amd import (HeadNormRotary, Orthogonalizer, SlowMo, make_config,  # noqa: E402
                                  rotary_table)

VOCAB, WIDTH, HEADS, DIM, LENGTH, BATCH = 64, 128, 4, 32, 48, 32
MATRICES = ["wq", "wk", "wv", "wo"]
OTHERS = {"embed": (VOCAB, WIDTH), "head": (VOCAB, WIDTH), "q_norm": (DIM,), "k_norm": (DIM,)}


def make_worker(device, seed):
    g = torch.Generator(device=device).manual_seed(seed)
    p = {n: torch.randn(WIDTH, WIDTH, device=device, generator=g) / WIDTH ** 0.5 for n in MATRICES}
    for n, s in OTHERS.items():
        p[n] = torch.ones(s, device=device) if len(s) == 1 else torch.randn(s, device=device, generator=g) * 0.5
    return {n: t.requires_grad_() for n, t in p.items()}


def loss_of(p, tokens, rotate, positions):
    """Cross entropy of every token from the third on against the one of two places before."""
    b, t = tokens.shape
    x = p["embed"][tokens]
    q, k, v = ((x @ p[n].t()).view(b * t, HEADS, DIM) for n in ("wq", "wk", "wv"))
    q, k = rotate(q, k, positions, p["q_norm"], p["k_norm"])
    q, k, v = (y.view(b, t, HEADS, DIM).transpose(1, 2).contiguous() for y in (q, k, v))
    scores = (q @ k.transpose(2, 3).contiguous()) * (4.0 / DIM ** 0.5)
    later = torch.ones(t, t, dtype=torch.bool, device=x.device).triu(1)
    mixed = torch.softmax(scores.masked_fill(later, float("-inf")), -1) @ v
    y = x + mixed.transpose(1, 2).reshape(b, t, WIDTH) @ p["wo"].t()
    logits = y @ p["head"].t()
    return torch.nn.functional.cross_entropy(logits[:, 2:].reshape(-1, VOCAB), tokens[:, :-2].reshape(-1))


def train(outer=20, m=2, tau=6, lr=0.02, adam_lr=3e-3, device="cuda:0"):
    """Returns the workers' mean loss of every local step."""
    workers = [make_worker(device, 1) for _ in range(m)]
    matrices = [[w[n].detach() for n in MATRICES] for w in workers]
    others = [[w[n].detach() for n in OTHERS] for w in workers]
    opt = SlowMo(matrices, make_config(m=m, tau=tau, alpha=1.0, beta=0.5, momentum=0.0, weight_decay=0.01))
    adam = SlowMo(others, make_config(m=m, tau=tau, alpha=1.0, beta=0.5, base="adam"))
    shapes = [tuple(t.shape) for w in matrices for t in w]
    orth = Orthogonalizer(shapes, dtype="f32", out_dtype="f32", scale="rms", device=device)
    momentum = [torch.zeros(s, device=device) for s in shapes]
    directions = [[torch.empty_like(t) for t in w] for w in matrices]
    rotate = HeadNormRotary(DIM, rotary_table(LENGTH, DIM // 2, device=device), dtype="f32")
    positions = torch.arange(LENGTH, device=device).repeat(BATCH)
    g = torch.Generator(device=device).manual_seed(7)
    losses = []
    for _ in range(outer):
        for step in range(tau):
            mean = 0.0
            for w in workers:
                tokens = torch.randint(0, VOCAB, (BATCH, LENGTH), device=device, generator=g)
                for t in w.values():
                    t.grad = None
                loss = loss_of(w, tokens, rotate, positions)
                loss.backward()
                mean += loss.detach() / m
            losses.append(mean)
            orth.momentum_orthogonalize([w[n].grad for w in workers for n in MATRICES], momentum,
                                        [t for d in directions for t in d], 0.95)
            opt.local_step(directions, lr)
            adam.local_step([[w[n].grad for n in OTHERS] for w in workers], adam_lr)
        opt.outer_step(lr)
        adam.outer_step(adam_lr)
    opt.close()
    adam.close()
    return [float(v) for v in losses]


if __name__ == "__main__":
    run = train(outer=int(sys.argv[1]) if len(sys.argv) > 1 else 20)
    for i in range(0, len(run), 6):
        print("local step %3d  loss %.4f" % (i, run[i]))
    print("last  loss %.4f" % run[-1])
