"""Local AdamW on a small Peri-LN network: M workers, each with its own data
shard and its own copy of the parameters in one GPU's memory.

The network's blocks are two matrix products each; everything between two of them is
``peri_norm`` (norm after a block, gate, residual, norm before the next), with
its gradients.  Each worker's gradient is clipped to norm 1 and applied by
``AdamW`` with m and v in 8 bits; every ``period`` steps parameters and states are
averaged over the workers.

    python examples/local_adamw.py [--steps 300] [--state-bits 8] [--workers 4]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2510_05361_gb300 as P  # noqa: E402

WIDTH, HIDDEN, BLOCKS, INPUTS, CLASSES = 128, 256, 3, 32, 10


def shapes():
    """Name and shape of every parameter: the embedding, for each block two
    matrices, then for each update between blocks two norms (weight, bias) and a gate, the head."""
    out = [("embed", (WIDTH, INPUTS))]
    for k in range(BLOCKS):
        out += [("up%d" % k, (HIDDEN, WIDTH)), ("down%d" % k, (WIDTH, HIDDEN))]
    for k in range(BLOCKS + 1):
        out += [("%s%d" % (n, k), (WIDTH,)) for n in ("post_w", "post_b", "pre_w", "pre_b", "gate")]
    return out + [("head", (CLASSES, WIDTH))]


def initial(generator):
    values = {}
    for name, shape in shapes():
        if len(shape) == 2:
            values[name] = torch.randn(shape, generator=generator) / shape[1] ** 0.5
        else:
            values[name] = torch.full(shape, 0.0 if name[:-1].endswith("_b") else 1.0)
    return values


def forward(p, inputs):
    """Class scores; p: name -> tensor.  The embedding is the first block's output and the
    stream starts at zero, so that it is normed like any other."""
    f = inputs @ p["embed"].t()
    x = torch.zeros_like(f)
    for k in range(BLOCKS + 1):
        x, h = P.peri_norm(x, f, p["post_w%d" % k], p["pre_w%d" % k], post_bias=p["post_b%d" % k],
                           pre_bias=p["pre_b%d" % k], gate=p["gate%d" % k], norm="layer")
        if k < BLOCKS:
            f = torch.nn.functional.silu(h @ p["up%d" % k].t()) @ p["down%d" % k].t()
    return h @ p["head"].t()


def train(workers=4, steps=300, period=16, state_bits=8, batch=256, lr=3e-3, seed=0, dtype=torch.float32):
    """Trains on a fixed random teacher; returns the loss on held-out data before and
    after, the workers' parameters and the optimizer."""
    generator = torch.Generator().manual_seed(seed)
    start = initial(generator)
    teacher = {k: v.cuda() for k, v in initial(generator).items()}
    names = [n for n, _ in shapes()]
    params = [[start[n].to("cuda", dtype) for n in names] for _ in range(workers)]
    grads = [[torch.zeros_like(t) for t in row] for row in params]
    opt = P.AdamW(params, grads, betas=(0.9, 0.99), state_bits=state_bits,
                  decay=[1.0 if t.dim() == 2 else 0.0 for t in params[0]], seed=seed)
    shards = [torch.Generator(device="cuda").manual_seed(100 + w) for w in range(workers)]

    def data(count, gen):
        inputs = torch.randn((count, INPUTS), device="cuda", generator=gen)
        with torch.no_grad():
            return inputs, forward(teacher, inputs).argmax(1)
    held = data(4096, torch.Generator(device="cuda").manual_seed(1))

    def loss_of(tensors, inputs, labels):
        scores = forward(dict(zip(names, (t.float() for t in tensors))), inputs)
        return torch.nn.functional.cross_entropy(scores, labels)

    def held_out():
        with torch.no_grad():
            return float(sum(loss_of(row, *held) for row in params) / workers)
    before = held_out()
    for step in range(steps):
        for row, buffers, shard in zip(params, grads, shards):
            leaves = [t.detach().requires_grad_() for t in row]
            loss = loss_of(leaves, *data(batch, shard))
            for buffer, g in zip(buffers, torch.autograd.grad(loss, leaves)):
                buffer.copy_(g)
        opt.step(lr, weight_decay=0.01, max_norm=1.0)
        if (step + 1) % period == 0:
            opt.average()
    return before, held_out(), params, opt


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--period", type=int, default=16)
    ap.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    first, last, _, _ = train(a.workers, a.steps, a.period, a.state_bits)
    print("held-out loss %.4f -> %.4f after %d steps of %d workers" % (first, last, a.steps, a.workers))
