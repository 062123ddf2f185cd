"""A small language model trained in pipeline stages with compressed boundaries (one GPU).

The model is cut into stages; after each but the last a CompressionBoundary sends the compressed
activation forward and the compressed gradient back.  The last stage's loss is the linear cross
entropy over the vocabulary, without its logits, and every stage takes its own AdamW step with
clipping by the gradient norm.  The data are synthetic: a random walk over the vocabulary in which
each word has a few likely successors, with some positions padded (target -100).

    python examples/train_stages.py [--steps 200] [--vocab 50257] [--width 256] [--stages 3]
        [--state-bits 8] [--topk 20]
"""

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2401_07788_gb300 as mpc  # noqa: E402


class Stage(torch.nn.Module):
    """Embedding (first stage only), then residual blocks of a causal average and an MLP."""

    def __init__(self, width, blocks, vocab=None):
        super().__init__()
        self.embed = None if vocab is None else torch.nn.Embedding(vocab, width)
        self.norms = torch.nn.ModuleList(torch.nn.LayerNorm(width) for _ in range(blocks))
        self.mix = torch.nn.ModuleList(torch.nn.Linear(2 * width, 2 * width) for _ in range(blocks))
        self.out = torch.nn.ModuleList(torch.nn.Linear(2 * width, width) for _ in range(blocks))

    def forward(self, x):
        if self.embed is not None:
            x = self.embed(x)
        for norm, mix, out in zip(self.norms, self.mix, self.out):
            y = norm(x)
            count = torch.arange(1, y.shape[1] + 1, device=y.device, dtype=y.dtype)[:, None]
            y = torch.cat([y, y.cumsum(1) / count], dim=-1)
            x = x + out(torch.nn.functional.gelu(mix(y)))
        return x


def batches(vocab, batch, length, seed, device):
    """Endless (inputs, targets) of a Markov walk; the tail of each sequence is padding."""
    gen = torch.Generator(device=device).manual_seed(seed)
    likely = torch.randint(0, vocab, (vocab, 4), device=device, generator=gen)
    while True:
        x = torch.empty(batch, length + 1, dtype=torch.int64, device=device)
        x[:, 0] = torch.randint(0, vocab, (batch,), device=device, generator=gen)
        for t in range(length):
            pick = torch.randint(0, 4, (batch, 1), device=device, generator=gen)
            x[:, t + 1] = likely[x[:, t]].gather(1, pick)[:, 0]
        y = x[:, 1:].clone()
        ends = torch.randint(length // 2, length + 1, (batch, 1), device=device, generator=gen)
        y[torch.arange(length, device=device)[None] >= ends] = -100
        yield x[:, :-1], y


def train(steps=200, vocab=50257, width=256, stages=3, blocks=2, batch=16, length=64, topk=20, state_bits=8,
          lr=2e-3, seed=0, log=print):
    device = torch.device("cuda")
    torch.manual_seed(seed)
    parts = [Stage(width, blocks, vocab if i == 0 else None).to(device) for i in range(stages)]
    body = mpc.with_boundaries(parts, lambda i: mpc.CompressionBoundary(
        mpc.TopK(topk, feedback="ef21"), mpc.Quant(8), rows="last"))
    head = mpc.LinearCrossEntropy(width, vocab, device=device)

    def optimizer(params):
        params = list(params)
        groups = [{"params": [p for p in params if p.dim() > 1], "weight_decay": 0.01},
                  {"params": [p for p in params if p.dim() <= 1], "weight_decay": 0.0}]
        return mpc.AdamW([g for g in groups if g["params"]], lr=lr, betas=(0.9, 0.95), state_bits=state_bits,
                         max_norm=1.0)

    optimizers = [optimizer(p.parameters()) for p in parts[:-1]]
    optimizers.append(optimizer(list(parts[-1].parameters()) + list(head.parameters())))
    losses = []
    for step, (x, y) in zip(range(steps), batches(vocab, batch, length, seed + 1, device)):
        loss = head(body(x), y)
        for o in optimizers:
            o.zero_grad()
        loss.backward()
        for o in optimizers:
            o.step()
        losses.append(loss.detach())
        if log is not None and (step % 20 == 0 or step + 1 == steps):
            log("step %4d  loss %.4f  (uniform %.4f)  last stage's gradient norm %.3f" % (
                step, float(loss.detach()), math.log(vocab), float(optimizers[-1].last_norm)))
    if mpc.mpc_get_status() != 0:
        raise RuntimeError(mpc.mpc_last_error())
    return torch.stack(losses).cpu()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 200), ("vocab", 50257), ("width", 256), ("stages", 3), ("topk", 20),
                        ("state-bits", 8)):
        ap.add_argument("--" + name, type=int, default=value)
    train(**vars(ap.parse_args()))
