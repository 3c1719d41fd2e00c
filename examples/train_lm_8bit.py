"""Trains a small language model on synthetic text: a token embedding, blocks of root-mean-square norm and
MLP whose backward pass works from activations in 8 bits, and an output layer tied to the embedding.  The
blocks' matrices are stepped by Muon, everything else by NOVAK.  Each token is followed by one of a few
others, so that a model without attention has something to learn.  Prints the loss.

    python examples/train_lm_8bit.py [--steps 60] [--width 512] [--hidden 1536] [--vocab 8192] [--tokens 8192] [--depth 3]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_07876_b200.block import Embedding, RmsLinear8, RmsMlpBlock8  # noqa: E402
from paper_2601_07876_b200.optim import Muon, Novak  # noqa: E402


class Model(torch.nn.Module):
    def __init__(self, vocab, width, hidden, depth, device="cuda"):
        super().__init__()
        self.embed = Embedding(vocab, width, scale=math.sqrt(width), device=device)
        self.blocks = torch.nn.ModuleList(RmsMlpBlock8(width, hidden, device=device) for _ in range(depth))
        self.out = RmsLinear8(width, vocab, device=device)
        self.out.weight = self.embed.weight         # one matrix, two gradients

    def forward(self, ids):
        delta, stream = self.embed(ids), None
        for block in self.blocks:
            delta, stream = block(delta, stream)
        return self.out(delta, stream)[0]

    def matrices(self):
        return [p for b in self.blocks for p in (b.up.weight, b.down.weight)]


def batch(gen, tokens, vocab, after):
    """Tokens and what comes next; a twentieth of the places hold none."""
    ids = torch.randint(vocab, (tokens,), generator=gen, device="cuda")
    target = after[ids, torch.randint(after.shape[1], (tokens,), generator=gen, device="cuda")]
    ids[torch.rand(tokens, generator=gen, device="cuda") < 0.05] = -1
    return ids, torch.where(ids < 0, torch.full_like(target, -100), target)


def run(steps=60, vocab=8192, width=512, hidden=1536, tokens=8192, depth=3):
    torch.manual_seed(0)
    model = Model(vocab, width, hidden, depth)
    matrices = model.matrices()
    ours = {id(p) for p in matrices}
    optimizers = (Muon(matrices, lr=2e-2), Novak([p for p in model.parameters() if id(p) not in ours], lr=2e-3, weight_decay=0.0))
    gen = torch.Generator(device="cuda").manual_seed(7)
    after = torch.randint(vocab, (vocab, 4), generator=gen, device="cuda")
    losses = []
    for _ in range(steps):
        ids, target = batch(gen, tokens, vocab, after)
        for opt in optimizers:
            opt.zero_grad(set_to_none=True)
        loss = torch.nn.functional.cross_entropy(model(ids).float(), target)
        loss.backward()
        for opt in optimizers:
            opt.step()
        losses.append(float(loss.detach()))
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for flag, default in (("--steps", 60), ("--vocab", 8192), ("--width", 512), ("--hidden", 1536), ("--tokens", 8192), ("--depth", 3)):
        ap.add_argument(flag, type=int, default=default)
    losses = run(**vars(ap.parse_args()))
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f}")
