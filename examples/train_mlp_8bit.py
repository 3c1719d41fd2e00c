"""Trains a few pre-norm MLP blocks on a synthetic regression with NOVAK, once with the
activations of the backward pass kept in 8 bits and once by torch's own operators in
bfloat16, from the same start; prints both losses and the memory that each keeps between
the forward and the backward pass.

    python examples/train_mlp_8bit.py [--steps 60] [--width 768] [--hidden 2304] [--tokens 12608]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_07876_b200.block import MlpBlock8  # noqa: E402
from paper_2601_07876_b200.optim import Novak  # noqa: E402


def plain_block(block, x):
    """The same block by torch's operators."""
    up, down = block.up, block.down
    h = torch.nn.functional.layer_norm(x.float(), x.shape[-1:], up.gamma, up.beta, up.eps).to(x.dtype)
    u = torch.nn.functional.linear(h, up.weight.to(x.dtype), up.bias.to(x.dtype))
    a = torch.nn.functional.gelu(u)
    return x + torch.nn.functional.linear(a, down.weight.to(x.dtype), down.bias.to(x.dtype))


def train(blocks, forward, steps, width, tokens):
    """(losses, bytes kept between the two passes)"""
    gen = torch.Generator(device="cuda").manual_seed(7)
    teacher = torch.empty(width, width, device="cuda").normal_(0.0, width ** -0.5, generator=gen)
    params = [p for b in blocks for p in b.parameters()]
    opt = Novak(params, lr=2e-3, weight_decay=0.0, lookahead_k=5)
    losses, kept = [], 0
    for _ in range(steps):
        x = torch.empty(tokens, width, device="cuda").normal_(generator=gen)
        target = torch.tanh(x @ teacher)
        opt.zero_grad(set_to_none=True)
        y = x.to(torch.bfloat16)
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        for block in blocks:
            y = forward(block, y)
        kept = torch.cuda.memory_allocated() - before
        loss = (y.float() - target).square().mean()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
    return losses, kept


def run(steps=60, width=768, hidden=2304, tokens=12608, depth=3):
    result = {}
    for name, forward in (("8 bits", lambda b, x: b(x)), ("torch bf16", plain_block)):
        torch.manual_seed(0)
        blocks = [MlpBlock8(width, hidden) for _ in range(depth)]
        result[name] = train(blocks, forward, steps, width, tokens)
    return result


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for flag, default in (("--steps", 60), ("--width", 768), ("--hidden", 2304), ("--tokens", 12608), ("--depth", 3)):
        ap.add_argument(flag, type=int, default=default)
    args = ap.parse_args()
    for name, (losses, kept) in run(**vars(args)).items():
        print(f"{name:>10}: loss {losses[0]:.4f} -> {losses[-1]:.4f}, {kept / 2**20:.0f} MiB kept for the backward pass")
