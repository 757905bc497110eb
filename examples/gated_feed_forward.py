"""Train a gated feed-forward block of sliding-channel layers, then answer single tokens with it.

The block learns a fixed random block of the same form: every step is the gated layer and the layer back, their gradients, and one
orthogonalised momentum update of all three weight matrices.  Serving, it is the branch of a residual stream.

    python examples/gated_feed_forward.py [--steps 200] [--dtype bf16]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2101_00745_amd.nn import GatedFeedForward  # noqa: E402
from paper_2101_00745_amd.optim import OrthogonalMomentum  # noqa: E402

CHANNELS, HIDDEN, TOKENS = 128, 256, 512


def train(steps=200, dtype=torch.float32, seed=0, lr=0.2):
    """The trained block and the losses, relative to that of a block whose result is zero."""
    torch.manual_seed(seed)
    teacher = GatedFeedForward(CHANNELS, HIDDEN, dtype=dtype)
    block = GatedFeedForward(CHANNELS, HIDDEN, dtype=dtype)
    optimiser = OrthogonalMomentum(block.parameters(), lr=lr)
    losses = []
    for step in range(steps):
        for group in optimiser.param_groups:
            group["lr"] = lr * (1 - step / steps)
        x = torch.randn(4, CHANNELS, TOKENS, 1, device="cuda").to(dtype)     # four sequences: tokens are the columns of a map
        with torch.no_grad():
            target = teacher(x).float()
        optimiser.zero_grad()
        loss = (block(x).float() - target).square().mean() / target.square().mean()
        loss.backward()
        optimiser.step()
        losses.append(loss.detach())
    return block, torch.stack(losses).cpu()


@torch.no_grad()
def serve(block, tokens):
    """tokens [N, channels] through the block's residual branch: N maps of one pixel."""
    return tokens + block(tokens[:, :, None, None])[:, :, 0, 0]


def main():
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=200)
    parser.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    args = parser.parse_args()
    block, losses = train(args.steps, {"f32": torch.float32, "bf16": torch.bfloat16}[args.dtype])
    for step in range(0, args.steps, max(1, args.steps // 6)):
        print("step %4d  loss %.4f" % (step, losses[step]))
    print("step %4d  loss %.4f" % (args.steps - 1, losses[-1]))
    tokens = torch.randn(8, CHANNELS, device="cuda", dtype=block.up.weight.dtype)
    print("one token alone and in a batch of eight differ by %.1e at most" % (serve(block, tokens[:1]) - serve(block, tokens)[:1]).abs().max())


if __name__ == "__main__":
    main()
