"""A gated feed-forward block on the FP8 operators with block scales: it is fine-tuned for some steps towards a target map
with 8-bit activation checkpoints, then serves single tokens from the same weights.

    python examples/gated_ffn_fp8.py [--tokens 256] [--features 512] [--hidden 1408] [--steps 40]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2307_09782_b200 import binding  # noqa: E402
from paper_2307_09782_b200.gated_ffn import GatedFfnFp8  # noqa: E402


def train(tokens: int, features: int, hidden: int, steps: int, lr: float = 3e-3, seed: int = 0, log=print):
    """FP32 master weights, quantized anew each step; Adam on the gradients of the quantized block.  Returns the losses
    and the block with the final weights."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std):
        return torch.randn(shape, generator=gen, device="cuda") * std

    x = normal(tokens, features, std=1.0).to(torch.bfloat16)
    target = torch.tanh(x.float() @ normal(features, features, std=features ** -0.5))
    master = [normal(hidden, features, std=features ** -0.5), normal(hidden, features, std=features ** -0.5),
              normal(features, hidden, std=hidden ** -0.5)]
    opt = torch.optim.Adam(master, lr=lr)
    losses = []
    for step in range(steps):
        ffn = GatedFfnFp8.from_weights(*master, mode="M1", training=True)
        y, saved = ffn.forward_train(x, out_dtype=torch.float32)
        diff = y - target
        losses.append(float((diff * diff).mean()))
        # gradients of small mean losses are far below 1: they are scaled per block, not globally
        _, dwgu, dwd = ffn.backward((diff * (2.0 / diff.numel())).to(torch.bfloat16), saved, out_dtype=torch.float32)
        for w, g in zip(master, (dwgu[0], dwgu[1], dwd)):
            w.grad = g
        opt.step()
        if log and step % 10 == 0:
            log(f"step {step:3d}  loss {losses[-1]:.5f}  kept for the backward pass: {saved.numel() / 1e6:.2f} MB "
                f"(bf16 would be {2 * tokens * (features + 3 * hidden) / 1e6:.2f} MB)")
    return losses, GatedFfnFp8.from_weights(*master, mode="M1"), x


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=256)
    ap.add_argument("--features", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1408)
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    losses, ffn, x = train(a.tokens, a.features, a.hidden, a.steps)
    print(f"loss {losses[0]:.5f} -> {losses[-1]:.5f}")
    whole = ffn.forward(x)
    one = torch.cat([ffn.forward(x[i:i + 1]) for i in range(8)])  # token by token, as in decoding
    print(f"single tokens against the batch: max difference {float((one - whole[:8]).abs().max()):.4f} "
          f"(bf16 results of another summation order); {binding.launch_count()} kernel launches")


if __name__ == "__main__":
    main()
