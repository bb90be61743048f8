"""A residual classifier trained from scratch: group normalisation with the residual addition and ReLU behind it in every block, log
probabilities at the end for the loss, the confidence and the accuracy.

    python examples/train_from_scratch.py [--steps 100] [--batch 64] [--dtype bf16]

The data are synthetic: each class is a fixed random pattern of coloured squares, shown at random strengths in noise.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch
from torch import nn

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1804_08378_amd.functional import GroupNormAct, log_probs  # noqa: E402


class Block(nn.Module):
    """Two 3x3 convolutions; the second normalisation adds the block's input before its ReLU, in one pass."""

    def __init__(self, cin, c, stride):
        super().__init__()
        self.conv1 = nn.Conv2d(cin, c, 3, stride, 1, bias=False)
        self.norm1 = GroupNormAct(8, c, "relu")
        self.conv2 = nn.Conv2d(c, c, 3, 1, 1, bias=False)
        self.norm2 = GroupNormAct(8, c, "relu")
        self.down = None
        if stride != 1 or cin != c:
            self.down = nn.Sequential(nn.Conv2d(cin, c, 1, stride, bias=False), GroupNormAct(8, c, "identity"))

    def forward(self, x):
        return self.norm2(self.conv2(self.norm1(self.conv1(x))), x if self.down is None else self.down(x))


class Classifier(nn.Module):
    def __init__(self, width=32, classes=10):
        super().__init__()
        self.stem = nn.Sequential(nn.Conv2d(3, width, 3, 1, 1, bias=False), GroupNormAct(8, width, "relu"))
        self.blocks = nn.Sequential(Block(width, width, 1), Block(width, 2 * width, 2), Block(2 * width, 4 * width, 2))
        self.fc = nn.Linear(4 * width, classes)

    def forward(self, x):
        return self.fc(self.blocks(self.stem(x)).mean((2, 3)))


def batches(batch, classes, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    patterns = 2 * torch.randn(classes, 3, 1, 1, generator=g, device="cuda") + \
        torch.randn(classes, 3, 8, 8, generator=g, device="cuda").repeat_interleave(4, 2).repeat_interleave(4, 3)
    while True:
        target = torch.randint(0, classes, (batch,), generator=g, device="cuda")
        strength = torch.rand(batch, 1, 1, 1, generator=g, device="cuda") + 0.5
        image = patterns[target] * strength + 0.5 * torch.randn(batch, 3, 32, 32, generator=g, device="cuda")
        yield image.to(dtype).contiguous(memory_format=torch.channels_last), target


def train(steps=100, batch=64, dtype=torch.bfloat16, classes=10, seed=0, report=print):
    """Returns the loss and the accuracy of every step."""
    torch.manual_seed(seed)
    model = Classifier(classes=classes).cuda().to(dtype).to(memory_format=torch.channels_last)
    optimizer = torch.optim.SGD(model.parameters(), lr=0.02, momentum=0.9)
    history = []
    for step, (image, target) in zip(range(steps), batches(batch, classes, dtype, seed)):
        r = log_probs(model(image), target, top=1)
        loss = -r.logp.mean()
        optimizer.zero_grad(set_to_none=True)
        loss.backward()
        optimizer.step()
        accuracy = (r.top_index[:, 0] == target).float().mean()
        history.append((float(loss.detach()), float(accuracy)))
        if step % 10 == 0 or step + 1 == steps:
            report(f"step {step:4d}  loss {history[-1][0]:.4f}  accuracy {history[-1][1]:.2f}  entropy {float(r.entropy.mean().detach()):.3f}")
    return history


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=100)
    p.add_argument("--batch", type=int, default=64)
    p.add_argument("--dtype", choices=["f32", "bf16", "f16"], default="bf16")
    a = p.parse_args()
    train(a.steps, a.batch, {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[a.dtype])
