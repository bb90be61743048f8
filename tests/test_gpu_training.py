"""A network trained from scratch with the group normalisation and the log probabilities: its gradients against the same network in plain
torch, and the example's loss."""
import importlib.util
import os

import pytest
import torch
from torch import nn

from paper_1804_08378_amd.functional import GroupNormAct, log_probs

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("train_from_scratch", os.path.join(ROOT, "examples", "train_from_scratch.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


class Plain(nn.Module):
    """GroupNormAct in elementary operations of any type, on any device."""

    def __init__(self, m):
        super().__init__()
        self.m = m

    def forward(self, x, residual=None):
        n, c, h, w = x.shape
        v = x.reshape(n, self.m.num_groups, -1)
        v = (v - v.mean(2, keepdim=True)) / (v.var(2, unbiased=False, keepdim=True) + self.m.eps).sqrt()
        v = v.view(x.shape) * self.m.weight.view(1, c, 1, 1) + self.m.bias.view(1, c, 1, 1)
        v = v if residual is None else v + residual
        return v.clamp(min=0) if self.m.activation == "relu" else v


def plain_copy(model):
    import copy
    model = copy.deepcopy(model).cpu().double()
    for parent in list(model.modules()):
        for name, child in list(parent.named_children()):
            if isinstance(child, GroupNormAct):
                setattr(parent, name, Plain(child))
    return model


def test_gradients_of_a_network():
    """float32 against 64 bits.  Seven normalised layers, each with roundings of 1e-6 relative to its gradient (convolutions among them); a ReLU
    whose input is within a rounding of 0 moves a gradient by one cell's share of some thousands: 1e-3 of a parameter's gradient norm covers both."""
    m = example()
    torch.manual_seed(1)
    model = m.Classifier(width=16).cuda().to(memory_format=torch.channels_last)
    image, target = next(m.batches(8, 10, torch.float32, 3))
    r = log_probs(model(image), target, top=3)
    (-r.logp.mean() - 0.1 * r.entropy.mean()).backward()
    ref = plain_copy(model)
    logp = torch.log_softmax(ref(image.cpu().double()), 1)
    want = -logp.gather(1, target.cpu()[:, None]).mean() + 0.1 * (logp.exp() * logp).sum(1).mean()
    ref.zero_grad()
    want.backward()
    assert abs(float((-r.logp.mean() - 0.1 * r.entropy.mean()).detach()) - float(want.detach())) <= 1e-5 * (1 + abs(float(want.detach())))
    grads = {n.replace(".m.", "."): p.grad for n, p in ref.named_parameters()}
    for name, p in model.named_parameters():
        a, b = p.grad.cpu().double(), grads[name]
        assert float((a - b).norm()) <= 1e-3 * float(b.norm()) + 1e-7, name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_example_learns(dtype):
    history = example().train(steps=100, batch=64, dtype=dtype, report=lambda line: print(line, flush=True))
    first, last = history[0][0], sum(h[0] for h in history[-5:]) / 5
    assert last < 0.5 * first and sum(h[1] for h in history[-5:]) / 5 > 0.8, history[-5:]
