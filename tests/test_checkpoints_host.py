"""What `checkpoints_in_8_bits` does with tensors that stay as they are, without a GPU: tensors in host memory all do."""
import gc
import weakref

import pytest
import torch
from torch import nn

from paper_1804_08378_amd import functional as F


def parameter_changed(w, x):
    y = (x * w).exp() * x
    with torch.no_grad():
        w.mul_(10.0)  # an optimiser's step
    return y


def result_changed(w, x):
    y = (x * w).sigmoid()
    y.mul_(5.0)
    return y


def view_changed(w, x):
    u = x * 1.0
    y = u[:, ::2].sin() * w
    u[:, 1::2].add_(1.0)  # another part of the same memory: autograd counts a tensor's versions together with its views'
    return y


@pytest.mark.parametrize("call", [parameter_changed, result_changed, view_changed])
def test_in_place_changes_are_seen_in_the_block(call):
    """With and without the block, a tensor that autograd keeps and that is changed before the backward pass is refused."""
    for block in (lambda w: torch.enable_grad(), lambda w: F.checkpoints_in_8_bits([w])):
        w, x = torch.ones((), requires_grad=True), torch.randn(3, 4, requires_grad=True)
        with block(w):
            y = call(w, x)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()


def test_changes_before_a_tensor_is_kept_or_of_others_are_allowed():
    w, x = nn.Parameter(torch.full((4,), 2.0)), torch.randn(3, 4, requires_grad=True)
    with F.checkpoints_in_8_bits([w]):
        with torch.no_grad():
            w.mul_(2.0)
        u = x * w
        u.mul_(3.0)            # neither product keeps its result
        y = u.clone().relu_()  # keeps its result as it is behind the change
        z = y.sin()
        other = y.detach().clone().add_(1.0)
    gx, gw = torch.autograd.grad(z.sum(), [x, w], retain_graph=True)
    on = (u.detach() > 0).float() * u.detach().clamp(min=0).cos() * 3.0
    assert torch.equal(other, y.detach() + 1) and torch.allclose(gx, on * 4.0, atol=0, rtol=1e-6) and torch.allclose(gw, (on * x.detach()).sum(0), rtol=1e-5)
    assert all(torch.equal(a, b) for a, b in zip((gx, gw), torch.autograd.grad(z.sum(), [x, w])))  # (a second pass)


class Marked(torch.autograd.Function):
    """x, by a node that holds an object which can be watched."""

    @staticmethod
    def forward(ctx, x, mark):
        ctx.mark = mark
        return x.view_as(x)

    @staticmethod
    def backward(ctx, g):
        return g, None


class Mark:
    pass


@pytest.mark.parametrize("keeps_its_result", [torch.exp, torch.sigmoid, torch.relu, torch.tanh, lambda t: t.softmax(-1), lambda t: t.clone().exp_()])
def test_graphs_without_a_backward_pass_are_freed(keeps_its_result):
    """An operation that keeps its own result: were that very tensor kept, node and tensor would hold each other."""
    for block in (torch.enable_grad, lambda: F.checkpoints_in_8_bits([])):
        x, mark = torch.randn(3, 4, requires_grad=True), Mark()
        alive = weakref.ref(mark)
        with block():
            y = keeps_its_result(Marked.apply(x, mark)) * 2.0
        del mark
        assert alive() is not None
        del y
        gc.collect()
        assert alive() is None


def test_a_model_that_holds_its_result_is_freed():
    """Graphs hold the block's hooks: these hold no model."""
    model, mark = nn.Linear(4, 4), Mark()
    model.mark, alive = mark, weakref.ref(mark)
    with F.checkpoints_in_8_bits(model):
        model.last = model(torch.randn(3, 4, requires_grad=True)).exp()
    del model, mark
    gc.collect()
    assert alive() is None


def test_a_result_that_its_node_keeps_and_that_a_program_holds():
    """The kept tensor is another one with the same memory: changes are still seen, gradients of gradients go through it."""
    x = torch.randn(5, dtype=torch.float64, requires_grad=True)
    with F.checkpoints_in_8_bits([]):
        y = x.exp()
        (g,) = torch.autograd.grad(y.sum(), x, create_graph=True)
        (h,) = torch.autograd.grad(g.sum(), x)
    assert torch.equal(h, x.detach().exp()) and torch.equal(g, y)


# ------------------------------------------------------------------------------------------------ statistics
def told(call, *operands):
    """Sizes of what `call` keeps, and which of them are taken for statistics."""
    statistics, seen = F._Statistics(), []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: seen.append((tuple(t.shape), statistics.found(t))) or t.detach(), lambda t: t):
        call(*operands)
    return [s for s, found in seen if found], [s for s, found in seen if not found]


def operand(*sizes):
    return torch.randn(*sizes, requires_grad=True) * 1.0


@pytest.mark.parametrize("call,statistic", [
    (lambda x: nn.functional.scaled_dot_product_attention(x, x * 2, x * 3), (4, 8, 16)),
    (lambda x: nn.functional.group_norm(x, 4), (4, 4)),
    (lambda x: x.logsumexp(-1), (4, 8, 16)),
    (lambda x: x.logsumexp(1), (4, 16, 32)),
    (lambda x: x.logsumexp(1, keepdim=True), (4, 1, 16, 32)),
    (lambda x: x.norm(dim=1), (4, 16, 32)),
    (lambda x: x.std(dim=2), (4, 8, 32)),
    (lambda x: nn.functional.layer_norm(x, (32,)), (4, 8, 16, 1)),
    (lambda x: nn.functional.normalize(x, dim=1), (4, 1, 16, 32)),
    (lambda x: nn.functional.dropout(x), (4, 8, 16, 32)),  # (a mask)
])
def test_statistics_are_told(call, statistic):
    found, others = told(call, operand(4, 8, 16, 32))
    assert statistic in found and statistic not in [s for s in others if s != (4, 8, 16, 32)]
    assert all(s == (4, 8, 16, 32) for s in others)


def test_operands_are_no_statistics():
    x = operand(4, 8, 16, 32)
    for call in (torch.exp, torch.sin, lambda t: t * t, lambda t: t.relu().view(32, 16, 32).sin().permute(1, 0, 2).exp(), lambda t: [u.sin() for u in t.chunk(2, 1)],
                 lambda t: [u.sin() for u in t.unbind(0)][:0], lambda t: t.softmax(-1), lambda t: nn.functional.avg_pool2d(t.relu(), 2).exp(),
                 lambda t: nn.functional.max_pool2d(t, 2)):
        found, others = told(call, x)
        assert others and found in ([], [(4, 8, 8, 16)]), (found, others)  # (a maximum's picks are whole numbers without a gradient)

    class Two(torch.autograd.Function):  # as a layer normalisation and its total
        @staticmethod
        def forward(ctx, t):
            a, b = t + 1, t + 2
            ctx.save_for_backward(t, b)
            return a, b

    assert told(Two.apply, x) == ([], [(4, 8, 16, 32)] * 2)


def test_sizes_are_forgotten():
    """A tensor of a step's sizes is an operand again once others have been kept: a loop over the steps of a sequence."""
    x, h = operand(50, 64, 96), operand(64, 96)

    def loop(x, h):
        x.sin()
        for _ in range(50):
            h = h.sin()

    found, others = told(loop, x, h)
    assert found == [(64, 96)] * 16 and len(others) == 35


def test_a_model_with_sparse_buffers():
    m = nn.Linear(4, 4)
    m.register_buffer("graph", torch.eye(4).to_sparse())
    x = torch.randn(4, 4, requires_grad=True)
    with F.checkpoints_in_8_bits(m):
        y = torch.sparse.mm(m.graph, m(x))
    assert torch.allclose(torch.autograd.grad(y.sum(), x)[0], m.weight.detach().sum(0).expand(4, 4), atol=1e-6)


def test_statistics_that_a_layer_updates_itself_are_no_change():
    """A batch normalisation in training mode keeps its running statistics, and moves them on in the next pass: no backward pass reads them."""
    m = nn.Sequential(nn.Conv2d(3, 4, 1), nn.BatchNorm2d(4))
    x = torch.randn(2, 3, 4, 4)
    grads = []
    for block in (torch.enable_grad, lambda: F.checkpoints_in_8_bits(m)):
        with block():
            y = m(x) * 1.0 + m(x * 2.0)
        grads.append(torch.autograd.grad(y.square().sum(), list(m.parameters())))
    assert all(torch.allclose(a, b, rtol=1e-4, atol=1e-4) for a, b in zip(*grads))
