"""Whoever records or derives operations on tensors: forward-mode derivatives are refused, torch.jit.trace records a call."""
import pytest
import torch
import torch.autograd.forward_ad as fwad

from paper_1804_08378_amd import functional as F

pytestmark = pytest.mark.gpu


def operands():
    g = torch.Generator().manual_seed(0)
    x = torch.randn(2, 24, 6, 5, generator=g).cuda().contiguous(memory_format=torch.channels_last)
    w, b = torch.rand(24, generator=g).cuda(), torch.randn(24, generator=g).cuda()
    return x, w, b, torch.randn(7, 300, generator=g).cuda(), torch.randint(0, 300, (7,), generator=g).cuda()


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("recorded", [False, True])
def test_forward_mode_is_refused(native, recorded, monkeypatch):
    if not native:
        monkeypatch.setattr(F, "_native", False)
    x, w, b, logits, t = operands()
    y, stats = F.group_norm_forward(x, 4, w, b, x)
    r = F.log_probs_forward(logits, t)
    ones = torch.ones(7, device="cuda")
    if recorded:
        for v in (x, w, b, logits):
            v.requires_grad_(True)

    def refused(call, v):
        with pytest.raises((RuntimeError, NotImplementedError)):
            call(fwad.make_dual(v, torch.ones_like(v)))

    with fwad.dual_level():
        refused(lambda v: F.group_norm(v, 4, w, b, x), x)
        refused(lambda v: F.group_norm(x, 4, v, b, x), w)
        refused(lambda v: F.group_norm(x, 4, w, v, x), b)
        refused(lambda v: F.group_norm(x, 4, w, b, v), x)
        refused(lambda v: F.log_probs(v, t), logits)
        refused(lambda v: F.log_probs(v, t, 5), logits)
        if not recorded:  # the single passes
            refused(lambda v: F.group_norm_forward(v, 4, w, b, x), x)
            refused(lambda v: F.group_norm(v, 4, w, b, x, out=torch.empty_like(x)), x)
            refused(lambda v: F.group_norm_backward(x, stats, v, 4, w, b, x), y)
            refused(lambda v: F.group_norm_backward(x, v, y, 4, w, b, x), stats)
            refused(lambda v: F.log_probs_forward(v, t), logits)
            refused(lambda v: F.log_probs_backward(logits, t, r.lse, r.entropy, v), ones)
            refused(lambda v: F.log_probs_backward(logits, t, v, r.entropy, ones), r.lse)
        # tensors without a derivative are taken
        assert torch.equal(F.group_norm(x, 4, w, b, x), y) and torch.equal(F.log_probs(logits, t).logp, r.logp)


def test_function_transforms_are_refused():
    x, w, b, logits, t = operands()
    with pytest.raises(RuntimeError):
        torch.func.jvp(lambda v: F.group_norm(v, 4, w, b), (x,), (torch.ones_like(x),))
    with pytest.raises(RuntimeError):
        torch.func.jvp(lambda v: F.log_probs(v, t).logp, (logits,), (torch.ones_like(logits),))
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda v: F.group_norm(v, 4))(torch.stack([x, x]))
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda v: F.log_probs(v, t).logp)(torch.stack([logits, logits]))


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("native", [True, False])
def test_traced_functions_answer_for_new_inputs(native, grad, monkeypatch):
    if not native:
        monkeypatch.setattr(F, "_native", False)
    x, w, b, logits, t = operands()

    class Twice(torch.nn.Module):  # (parameters of a traced module are its own, not constants)
        def __init__(self):
            super().__init__()
            self.norm = F.GroupNormAct(4, 24, "silu")

        def forward(self, v):
            return self.norm(v, v)

    m = Twice().cuda()
    m.requires_grad_(grad)

    def head(v):
        r = F.log_probs(v, t, 3)
        return r.logp, r.entropy, r.top_index

    with torch.set_grad_enabled(grad):
        traced = torch.jit.trace(m, x, check_trace=False)
        traced_head = torch.jit.trace(head, logits, check_trace=False)
        for i in range(3):
            v, u = x * (i + 1) + i, logits.flip(0) * (i + 1)
            assert torch.equal(traced(v), m(v)), i
            assert all(torch.equal(p, q) for p, q in zip(traced_head(u), head(u))), i


def test_single_passes_are_not_traced():
    x, w, b, logits, t = operands()
    y, stats = F.group_norm_forward(x, 4, w, b)
    r = F.log_probs_forward(logits, t)
    for call, v in ((lambda v: F.group_norm_forward(v, 4, w, b), x), (lambda v: F.group_norm(v, 4, w, b, out=torch.empty_like(x)), x),
                    (lambda v: F.group_norm_backward(x, stats, v, 4, w, b)[:3], y), (lambda v: F.log_probs_forward(v, t)[:2], logits),
                    (lambda v: F.log_probs_backward(v, t, r.lse, r.entropy, r.entropy), logits)):
        with torch.no_grad(), pytest.raises(RuntimeError, match="trace"):
            torch.jit.trace(call, v, check_trace=False)


def test_results_written_over_a_tensor_that_autograd_keeps():
    """`out` counts as a change in place: the gradient that needs the old values is refused, not computed from the new ones."""
    x, w, b, logits, t = operands()
    r = F.log_probs_forward(logits, t)

    def kept(v):
        v = v.clone(memory_format=torch.preserve_format)
        return v, (v * torch.ones_like(v).requires_grad_(True)).sum()

    for like, write in ((x, lambda v: F.group_norm(x, 4, w, b, out=v)), (x, lambda v: F.group_norm_forward(x, 4, w, b, out=v)),
                        (logits, lambda v: F.log_probs_backward(logits, t, r.lse, r.entropy, r.entropy, out=v)),
                        (logits, lambda v: F.log_probs_backward(v, t, r.lse, r.entropy, r.entropy, out=v))):
        v, loss = kept(like)
        loss.backward()  # nothing written: taken
        v, loss = kept(like)
        write(v)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    with torch.inference_mode():
        v = torch.empty_like(x)
        assert torch.equal(F.group_norm(x, 4, w, b, out=v), F.group_norm(x, 4, w, b))
