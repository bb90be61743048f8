"""Operands whose memory holds the numbers with the other sign: the imaginary part of a conjugate is a view that turns it when it is read."""
import pytest
import torch

from paper_1804_08378_amd import functional as F

pytestmark = pytest.mark.gpu


def negated(*sizes):
    """Such a view, and the same numbers as an ordinary tensor."""
    t = torch.randn(*sizes, dtype=torch.complex64, device="cuda").conj().imag
    assert t.is_neg()
    return t, t.resolve_neg().contiguous()


@pytest.mark.parametrize("native", [True, False])
def test_group_normalisation_of_one_channel(native, monkeypatch):
    """Pixels two elements apart are read in place."""
    if not native:
        monkeypatch.setattr(F, "_native", False)
    (x, px), (r, pr), (g, pg) = (negated(3, 1, 5, 7) for _ in range(3))
    y, stats = F.group_norm_forward(x, 1, residual=r, activation="silu")
    want, _ = F.group_norm_forward(px, 1, residual=pr, activation="silu")
    assert torch.equal(y, want)
    for a, b in zip(F.group_norm_backward(x, stats, g, 1, residual=r, activation="silu"), F.group_norm_backward(px, stats, pg, 1, residual=pr, activation="silu")):
        assert (a is None and b is None) or torch.equal(a, b)
    with pytest.raises(ValueError):
        F.group_norm(px, 1, out=negated(3, 1, 5, 7)[0])


@pytest.mark.parametrize("native", [True, False])
def test_parameters_and_rows_of_one_element(native, monkeypatch):
    if not native:
        monkeypatch.setattr(F, "_native", False)
    x = torch.randn(4, 1, 2, 2, device="cuda")
    w, b = negated(1)[0], negated(1)[0]
    for call in (lambda: F.group_norm(x, 1, w), lambda: F.group_norm(x, 1, None, b), lambda: F.layer_norm(x[:, :, 0, :1], w), lambda: F.layer_norm(x[:, :, 0, :1], None, b),
                 lambda: F.layer_norm_backward(x[:, :, 0, :1], torch.ones(4, 1, 2, device="cuda"), x[:, :, 0, :1], w)):
        with pytest.raises(ValueError, match="negated"):
            call()
    (z, pz), (g, pg) = negated(6, 1), negated(6, 1)
    r = F.layer_norm_forward(z, eps=1.0, checkpoint=True)
    assert torch.equal(r.y, F.layer_norm(pz, eps=1.0)) and torch.equal(F.unpack8(r.kept), F.unpack8(F.pack8(pz)))
    assert torch.equal(F.activate(z, "silu", g), F.activate(pz, "silu", pg))
    assert all(torch.equal(a, b) for a, b in zip(F.activate_backward(z, g, "silu", z), F.activate_backward(pz, pg, "silu", pz)))


@pytest.mark.parametrize("native", [True, False])
def test_log_probabilities(native, monkeypatch):
    if not native:
        monkeypatch.setattr(F, "_native", False)
    (z, pz), t = negated(5, 1), torch.zeros(5, dtype=torch.int64, device="cuda")
    r, want = F.log_probs(z, t, top=1), F.log_probs(pz, t, top=1)
    assert all(torch.equal(a, b) for a, b in zip(r, want))  # (the sum of exponentials is the class's own logit)
    logits, one = torch.randn(1, 9, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    r, (g, pg) = F.log_probs(logits, one), negated(1)
    assert torch.equal(F.log_probs_backward(logits, one, r.lse, r.entropy, g, g), F.log_probs_backward(logits, one, r.lse, r.entropy, pg, pg))
    with pytest.raises(ValueError):
        F.log_probs_backward(pz, t, want.lse, want.entropy, pz[:, 0].contiguous(), out=z)
