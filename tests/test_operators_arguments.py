"""Integer arguments that a 32- or 64-bit field cannot hold, or that are no integers: refused, not cut off (no GPU: nothing is launched)."""
import pytest
import torch

from paper_1804_08378_amd import functional as F


@pytest.fixture(autouse=True)
def host_tensors(monkeypatch):
    """Tensors in host memory stand for device tensors; a call that reaches the library fails the test."""
    monkeypatch.setattr(F, "_native", False)
    monkeypatch.setattr(F, "_on_gpu", lambda t, what: None)
    for name in ("bs_group_norm", "bs_group_norm_backward", "bs_log_probs", "bs_log_probs_backward"):
        monkeypatch.setattr(F.bs, name, lambda *a: pytest.fail("called"))


@pytest.mark.parametrize("groups,error", [((1 << 32) + 4, ValueError), (-(1 << 32) + 4, ValueError), (1 << 31, ValueError), (2.5, TypeError), (4.0, TypeError),
                                          ("4", TypeError), (None, TypeError)])
def test_groups(groups, error):
    x = torch.zeros(2, 8, 3, 3).contiguous(memory_format=torch.channels_last)
    with pytest.raises(error):
        F.group_norm(x, groups)
    with pytest.raises(error):
        F.group_norm_forward(x, groups)
    with pytest.raises(error):
        F.group_norm_backward(x, torch.zeros(2, 4, 2), x, groups)


@pytest.mark.parametrize("top,ignore,error", [((1 << 32) + 3, -100, ValueError), (-(1 << 32) + 3, -100, ValueError), (2.0, -100, TypeError), (3, 1.5, TypeError),
                                              (3, 1 << 64, ValueError), (3, (1 << 64) - 100, ValueError), (3, None, TypeError)])
def test_alternatives_and_the_ignored_index(top, ignore, error):
    logits, t = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64)
    with pytest.raises(error):
        F.log_probs(logits, t, top, ignore)
    with pytest.raises(error):
        F.log_probs_forward(logits, t, top, ignore)
    if top == 3:
        with pytest.raises(error):
            F.log_probs_backward(logits, t, torch.zeros(2, dtype=torch.float64), torch.zeros(2), torch.zeros(2), ignore_index=ignore)
