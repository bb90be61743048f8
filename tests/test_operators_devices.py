"""Tensors on a device that is not the current one."""
import contextlib

import pytest
import torch

from paper_1804_08378_amd import functional as F


def everything(device):
    g = torch.Generator().manual_seed(0)
    x = torch.randn(2, 64, 60, 60, generator=g).to(device).contiguous(memory_format=torch.channels_last)
    logits, t = torch.randn(5, 3000, generator=g).to(device), torch.arange(5, device=device)
    y, stats = F.group_norm_forward(x, 8, activation="silu")
    r = F.log_probs_forward(logits, t, 3)
    ones = torch.ones(5, device=device)
    return [y, stats, F.group_norm_backward(x, stats, y, 8, activation="silu")[0], *r, F.log_probs_backward(logits, t, r.lse, r.entropy, ones)]


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_tensors_of_another_device(native, monkeypatch):
    if torch.cuda.device_count() < 2:
        pytest.skip("needs two GPUs")
    if not native:
        monkeypatch.setattr(F, "_native", False)
    want = everything("cuda:0")
    got = everything("cuda:1")
    assert torch.cuda.current_device() == 0
    assert all(torch.equal(a, b.to("cuda:0")) for a, b in zip(want, got))


def test_the_tensors_device_is_current_while_the_library_is_called(monkeypatch):
    """The Python calls, without a GPU: tensors in host memory stand for device tensors and nothing is launched."""
    inside, seen = [], []

    @contextlib.contextmanager
    def device(dev):
        inside.append(dev)
        yield
        inside.pop()

    class Stream:
        cuda_stream = 0

    monkeypatch.setattr(F, "_native", False)
    monkeypatch.setattr(F, "_on_gpu", lambda t, what: None)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev: Stream)
    for name in ("bs_group_norm", "bs_group_norm_backward", "bs_log_probs", "bs_log_probs_backward"):
        monkeypatch.setattr(F.bs, name, lambda *a, name=name: seen.append((name, list(inside))))
    everything("cpu")
    here = [torch.device("cpu")]
    assert seen == [("bs_group_norm", here), ("bs_log_probs", here), ("bs_group_norm_backward", here), ("bs_log_probs_backward", here)]
