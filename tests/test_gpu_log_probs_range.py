"""Log probabilities of rows whose logits, or whose masks, are large: against the definition in 64 bits, with tolerances that do not grow with
the logits.

Tolerances.  u = 2^-24.  Everything is a function of the differences from the row's maximum, which 32 bits hold to u of themselves.  A sum of
positive terms is off by under 300 u = 2e-5, so a log probability by 2e-5 and 4 u of itself, the entropy by 2e-5 (1 + entropy).
"""
import math

import pytest
import torch

from paper_1804_08378_amd import functional as F

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U, SUMS = 2.0 ** -24, 2e-5


def definition(x, t):
    """(values, tolerances) of logp and entropy; rows with at least one class that is not at -infinity."""
    x, t = x.cpu().double(), t.cpu()
    d = x - x.amax(1, keepdim=True)
    logp = d - torch.log(torch.exp(d).sum(1, keepdim=True))
    p = torch.exp(logp)
    entropy = (p * torch.where(p > 0, logp.abs(), 0.0)).sum(1)
    mine = logp.gather(1, t[:, None])[:, 0]
    return {"logp": (mine, SUMS + 4 * U * mine.abs()), "entropy": (entropy, SUMS * (1 + entropy))}, logp


def close(got, want, off, label):
    got = got.detach().cpu().double()
    bound = off + U * 1.01 * (want.abs() + off)
    bad = ~((got == want) | ((got - want).abs() <= bound))
    assert not bad.any(), (label, int(bad.sum()), torch.nonzero(bad)[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())


def check(x, t, top=0, label=""):
    print(f"[log probs] {tuple(x.shape)} {x.dtype} top {top} {label}", flush=True)
    want, logp = definition(x, t)
    r = F.log_probs_forward(x, t, top)
    close(r.logp, *want["logp"], "logp")
    close(r.entropy, *want["entropy"], "entropy")
    if top:
        index = torch.sort(x.cpu().float(), dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(r.top_index.cpu().long(), index), "alternatives"
        best = logp.gather(1, index)
        close(r.top_logp, best, SUMS + 4 * U * torch.nan_to_num(best, neginf=0.0).abs(), "top_logp")
    return r


def magnitudes(dtype):
    m = [1e5, 1e6, 1e7, 1e8, 2.0 ** 29, 1e9, 2.0 ** 30, 2.0 ** 30 + 256, 4e9, 1e10, 1e20, 1e30, 2e38, torch.finfo(DTYPES[dtype]).max] if dtype != "f16" else [1e3, 3e4, 65504]
    return m


def masked_rows(classes, mask, dtype):
    """Ordinary logits with masks at the front, at the back, in between, nearly everywhere, over all of the row."""
    g = torch.Generator().manual_seed(classes)
    x = torch.randn(7, classes, generator=g) * 3
    j = torch.arange(classes)
    x[0, : classes // 2] = mask
    x[1, classes - classes // 3:] = mask
    x[2, ::2] = mask
    x[3, j // 8 % 2 == 0] = mask           # whole vectors
    x[4, : classes - 1] = mask
    x[5, 1:] = mask
    x[6] = mask
    return x.to(DTYPES[dtype]).cuda(), torch.tensor([classes - 1, 0, min(1, classes - 1), classes - 1, classes - 1, 0, 0]).cuda()


@pytest.mark.parametrize("classes", [4, 70, 1000, 5003, 60001])
@pytest.mark.parametrize("dtype", DTYPES)
def test_masks_of_any_size(dtype, classes):
    for m in magnitudes(dtype):
        x, t = masked_rows(classes, -m, dtype)
        check(x, t, 3 if classes > 4 else 0, label=f"mask {-m:g}")
        if classes == 5003:  # many rows: none is cut
            check(x.repeat(20, 1), t.repeat(20), 3, label=f"mask {-m:g}")


@pytest.mark.parametrize("classes", [4, 70, 1000, 5003, 60001])
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_at_any_level(dtype, classes):
    """The same row moved up and down: rows of values next to each other, and rows that hold one value only."""
    g = torch.Generator().manual_seed(classes + 1)
    for m in magnitudes(dtype):
        for level in (m, -m):
            limit = torch.finfo(DTYPES[dtype]).max
            x = (torch.randn(4, classes, generator=g).double() * 3 + level).clamp(-limit, limit)
            x[2] = level
            x[3, ::2] = level
            x[3, 1::2] = level * (1 - 2.0 ** -7)
            x = x.to(DTYPES[dtype]).cuda()
            t = torch.tensor([0, classes - 1, 1, 2]).cuda()
            check(x, t, 3 if classes > 4 else 0, label=f"level {level:g}")


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_of_one_value(dtype):
    """n equal classes have probability 1 / n each, whatever the value."""
    n = 32000
    for level in magnitudes(dtype):
        for value in (level, -level):
            x = torch.full((3, n), value, dtype=DTYPES[dtype], device="cuda")
            t = torch.tensor([0, 77, n - 1]).cuda()
            r = F.log_probs_forward(x, t)
            want = torch.full((3,), math.log(n))
            assert torch.allclose(r.entropy.cpu(), want, rtol=2e-5, atol=0) and torch.allclose(r.logp.cpu(), -want, rtol=2e-5, atol=0), value


def test_real_logits_among_far_ones_of_both_signs():
    """Every lane, and every part of a cut row, sees other magnitudes."""
    for classes in (2048, 100003):
        j = torch.arange(classes)
        g = torch.Generator().manual_seed(3)
        noise = torch.randn(6, classes, generator=g) * 2
        x = noise.clone()
        x[0, j % 3 == 0], x[0, j % 3 == 1] = -1e10, -1e30
        x[1] = torch.where(j < classes // 2, -1e38, -1e12)
        x[1, classes - 3] = -2e9                        # the maximum is far too
        x[2] = torch.where(j % 5 == 0, 3e9, 2.9e9)
        x[3] = -1e9 * (1 + j % 7)
        x[4] = torch.where(j // 64 % 2 == 0, -(2.0 ** 30), -(2.0 ** 30) - 128)
        x[5, :] = -math.inf
        x[5, 7], x[5, 9] = -1e30, -1e31
        t = torch.tensor([2, classes - 3, 5, 0, 0, 7]).cuda()
        for dtype in (torch.float32, torch.bfloat16):
            check(x.to(dtype).cuda(), t, 5)
