"""Log probabilities, entropy, top alternatives and their gradient on the GPU, against the definition in 64 bits.

Tolerances.  u = 2^-24.  The sums' terms are positive and are added in chains of at most a few hundred; relative error under 300 u = 2e-5 at
worst.  lse then is off by 2e-5 and by 2 u of the largest logit and of itself, a log probability by 2 u of its logit more, the entropy
(a sum of terms p |log p|, at most 2e-5 of their sum) by 2e-5 (1 + entropy) and the same roundings.  p is off by the error of lse and of its own exponent, 2 u of it.
"""
import math

import pytest
import torch

from paper_1804_08378_amd import functional as F

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROUNDING = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a unit in the last place of 24, 8, 11 significant bits
U = 2.0 ** -24


class Reference:
    def __init__(self, logits, targets, top, ignore=-100):
        x = logits.detach().cpu().double()
        self.x, self.targets, self.ignore = x, None if targets is None else targets.cpu().long(), ignore
        m = x.amax(1, keepdim=True)
        base = torch.where(m == -math.inf, 0.0, m)
        self.lse = (base + torch.log(torch.exp(x - base).sum(1, keepdim=True)))[:, 0]
        self.none = self.lse == -math.inf
        self.logp = torch.where(self.none[:, None], -math.inf, x - self.lse[:, None])
        self.p = torch.exp(self.logp)
        self.plogp = torch.where(self.p > 0, self.p * self.logp, torch.where(self.p == 0, 0.0, math.nan))
        self.entropy = -self.plogp.sum(1)
        finite = torch.where(torch.isfinite(x), x.abs(), 0.0)
        self.off = 2e-5 + 4 * U * (finite.amax(1) + torch.nan_to_num(self.lse, 0, 0, 0).abs())
        if self.targets is not None:
            known = (self.targets >= 0) & (self.targets < x.shape[1])
            mine = self.logp.gather(1, self.targets.clamp(0, x.shape[1] - 1)[:, None])[:, 0]
            self.mine = torch.where(self.targets == ignore, 0.0, torch.where(known, mine, math.nan))
        if top:
            self.index = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
            self.top = self.logp.gather(1, self.index)

    def grad(self, g, h):
        g = torch.zeros_like(self.lse) if g is None else g.cpu().double()
        h = torch.zeros_like(self.lse) if h is None else h.cpu().double()
        if self.targets is not None:
            g = torch.where(self.targets == self.ignore, 0.0, g)
        dx = -g[:, None] * self.p - h[:, None] * (self.plogp + self.p * self.entropy[:, None])
        if self.targets is not None:
            rows = torch.nonzero((self.targets >= 0) & (self.targets < dx.shape[1]))[:, 0]
            dx[rows, self.targets[rows]] += g[rows]
        dx[self.none] = 0.0
        rel = 2 * self.off[:, None] + 4 * U * torch.where(torch.isfinite(self.logp), self.logp.abs(), 0.0)
        lp = torch.where(torch.isfinite(self.logp), self.logp.abs(), 0.0) + self.entropy.abs()[:, None]
        off = rel * self.p * (g.abs()[:, None] + h.abs()[:, None] * (lp + 1)) + 4 * U * dx.abs() + 1e-30
        off = off + self.p * h.abs()[:, None] * 2 * (self.off + 2e-5 * (1 + self.entropy))[:, None]
        return dx, off


def close(got, want, off, label, rounding=2.0 ** -24):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, label
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bound = off + rounding * 1.01 * (want.abs() + off) + (2.0 ** -25 if rounding == ROUNDING["f16"] else 0)
    bad = ~(same | ((got - want).abs() <= bound))
    assert not bad.any(), (label, int(bad.sum()), got[bad][:4].tolist(), want[bad][:4].tolist())


def make(rows, classes, dtype, seed=0, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, classes, generator=g) * scale).to(DTYPES[dtype]).cuda()
    t = torch.randint(0, classes, (rows,), generator=g).cuda()
    return x, t, (torch.randn(rows, generator=g)).cuda(), (torch.randn(rows, generator=g) * 0.3).cuda()


def check(x, t, top, g=None, h=None, ignore=-100):
    dtype = [k for k, v in DTYPES.items() if v == x.dtype][0]
    print(f"[log probs] {tuple(x.shape)} {dtype} strides {x.stride()} top {top}", flush=True)
    ref = Reference(x, t, top, ignore)
    r = F.log_probs_forward(x, t, top, ignore)
    torch.cuda.synchronize()
    close(r.lse, ref.lse, ref.off, "lse")
    close(r.entropy, ref.entropy, ref.off + 2e-5 * (1 + torch.nan_to_num(ref.entropy)), "entropy")
    if t is not None:
        close(r.logp, ref.mine, ref.off + 4 * U * torch.nan_to_num(ref.mine, 0, 0, 0).abs(), "logp")
    if top:
        assert torch.equal(r.top_index.cpu().long(), ref.index), "indices"
        close(r.top_logp, ref.top, ref.off[:, None] + 4 * U * torch.nan_to_num(ref.top, 0, 0, 0).abs(), "top_logp")
    if g is not None or h is not None:
        dx = F.log_probs_backward(x, t, r.lse, r.entropy, g, h, ignore)
        torch.cuda.synchronize()
        want, off = ref.grad(g, h)
        close(dx, want, off, "grad", ROUNDING[dtype])
    return r, ref


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,classes", [(1, 1), (1, 2), (5, 7), (3, 63), (4, 64), (2, 65), (17, 1000), (3, 1023), (2, 4097), (64, 10),
                                          (9, 50021), (1, 131072), (2, 262147), (700, 333)])
def test_sizes(rows, classes, dtype):
    x, t, g, h = make(rows, classes, dtype, rows + classes)
    check(x, t, min(classes, 5), g, h)


@pytest.mark.parametrize("top", [0, 1, 2, 7, 20, 31, 32])
@pytest.mark.parametrize("dtype", DTYPES)
def test_top_alternatives(top, dtype):
    for rows, classes in ((33, 32), (6, 1000), (2, 30011), (1, 100003)):
        x, t, _, _ = make(rows, classes, dtype, top)
        check(x, t, min(top, classes))


@pytest.mark.parametrize("classes", [40, 777, 20011, 140001])
def test_ties_go_to_the_lowest_index(classes):
    """All equal; few values; ascending and descending rows; the best ones together; zeros of either sign."""
    j = torch.arange(classes)
    rows = [torch.full((classes,), 1.5), (j * 7919 % 5).float(), j.float() / classes, -j.float() / classes, torch.where(j >= classes - 40, 5.0, 0.0),
            torch.where(j % 2 == 0, 0.0, -0.0), (j // 64 % 3).float(), torch.where(j < 33, 2.0, (j % 100) / 100.0)]
    x = torch.stack(rows).cuda()
    t = torch.zeros(len(rows), dtype=torch.int64).cuda()
    for dtype in DTYPES.values():
        check(x.to(dtype), t, 32)


def test_masked_classes_and_empty_rows():
    x, t, g, h = make(8, 3001, "f32", 3)
    x[0, 100:] = -math.inf           # most classes masked
    x[1, :] = -math.inf              # nothing left
    x[2, :] = -math.inf
    x[2, 2999] = -3.0                # one class left
    t[2] = 2999
    t[0] = 2000                      # a masked target: log probability -infinity
    x[3] = torch.finfo(torch.float32).min  # masked by the type's lowest value: all equal
    x[4, 1::2] = torch.finfo(torch.float32).min
    t[5] = -100                      # ignored
    t[6] = 3001                      # not a class
    t[7] = -1
    h[6] = h[7] = 0
    for top in (0, 20):
        r, ref = check(x, t, top, None, h)
        assert r.logp[1] == -math.inf and r.entropy[1] == 0 and r.entropy[2] == 0 and r.logp[2] == 0 and r.logp[5] == 0
        assert r.logp[0] == -math.inf and torch.isnan(r.logp[6:]).all()
    r, ref = check(x[:6].contiguous(), t[:6], 0, g[:6], h[:6])
    r = F.log_probs_forward(x, t)
    dx = F.log_probs_backward(x, t, r.lse, r.entropy, g, None)
    assert torch.isnan(dx[6:]).all() and torch.equal(dx[1], torch.zeros_like(dx[1])) and torch.equal(dx[5], torch.zeros_like(dx[5]))


@pytest.mark.parametrize("dtype", DTYPES)
def test_masked_classes_in_every_type(dtype):
    x, t, g, h = make(5, 2050, dtype, 4)
    x[:, 2000:] = -math.inf
    x[1, 3:] = -math.inf
    x[2] = -math.inf
    t.clamp_(max=2)
    check(x, t, 20, g, h)


def test_infinite_and_nan_logits():
    x, t, g, h = make(4, 500, "f32", 9)
    x[1, 77] = math.nan
    x[2, 400] = math.inf
    x[3, 10] = math.nan
    x[3, :5] = -math.inf
    r = F.log_probs_forward(x, t, 3)
    for i in (1, 2, 3):
        assert torch.isnan(r.logp[i]) and torch.isnan(r.entropy[i]) and torch.isnan(r.lse[i]) and torch.isnan(r.top_logp[i]).all()
    assert r.top_index[1, 0] == 77 and r.top_index[2, 0] == 400 and r.top_index[3, 0] == 10
    dx = F.log_probs_backward(x, t, r.lse, r.entropy, g, h)
    assert torch.isnan(dx[1:]).all() and torch.isfinite(dx[0]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_and_sharp_logits(dtype):
    x, t, g, h = make(6, 900, dtype, 12, scale=10.0)
    x[0] += 1000
    x[1] -= 1000
    x[2, 5] += 200  # nearly certain
    t[2] = 5
    check(x, t, 8, g, h)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset,larger", [(0, 1024), (1, 1003), (8, 1016)])
def test_rows_apart_and_unaligned(offset, larger, dtype):
    x, t, g, h = make(7, 1001, dtype, 5)
    big = torch.full((7, larger), 50.0, dtype=x.dtype, device="cuda")
    inside = big[:, offset:offset + 1001]
    inside.copy_(x)
    r, _ = check(inside, t, 5, g, h)
    out = torch.full_like(big, 9.0)
    F.log_probs_backward(inside, t, r.lse, r.entropy, g, h, out=out[:, offset:offset + 1001])
    assert torch.equal(out[:, offset:offset + 1001], F.log_probs_backward(x, t, r.lse, r.entropy, g, h))
    assert (out[:, :offset] == 9).all() and (out[:, offset + 1001:] == 9).all()
    spread = torch.stack([x, x], 2)[:, :, 0]  # classes not contiguous: copied
    assert torch.equal(F.log_probs_forward(spread, t).logp, F.log_probs_forward(x, t).logp)


def test_forms_of_the_call():
    x, t, g, h = make(12, 345, "bf16", 2)
    a, b = F.log_probs_forward(x, t, 4), F.log_probs_forward(x, t.int(), 4)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    c = F.log_probs_forward(x, None, 4)
    assert c.logp is None and torch.equal(c.entropy, a.entropy) and torch.equal(c.top_index, a.top_index)
    check(x, None, 0, None, h)
    check(x, t, 0, g, None)
    want = F.log_probs_backward(x, t, a.lse, a.entropy, g, h)
    F.log_probs_backward(x, t, a.lse, a.entropy, g, h, out=x)
    assert torch.equal(x, want)
    empty = F.log_probs_forward(x[:0], t[:0], 4)
    assert empty.logp.shape == (0,) and empty.top_index.shape == (0, 4)
    assert F.log_probs_backward(x[:0], t[:0], empty.lse, empty.entropy, g[:0]).shape == (0, 345)


def test_autograd():
    x, t, g, h = make(20, 1000, "f32", 8)
    t[3] = -100
    x.requires_grad_(True)
    r = F.log_probs(x, t, 5)
    assert not r.top_logp.requires_grad and not r.lse.requires_grad
    ((r.logp * g).sum() + (r.entropy * h).sum()).backward()
    with torch.no_grad():
        want = F.log_probs_backward(x, t, r.lse, r.entropy, g, h)
    assert torch.equal(x.grad, want)
    x.grad = None
    (-F.log_probs(x, t).logp).sum().backward()
    z = x.detach().double().requires_grad_(True)
    torch.nn.functional.cross_entropy(z.cpu(), t.cpu(), ignore_index=-100, reduction="sum").backward()
    close(x.grad, z.grad.cpu(), torch.full((20, 1000), 1e-4), "cross entropy")
    assert F.log_probs(x.detach(), t).logp.requires_grad is False


def test_gradient_against_differences():
    """Central differences of the forward pass.  Steps of 2^-6 along a direction whose largest entry is 1: third-order terms under 1e-4, the
    roundings of a row's two results (values of size 10) 10 * 2^-23 / 2^-6 = 1e-4 each, 8 rows."""
    x, t, g, h = make(8, 50, "f32", 21, scale=1.0)
    r = F.log_probs_forward(x, t)
    dx = F.log_probs_backward(x, t, r.lse, r.entropy, g, h)
    v = torch.randn(8, 50, generator=torch.Generator().manual_seed(1)).cuda()
    v = v / v.abs().max()
    value = []
    for sign in (1, -1):
        q = F.log_probs_forward(x + sign * 2.0 ** -6 * v, t)
        value.append(float((q.logp.double() * g).sum() + (q.entropy.double() * h).sum()))
    assert abs((value[0] - value[1]) * 2.0 ** 5 - float((dx.double() * v).sum())) <= 5e-3


def test_offsets_beyond_32_bits():
    """33 rows of 2^26 + 3 classes: 2.2 G elements; the row's head repeats down to its end."""
    rows, classes = 33, (1 << 26) + 3
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GiB")
    x = torch.full((rows, classes), -20.0, dtype=torch.bfloat16, device="cuda")
    x[:, classes - 1] = 8.0
    x[:, 12345] = 9.0
    x[32, classes - 2] = 10.0
    t = torch.full((rows,), classes - 1, dtype=torch.int64, device="cuda")
    r = F.log_probs_forward(x, t, 3)
    small = math.exp(-20.0) * (classes - 2)
    lse = math.log(math.exp(8) + math.exp(9) + small)
    # 2^26 terms of equal size: chains of 2^18 a lane at most, each step's rounding half a unit: 2^18 * 2^-24 of that part of the sum, which is 1e-2 of all
    assert abs(float(r.lse[0]) - lse) < 1e-3 and abs(float(r.logp[0]) - (8 - lse)) < 1e-3
    assert r.top_index[0].tolist() == [12345, classes - 1, 0] and r.top_index[32].tolist() == [classes - 2, 12345, classes - 1]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_at_the_ends_of_the_range(dtype):
    """Logits whose product with log2(e) is no float32 any more; masks of the type's lowest value next to real logits."""
    low = torch.finfo(DTYPES[dtype]).min
    for classes in (70, 5000, 120000):
        x, t, g, h = make(6, classes, dtype, 30)
        x[0, 0], x[0, classes - 1] = 3.0e38, 2.9e38
        x[1] = low
        x[2, :classes - 3] = low        # real logits come last
        x[3, 1:] = -math.inf
        x[3, 0] = low                   # one class left, the lowest of all
        x[4] = 3.2e38
        x[4, 5] = low
        x[5, ::2] = low
        t[0], t[2], t[3], t[4] = 0, classes - 1, 0, 1
        h[0] = h[4] = 0  # (an entropy's gradient next to differences of 1e38: products with probabilities 0)
        check(x, t, 5, g, h)


@pytest.mark.parametrize("classes", [20011, 140001])
def test_best_classes_all_in_a_few_lanes(classes):
    """Periods of 2048 and of 512 classes with eight good ones at their start: the bound that the lanes' bests give lets thousands of candidates pass."""
    j = torch.arange(classes)
    g = torch.Generator().manual_seed(5)
    noise = torch.rand(4, classes, generator=g)
    x = torch.stack([noise[0] + 5 * (j // 8 % 256 < 8), noise[1] + 5 * (j // 8 % 256 == 3), noise[2] + 5 * (j // 4 % 128 < 2), noise[3] + 5 * (j % 2048 < 300)]).cuda()
    t = torch.zeros(4, dtype=torch.int64).cuda()
    for dtype in DTYPES.values():
        for top in (5, 32):
            check(x.to(dtype), t, top)
            check(x[:1].to(dtype), t[:1], top)


@pytest.mark.parametrize("classes", [9001, 131072])
def test_best_classes_of_rows_that_are_mostly_alike(classes):
    """More classes pass the first bound than are kept: equal ones, masked ones, NaN, rising and falling rows."""
    j = torch.arange(classes, dtype=torch.float32)
    x, t, _, _ = make(9, classes, "f32", seed=8)
    x[0] = 1.5
    x[1] = -math.inf
    x[1, classes - 7:] = 0.25
    x[2, 1::3] = math.nan
    x[3] = math.nan
    x[4, classes - 20:] = math.nan
    x[5, ::2] = math.inf
    x[6] = (j / classes).cuda()
    x[7] = (-j / classes).cuda()
    x[8] = (j // 8 % 512 < 12).cuda() * j.cuda() / classes
    for dtype in DTYPES.values():
        for top in (1, 7, 32):
            check(x.to(dtype), t, top)
            check(x[2:3].to(dtype), t[2:3], top)
