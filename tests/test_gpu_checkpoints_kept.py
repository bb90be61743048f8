"""What `checkpoints_in_8_bits` holds in 8 bits on the GPU, and what stays as it is."""
import pytest
import torch
from torch import nn

import rows_reference as ref
from paper_1804_08378_amd import functional as F
from paper_1804_08378_amd.frontend import optimize

pytestmark = pytest.mark.gpu


@pytest.fixture
def held(monkeypatch):
    """How many elements each of the tensors has that are held."""
    seen, pack = [], F.pack8
    monkeypatch.setattr(F, "pack8", lambda t: seen.append(t.numel()) or pack(t))
    return seen


# ------------------------------------------------------------------------------------------------ statistics
def test_attention_keeps_its_log_sums(held):
    q, k, v = (torch.randn(2, 8, 1024, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True) for _ in range(3))
    with F.checkpoints_in_8_bits([]):
        y = nn.functional.scaled_dot_product_attention(q, k, v)
    assert held and 2 * 8 * 1024 not in held and all(n >= q.numel() for n in held)
    assert all(g.isfinite().all() for g in torch.autograd.grad(y.sum(), (q, k, v)))


def test_a_group_normalisations_gradients_are_those_at_the_held_values(held):
    """torch's group normalisation of groups of 8 numbers, of another scale each, float32, in the block, against the formula in 64 bits at the images' values
    in 8 bits and exact statistics.  torch computes sums of dy * x and of dy, and from them their difference mean * sum dy - sum dy * x: a dozen
    roundings of 2^-24 of terms up to 1 + (mean / deviation)^2, under 9 but for a few of the groups: 1e-5 of the gradient's norm.  (Means and deviations in
    8 bits, up to 0.8 % off each, miss it by a percent.)  The weight's gradient is not compared: torch 2.10's own, for more than 128 images, is off by as much
    as it is long on this GPU, without the block too."""
    torch.manual_seed(1)
    scale = torch.exp2(torch.rand(512, 64, 1, 1, device="cuda").mul(6).sub(3))
    x = (torch.randn(512, 64, 1, 4, device="cuda") * scale).requires_grad_(True)
    norm = nn.GroupNorm(32, 64).cuda()
    with torch.no_grad():
        norm.weight.uniform_(0.5, 1.5)
    with F.checkpoints_in_8_bits(norm):
        y = norm(x)
    assert held == [x.numel()]
    dy = torch.randn_like(y)
    (gx,) = torch.autograd.grad(y, x, dy)
    exact, g, w = (t.detach().cpu().double() for t in (x, dy, norm.weight))
    grouped = lambda t: t.reshape(512, 32, 8)
    mean = grouped(exact).mean(-1, keepdim=True)
    rstd = 1 / ((grouped(exact) - mean) ** 2).mean(-1, keepdim=True).add(norm.eps).sqrt()
    xh = (grouped(ref.held(x.detach().reshape(1, -1)).view(x.shape)) - mean) * rstd
    u = grouped(g * w.view(1, 64, 1, 1))
    want = rstd * (u - u.mean(-1, keepdim=True) - xh * (u * xh).mean(-1, keepdim=True))
    assert float((grouped(gx.cpu().double()) - want).norm()) <= 1e-5 * float(want.norm())


def test_a_log_sum_stays_as_it_is(held):
    """Its gradient is exp(x - log sum): of a log sum of 50 half a step would be a factor of e^0.25.  Of x at values half a step (2^-7 of 50 at most) off it is."""
    x = (torch.randn(128, 128, 40, device="cuda") + 50).requires_grad_(True)
    with F.checkpoints_in_8_bits([], least=64):
        y = x.logsumexp(-1)
    assert held == [x.numel()]
    (g,) = torch.autograd.grad(y.sum(), x)
    at = ref.held(x.detach().reshape(1, -1)).view(x.shape)
    want = (at - x.detach().cpu().double().logsumexp(-1, keepdim=True)).exp()
    assert float((g.cpu().double() - want).abs().max()) <= 2e-5 * float(want.max())  # (arguments of up to 55 and results: roundings of 2^-24 of 55, 8e-6 in all)


def test_norms_of_parameters_stay_as_they_are(held):
    w = nn.Parameter(torch.randn(64, 512, 8, device="cuda"))
    with F.checkpoints_in_8_bits([w]):
        y = w.norm(dim=-1)
    assert not held
    torch.testing.assert_close(torch.autograd.grad(y.sum(), w)[0], w.detach() / y.detach()[..., None])


def test_what_has_no_gradient_stays_as_it_is(held):
    x, constant = torch.randn(256, 256, device="cuda", requires_grad=True), torch.randn(256, 256, device="cuda")
    with F.checkpoints_in_8_bits([]):
        y = x * constant
    assert not held and torch.equal(torch.autograd.grad(y.sum(), x)[0], constant)
    with F.checkpoints_in_8_bits([]):
        y = x * (x * 1.0)
    assert held == [x.numel()] * 2


def test_the_operators_here_keep_their_operands_so(held):
    """The total of a layer normalisation, a second result, is an operand; statistics stay."""
    x, a = (torch.randn(1024, 64, device="cuda", requires_grad=True) for _ in range(2))
    with F.checkpoints_in_8_bits([], least=64):
        y, total = F.layer_norm(x, addend=a)
        z = F.activate(y, "silu", total)
    assert held == [x.numel()] * 3
    n = F.GroupNormAct(4, 32, "silu").cuda()
    m = torch.randn(64, 32, 8, 8, device="cuda", requires_grad=True).contiguous(memory_format=torch.channels_last)
    with F.checkpoints_in_8_bits(n, least=64):
        v = n(m)
    assert held == [x.numel()] * 3 + [m.numel()]
    assert all(g.isfinite().all() for g in torch.autograd.grad(z.sum() + v.sum(), (x, a, m)))


def test_stacks_and_batch_normalisations(held):
    """A stack's operand, the result of a convolution, is held; a batch normalisation in training mode too keeps its operand so, and may run twice."""
    model = nn.Sequential(nn.Conv2d(8, 32, 3, padding=1), nn.BatchNorm2d(32), nn.ReLU(), nn.AvgPool2d(2)).cuda().eval()
    for p in model[1].parameters():
        p.requires_grad_(False)
    fast = optimize(model)
    x = torch.randn(8, 8, 32, 32, device="cuda")
    with F.checkpoints_in_8_bits(fast, least=64):
        y = fast(x)
    assert held == [8 * 32 * 32 * 32]
    assert all(g.isfinite().all() for g in torch.autograd.grad(y.sum(), [*model[0].parameters()]))
    held.clear()
    m = nn.Sequential(nn.Conv2d(8, 32, 1), nn.BatchNorm2d(32)).cuda()
    with F.checkpoints_in_8_bits(m, least=64):
        y = m(x) + m(x * 2.0)
    assert held == [8 * 32 * 32 * 32] * 2
    assert all(g.isfinite().all() for g in torch.autograd.grad(y.sum(), [*m.parameters()]))


# ------------------------------------------------------------------------------------------------ parameters
def test_a_model_that_moves_behind_the_blocks_making(held):
    """Its parameters and buffers are those that it has where the block begins."""
    m = nn.Linear(128, 96)
    m.register_buffer("table", torch.randn(128, 128, requires_grad=True))
    block = F.checkpoints_in_8_bits(m, least=64)
    m.cuda()
    x = torch.randn(64, 128, device="cuda", requires_grad=True)
    for _ in range(2):
        with block:
            y = m(x @ m.table)
        (gx,) = torch.autograd.grad(y.sum(), x)
        want = (m.weight.sum(0) @ m.table.t()).detach().expand_as(gx)
        assert float((gx - want).norm()) <= 1e-5 * float(want.norm())  # (sums of 224 terms; weights in 8 bits miss it by some 0.3 %)
        assert sorted(held) == [x.numel()] * 2  # the operands of both products
        held.clear()
        m.double().float()  # (a round trip: new memory)


def test_parameters_made_inside_the_block(held):
    m = nn.Sequential(nn.LazyLinear(96), nn.ReLU(), nn.Linear(96, 64)).cuda()
    x = torch.randn(64, 128, device="cuda", requires_grad=True)
    with F.checkpoints_in_8_bits(m, least=64):
        y = m(x)
    assert sorted(held) == [64 * 96, 64 * 96, 64 * 128]  # operands of the products and the ReLU's result
    (gx,) = torch.autograd.grad(y.sum(), x)
    assert gx.isfinite().all()


def test_sparse_tensors_stay_as_they_are(held):
    t = torch.sparse_coo_tensor(torch.arange(64, device="cuda").repeat(2, 1), torch.randn(64, device="cuda"), (4096, 4096)).requires_grad_(True)
    block = F.checkpoints_in_8_bits([], least=64)
    kept = block.pack_hook(t)
    assert not held and torch.equal(block.unpack_hook(kept)._values(), t.detach()._values())
