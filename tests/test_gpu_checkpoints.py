"""The operators together, as a training step uses them, what autograd keeps in 8 bits, and calls on other streams and in graphs."""
import gc
import threading

import pytest
import torch
from torch import nn

import rows_reference as ref
from paper_1804_08378_amd import functional as F
from paper_1804_08378_amd.frontend import optimize

pytestmark = pytest.mark.gpu


class Block(nn.Module):
    """A residual block: total = x + delta, normalised, through a gated layer; returns the block's share and the total."""

    def __init__(self, width, inner, checkpoint):
        super().__init__()
        self.norm = F.LayerNorm(width, checkpoint=checkpoint)
        self.up, self.down = nn.Linear(width, 2 * inner, bias=False), nn.Linear(inner, width, bias=False)
        self.checkpoint = checkpoint

    def forward(self, x, delta):
        y, total = self.norm(x, delta)
        x, gate = self.up(y).chunk(2, -1)
        return self.down(F.activate(x, "silu", gate, self.checkpoint)), total


class Exact(torch.autograd.Function):
    """A value whose gradient's formulas are taken at another one."""

    @staticmethod
    def forward(ctx, x, at, f):
        ctx.save_for_backward(at)
        ctx.f = f
        return f(x)

    @staticmethod
    def backward(ctx, g):
        at = ctx.saved_tensors[0].requires_grad_(True)
        with torch.enable_grad():
            return torch.autograd.grad(ctx.f(at), at, g)[0], None, None


def plain_blocks(blocks, x, delta, checkpoint):
    """The same in 64 bits on the CPU; with checkpoints the activations' gradients at the float32 operands' values in 8 bits."""
    params = []
    for blk in blocks:
        w, b, up, down = (p.detach().cpu().double().requires_grad_(True) for p in (blk.norm.weight, blk.norm.bias, blk.up.weight, blk.down.weight))
        params += [w, b, up, down]
        total = x + delta
        mean = total.mean(-1, keepdim=True)
        rstd = 1 / ((total - mean) ** 2).mean(-1, keepdim=True).add(1e-5).sqrt()
        y = (total - mean) * rstd * w + b
        if checkpoint:
            y = AtHeld.apply(total, w, b, mean.detach(), rstd.detach())
        h = y @ up.t()
        n = h.shape[-1] // 2
        if checkpoint:
            at = torch.cat([ref.held(t.float()) for t in h.detach().chunk(2, -1)], -1)  # (the blocks of either half are its own)
            act = Exact.apply(h, at, lambda v: v[..., :n] * torch.sigmoid(v[..., :n]) * v[..., n:])
        else:
            act = h[..., :n] * torch.sigmoid(h[..., :n]) * h[..., n:]
        x, delta = total, act @ down.t()
    return delta, x, params


class AtHeld(torch.autograd.Function):
    @staticmethod
    def forward(ctx, total, w, b, mean, rstd):
        ctx.save_for_backward((ref.held(total.float()) - mean) * rstd, w, rstd)
        return (total - mean) * rstd * w + b

    @staticmethod
    def backward(ctx, g):
        xh, w, rstd = ctx.saved_tensors
        u = g * w
        dx = rstd * (u - u.mean(-1, keepdim=True) - xh * (u * xh).mean(-1, keepdim=True))
        return dx, (g * xh).sum((0, 1)), g.sum((0, 1)), None, None


@pytest.mark.parametrize("checkpoint", [False, True])
def test_a_run_of_blocks(checkpoint):
    """Two blocks in float32 against 64 bits: 1e-5 of a gradient's norm for the roundings of some ten operations over sums of 64 to 200 terms (1e-7
    each).  With checkpoints an element of the second block's operands that is next to a border between two codes, within a rounding of 1e-6 of its
    size, may fall to either: a share of 1e-4 of the elements at most, each a step (2^-6 of its size) off, 1e-2 * 2^-6 in norm: 3e-4."""
    torch.manual_seed(2)
    blocks = [Block(64, 100, checkpoint).cuda() for _ in range(2)]
    x, delta, g1, g2 = (torch.randn(3, 50, 64, device="cuda") for _ in range(4))
    x.requires_grad_(True)
    t, d = x, delta
    for blk in blocks:
        d, t = blk(t, d)
    params = [p for blk in blocks for p in (blk.norm.weight, blk.norm.bias, blk.up.weight, blk.down.weight)]
    grads = torch.autograd.grad([d, t], [x, *params], [g1, g2])
    y = x.detach().cpu().double().requires_grad_(True)
    rd, rt, rparams = plain_blocks(blocks, y, delta.cpu().double(), checkpoint)
    want = torch.autograd.grad([rd, rt], [y, *rparams], [g1.cpu().double(), g2.cpu().double()])
    assert float((d.detach().cpu().double() - rd.detach()).norm()) <= 1e-5 * float(rd.detach().norm())
    for a, b in zip(grads, want):
        assert float((a.cpu().double() - b).norm()) <= (3e-4 if checkpoint else 1e-5) * float(b.norm())


def test_checkpoints_use_less_memory():
    """Bytes that the graph of a gated layer keeps: two operands of 2 bytes an element, in 8 bits 33 bytes for 32 of them each."""
    x, gate = (torch.randn(512, 4096, device="cuda", dtype=torch.bfloat16, requires_grad=True) for _ in range(2))
    sizes = []
    for checkpoint in (False, True):
        a, b = x * 1.0, gate * 1.0  # (made here: freed unless the graph keeps them)
        y = F.activate(a, "silu", b, checkpoint)
        del a, b
        torch.cuda.synchronize()
        sizes.append(torch.cuda.memory_allocated())
        del y
    assert sizes[0] - sizes[1] >= 0.95 * (2 * 512 * 4096 * (2 - 33 / 32))


# ------------------------------------------------------------------------------------------------ what autograd keeps
def values_of(t):
    """What the block's tensors come back as."""
    p = F.pack8(t.reshape(1, -1))
    return F.unpack8(p, t.dtype).view(t.shape)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_convolution_keeps_8_bits(dtype):
    torch.manual_seed(3)
    conv = nn.Conv2d(16, 24, 3, padding=1).cuda().to(dtype)
    for fmt in (torch.contiguous_format, torch.channels_last):
        x = torch.randn(4, 16, 20, 20, device="cuda", dtype=dtype).contiguous(memory_format=fmt).requires_grad_(True)
        with F.checkpoints_in_8_bits(conv):
            y = conv(x)
        assert torch.equal(y, conv(x)) or float((y - conv(x)).detach().norm()) <= 1e-2 * float(y.detach().norm())
        gx, gw = torch.autograd.grad(y, [x, conv.weight], torch.ones_like(y))
        flat = x.detach().permute(0, 2, 3, 1) if fmt == torch.channels_last else x.detach()
        at = values_of(flat)
        at = (at.permute(0, 3, 1, 2) if fmt == torch.channels_last else at).requires_grad_(True)
        z = nn.functional.conv2d(at, conv.weight, conv.bias, padding=1)
        want = torch.autograd.grad(z, [at, conv.weight], torch.ones_like(z))
        # the same products, whose sums a library may take in another order: roundings of the type, 4 units in norm
        tol = 4 * torch.finfo(dtype).eps
        assert float((gw - want[1]).norm()) <= tol * float(want[1].norm()) and float((gx - want[0]).norm()) <= tol * float(want[0].norm())
        full = torch.autograd.grad(conv(x), conv.weight, torch.ones_like(y))[0]
        assert float((gw - full).norm()) <= 0.02 * float(full.norm()) and not torch.equal(gw, full)


def test_what_is_held():
    m = nn.Linear(64, 64).cuda()
    seen = []
    pack = F.pack8
    x = torch.randn(512, 64, device="cuda", requires_grad=True)
    try:
        F.pack8 = lambda t: seen.append(tuple(t.shape)) or pack(t)
        with F.checkpoints_in_8_bits(m, least=4096):
            y = m(x)                                    # x is held, the weight stays
            z = (y * y.detach()[:8].repeat(64, 1)).sum()  # the other factor: 512 x 64
            (x[:4] * x[:4]).sum()                       # too small
            torch.where(x > 0, x, 0.0)                  # a mask: no number
            (x.sum(1, keepdim=True) * x[:, :1]).exp()   # one number a row
            (x.double() * x.double()).sum()             # another type
            x.t()[::2].exp()                            # exp keeps its result, dense
            w = torch.randn(64, 64, device="cpu", requires_grad=True)
            w * w                                       # not on the GPU
    finally:
        F.pack8 = pack
    assert seen and all(s[0] * s[1] >= 4096 for s in seen) and (1, 512 * 64) in seen and (1, 64 * 64) not in seen
    z.backward()
    assert x.grad is not None and m.weight.grad is not None
    # nothing is held outside of the block
    n = len(seen)
    m(x)
    assert len(seen) == n


def test_views_and_parameters_stay_as_they_are():
    w = nn.Parameter(torch.randn(200, 300, device="cuda"))
    x = torch.randn(100, 200, device="cuda", requires_grad=True)
    with F.checkpoints_in_8_bits([w], least=1):
        y = (x @ w) @ w.t() @ w  # a view of a parameter is its memory
    (gx,) = torch.autograd.grad(y.sum(), x)
    with torch.no_grad():
        want = torch.ones(100, 300, device="cuda") @ w.t() @ w @ w.t()
    assert float((gx - want).norm()) <= 1e-5 * float(want.norm())
    big = torch.randn(64, 300, device="cuda", requires_grad=True)
    with F.checkpoints_in_8_bits([], least=1):
        y = big[:, :200].sin()  # its operand is a view with gaps: kept as it is
    assert torch.allclose(torch.autograd.grad(y.sum(), big)[0][:, :200], big.detach()[:, :200].cos(), atol=1e-6)


def test_refuses_autocast():
    m = nn.Linear(64, 64).cuda()
    x = torch.randn(512, 64, device="cuda", requires_grad=True)
    with torch.autocast("cuda", torch.bfloat16), pytest.raises(RuntimeError, match="autocast"):
        with F.checkpoints_in_8_bits(m, least=1):
            m(x)
    with F.checkpoints_in_8_bits(m, least=1), pytest.raises(RuntimeError, match="autocast"), torch.autocast("cuda", torch.bfloat16):
        m(x)
    with torch.autocast("cuda", enabled=False), F.checkpoints_in_8_bits(m, least=1):
        m(x).sum().backward()
    assert m.weight.grad is not None


@pytest.mark.parametrize("native", [True, False])
def test_stacks_and_the_operators_in_the_block(native, monkeypatch):
    """A fine-tuned model of stacks and convolutions, and every function here: finite gradients near those without the block.  An element is off by half
    a step, a step a 63rd of its block's largest element at most, which is under 4 deviations: 3 % of a deviation, 2 % (of uniformly spread errors,
    a root of 3 less) of a gradient's norm for every product with a held operand, of which a gradient meets up to six.  A ReLU's slope is another one for
    the elements that are within that of 0: of a density of 0.4 at most in a band of two times 3 %, half of which fall to the other side, 1.3 %, a share
    of sqrt(0.013) = 11 % of a norm.  Together under 25 %."""
    if not native:
        monkeypatch.setattr(F, "_native", False)
    torch.manual_seed(4)
    model = nn.Sequential(nn.Conv2d(8, 32, 3, padding=1), nn.BatchNorm2d(32), nn.ReLU(), nn.AvgPool2d(2), nn.Conv2d(32, 32, 3, padding=1)).cuda().eval()
    for p in model[1].parameters():
        p.requires_grad_(False)
    fast = optimize(model)
    norm, rows = F.GroupNormAct(4, 32, "silu").cuda(), F.LayerNorm(32).cuda()
    x = torch.randn(8, 8, 32, 32, device="cuda")
    t = torch.arange(8, device="cuda")

    def features():
        y = norm(fast(x).contiguous(memory_format=torch.channels_last))
        y = rows(y.permute(0, 2, 3, 1))
        return F.activate(y, "gelu", y).reshape(8, -1)

    def loss(y):
        return -F.log_probs(y, t).logp.mean()

    params = [*model[0].parameters(), *fast[-1].parameters(), *norm.parameters(), *rows.parameters()]
    full = torch.autograd.grad(loss(features()), params)
    with F.checkpoints_in_8_bits(nn.ModuleList([fast, norm, rows]), least=64):
        y = features()
    held = torch.autograd.grad(loss(y), params)
    for a, b in zip(held, full):
        assert a.isfinite().all() and 0 < float((a - b).norm()) <= 0.25 * float(b.norm())


# ------------------------------------------------------------------------------------------------ streams, graphs, threads
def operands(rows=300, n=515, dtype=torch.bfloat16, seed=5):
    g = torch.Generator().manual_seed(seed)
    x, a, dy, dt = (torch.randn(rows, n, generator=g).to(dtype).cuda() for _ in range(4))
    return x, a, dy, dt, torch.rand(n, generator=g).cuda(), torch.randn(n, generator=g).cuda()


def everything(x, a, dy, dt, w, b):
    r = F.layer_norm_forward(x, w, b, a, checkpoint=True)
    s = F.activate_forward(r.y, "silu", r.total, checkpoint=True)
    return [r.y, r.total, r.stats, *r.kept, s.y, *s.x, *s.gate, *F.activate_backward(s.x, dy, "silu", s.gate), *F.layer_norm_backward(r.kept, r.stats, dy, w, b, dt),
            *F.layer_norm_backward(r.total, r.stats, dy, w, b, dt), F.unpack8(F.pack8(x), x.dtype)]


def test_another_stream():
    ops = operands()
    want = everything(*ops)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        copies = [t.clone() for t in ops]  # (made on that stream: a call on another one would not wait for them)
        for _ in range(3):
            copies = [t + 0 for t in copies]
        got = everything(*copies)
    stream.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_two_streams_at_once():
    sets = [operands(seed=6), operands(2000, 515, seed=7)]
    want = [everything(*ops) for ops in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(5):
        for i, (s, ops) in enumerate(zip(streams, sets)):
            with torch.cuda.stream(s):
                got[i].append(everything(*ops))
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for i in range(2) for run in got[i] for p, q in zip(want[i], run))


def test_threads():
    ops = operands()
    want = everything(*ops)
    torch.cuda.synchronize()
    wrong = []

    def work():
        for _ in range(20):
            got = everything(*ops)
            torch.cuda.synchronize()
            if not all(torch.equal(p, q) for p, q in zip(want, got)):
                wrong.append(1)

    threads = [threading.Thread(target=work) for _ in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not wrong


@pytest.mark.parametrize("rows,n", [(300, 515), (1, 4096), (3000, 64), (20, 20011)])
def test_captured_and_replayed(rows, n):
    """Two graphs with workspaces of their own, replayed in turn with eager work between them."""
    ops = operands(rows, n)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        everything(*ops)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        static = [t.clone() for t in ops]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = everything(*static)
        graphs.append((graph, static, out))
    for i in range(4):
        fresh = operands(rows, n, seed=20 + i)
        want = everything(*fresh)
        for graph, static, out in graphs:
            for s, t in zip(static, fresh):
                s.copy_(t)
            graph.replay()
        torch.cuda.synchronize()
        again = everything(*fresh)
        for _, _, out in graphs:
            assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(want, out, again)), i


def test_a_captured_training_step():
    """Forward and backward through autograd in one graph, with leaves of its own that no eager graph is alive for."""
    x, a, dy, dt, w, b = operands(64, 320, torch.float32)
    leaves = [t.clone().requires_grad_(True) for t in (x, a, w, b)]

    def step():
        y, total = F.layer_norm(leaves[0], leaves[2], leaves[3], leaves[1], checkpoint=True)
        z = F.activate(y, "gelu", total, checkpoint=True)
        return torch.autograd.grad(z, leaves, dy)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    gc.collect()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        with torch.no_grad():
            leaves[0].copy_(x * (i + 1))
            leaves[1].copy_(a + i)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        others = [t.detach().clone().requires_grad_(True) for t in leaves]
        y, total = F.layer_norm(others[0], others[2], others[3], others[1], checkpoint=True)
        want = torch.autograd.grad(F.activate(y, "gelu", total, checkpoint=True), others, dy)
        assert all(torch.equal(p, q) for p, q in zip(got, want)), i


def test_in_place_changes_are_seen():
    """Autograd keeps x itself without a checkpoint, and a copy with one."""
    x, a, dy, dt, w, b = operands(8, 100, torch.float32)
    for checkpoint in (False, True):
        v = (x * 1.0).requires_grad_(True)
        u = v * 1.0
        y = F.layer_norm(u, w, b, checkpoint=checkpoint)
        u.add_(1.0)
        if checkpoint:
            r = F.layer_norm_forward(x, w, b, checkpoint=True)
            assert torch.equal(torch.autograd.grad(y, v, dy)[0], F.layer_norm_backward(r.kept, r.stats, dy, w, b)[0])
        else:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                torch.autograd.grad(y, v, dy)
    v = x.clone().requires_grad_(True)
    y, total = F.layer_norm(v, w, b, a)
    total.add_(1.0)  # (the kept sum)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(y, v, dy)


def test_gradients_of_gradients_are_refused():
    x, a, dy, dt, w, b = operands(4, 50, torch.float32)
    v = x.clone().requires_grad_(True)
    for y in (F.layer_norm(v, w, b), F.activate(v, "silu", a)):
        (g,) = torch.autograd.grad(y, v, dy.requires_grad_(True), create_graph=True)
        with pytest.raises(RuntimeError):
            g.sum().backward()
