"""Group normalisation with a residual operand and an activation on the GPU, against its definition in 64 bits.

Tolerances.  With u = 2^-24: float32 sums here run over chains of at most a few hundred terms (pixels of a lane, then lanes, then chunks), so
a sum is off by less than 300 u = 2e-5 of the sum of its terms' magnitudes, a mean by 2e-5 deviations and 4 u of its own size (the last
roundings), results by that times the factors behind it.  16-bit results add half a unit in the last place, 2^-8 (bfloat16) or 2^-11
(binary16, and its smallest steps 2^-25) of the value.
"""
import math

import pytest
import torch

from paper_1804_08378_amd import brainslug as bs
from paper_1804_08378_amd import functional as F

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROUNDING = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a unit in the last place of 24, 8, 11 significant bits
SUMS = 2e-5

SHAPES = [  # n, c, h, w, groups
    (1, 16, 32, 32, 4),
    (2, 64, 8, 8, 32),
    (3, 60, 7, 5, 12),       # groups of five channels
    (2, 7, 5, 3, 7),         # one channel a group, odd
    (1, 1, 1, 1, 1),         # one cell
    (2, 6, 1, 1, 3),         # groups of two cells
    (1, 320, 9, 9, 1),       # one group
    (2, 2048, 3, 3, 32),
    (1, 771, 4, 5, 3),       # groups of 257 channels, odd
    (1, 8, 150, 130, 2),     # a long plane
    (40, 24, 3, 2, 4),       # many images
    (2, 128, 28, 28, 32),
    (1, 96, 61, 1, 32),      # groups of three channels, one column
]


def act(name, z):
    return {"identity": lambda v: v, "relu": lambda v: torch.where(v > 0, v, 0.0), "silu": lambda v: v * torch.sigmoid(v),
            "gelu": lambda v: 0.5 * v * torch.erfc(-v / math.sqrt(2))}[name](z)


def slope(name, z):
    s = torch.sigmoid(z)
    return {"identity": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(), "silu": lambda: s * (1 + z * (1 - s)),
            "gelu": lambda: 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)}[name]()


class Reference:
    """The definition in 64 bits, on the CPU, with what the tolerances need."""

    def __init__(self, x, groups, weight, bias, residual, name, eps):
        n, c, h, w = x.shape
        self.shape, self.groups, self.name = x.shape, groups, name
        cpu = lambda t: None if t is None else t.detach().cpu().double().contiguous()
        x, weight, bias, residual = cpu(x), cpu(weight), cpu(bias), cpu(residual)
        self.weight = torch.ones(c).double() if weight is None else weight
        bias = torch.zeros(c).double() if bias is None else bias
        v = x.reshape(n, groups, -1)
        mean = v.mean(2, keepdim=True)
        var = ((v - mean) ** 2).mean(2, keepdim=True)
        self.mean, self.rstd = mean, 1 / torch.sqrt(var + eps)
        self.xh = ((v - mean) * self.rstd).reshape(self.shape)
        self.z = self.xh * self.weight.view(1, c, 1, 1) + bias.view(1, c, 1, 1)
        if residual is not None:
            self.z = self.z + residual
        self.y = act(name, self.z)
        # how far xh may be off: the mean's error in deviations, the deviation's relative error
        off = SUMS + 4 * 2.0 ** -24 * (mean.abs() * self.rstd)
        self.xh_off = ((off + 2 * SUMS * self.xh.reshape(v.shape).abs())).reshape(self.shape)
        self.z_off = self.xh_off * self.weight.abs().view(1, c, 1, 1) + 4 * 2.0 ** -24 * (self.z.abs() + (residual.abs() if residual is not None else 0))

    def backward(self, dy):
        n, c, h, w = self.shape
        dy = dy.detach().cpu().double().contiguous()
        dz = dy * slope(self.name, self.z)
        dxh = (dz * self.weight.view(1, c, 1, 1)).reshape(n, self.groups, -1)
        xh = self.xh.reshape(dxh.shape)
        m1, m2 = dxh.mean(2, keepdim=True), (dxh * xh).mean(2, keepdim=True)
        dx = (self.rstd * (dxh - m1 - xh * m2)).reshape(self.shape)
        # every slope is at most 1.13 and changes by at most 0.8 a unit of z
        dz_off = dy.abs() * (self.z_off if self.name in ("silu", "gelu") else 0) + 8 * 2.0 ** -24 * dz.abs() + 2e-6 * dy.abs()
        dxh_off = (dz_off * self.weight.abs().view(1, c, 1, 1)).reshape(dxh.shape)
        mags = dxh.abs().mean(2, keepdim=True), (dxh * xh).abs().mean(2, keepdim=True)
        x_off = self.xh_off.reshape(dxh.shape)
        m1_off = dxh_off.mean(2, keepdim=True) + SUMS * mags[0]
        m2_off = (dxh_off * xh.abs() + dxh.abs() * x_off).mean(2, keepdim=True) + SUMS * mags[1]
        dx_off = (self.rstd * (dxh_off + m1_off + xh.abs() * m2_off + x_off * m2.abs() + 2 * SUMS * (dxh.abs() + m1.abs() + (xh * m2).abs()))).reshape(self.shape)
        dw_off = (dz_off * self.xh.abs() + dz.abs() * self.xh_off).sum((0, 2, 3)) + SUMS * (dz * self.xh).abs().sum((0, 2, 3))
        db_off = dz_off.sum((0, 2, 3)) + SUMS * dz.abs().sum((0, 2, 3))
        return (dx, dx_off), ((dz * self.xh).sum((0, 2, 3)), dw_off), (dz.sum((0, 2, 3)), db_off), (dz, dz_off)


def close(got, want, off, dtype, label):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, label
    bound = off + ROUNDING[dtype] * 1.01 * (want.abs() + off) + (2.0 ** -25 if dtype == "f16" else 1e-30)
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (label, int(bad.sum()), float(((got - want).abs() / bound).max()))


def tensors(shape, dtype, seed, residual, params="f32", mean=0.0):
    n, c, h, w, _ = shape
    g = torch.Generator().manual_seed(seed)
    dt = DTYPES[dtype]
    make = lambda scale=1.0, shift=0.0: (torch.randn(n, h, w, c, generator=g) * scale + shift).to(dt).cuda().permute(0, 3, 1, 2)
    pt = DTYPES[params]
    x = make(1.5, mean)
    return x, (torch.rand(c, generator=g) + 0.5).to(pt).cuda(), (torch.randn(c, generator=g) * 0.3).to(pt).cuda(), make() if residual else None, make()


def check(shape, dtype, name, residual, seed=0, eps=1e-5, affine=True, params="f32", mean=0.0, change=None):
    print(f"[group norm] {shape} {dtype} {name} residual={residual} params={params} mean={mean}", flush=True)
    x, weight, bias, res, dy = tensors(shape, dtype, seed, residual, params, mean)
    if not affine:
        weight = bias = None
    if change is not None:
        x, res, dy = change(x), change(res) if res is not None else None, change(dy)
    ref = Reference(x, shape[4], weight, bias, res, name, eps)
    if name == "relu":  # next to the kink either gradient is right: none is asked for there
        dy = torch.where(ref.z.abs().cuda() <= 2 * ref.z_off.cuda() + 1e-6, torch.zeros_like(dy), dy)
    args = (shape[4], weight, bias, res, name, eps)
    y, stats = F.group_norm_forward(x, *args)
    torch.cuda.synchronize()
    # |act(a) - act(b)| <= 1.13 |a - b|
    close(y, ref.y, 1.13 * ref.z_off + 2e-6 * ref.y.abs() + 1e-7, dtype, "y")
    rstd_off = (2 * SUMS + 4 * 2.0 ** -24) * ref.rstd
    close(stats[..., 0], ref.mean[..., 0], (SUMS / ref.rstd + 4 * 2.0 ** -24 * ref.mean.abs())[..., 0], "f32", "mean")
    close(stats[..., 1], ref.rstd[..., 0], rstd_off[..., 0], "f32", "rstd")
    got = F.group_norm_backward(x, stats, dy, *args)
    torch.cuda.synchronize()
    for g, (want, off), label in zip(got, ref.backward(dy), ("grad_x", "grad_weight", "grad_bias", "grad_residual")):
        if g is not None:
            close(g, want, off, params if label in ("grad_weight", "grad_bias") else dtype, label)
    assert (got[1] is None) == (weight is None) and (got[3] is None) == (res is None)
    again = F.group_norm_backward(x, stats, dy, *args)
    assert all(a is None or torch.equal(a, b) for a, b in zip(got, again)), "equal calls give equal bits"
    assert torch.equal(F.group_norm(x, *args), y)
    return x, y, got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_both_directions(shape, dtype):
    check(shape, dtype, "silu", True)
    check(shape, dtype, "identity", False, seed=1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", F.ACTIVATIONS)
@pytest.mark.parametrize("residual", [False, True])
def test_activations(name, residual, dtype):
    check((2, 48, 11, 9, 6), dtype, name, residual, seed=3)


def test_parameters_absent_and_in_the_storage_type():
    check((2, 48, 6, 5, 6), "f32", "gelu", True, affine=False)
    check((2, 48, 6, 5, 6), "bf16", "silu", True, params="bf16")
    check((2, 48, 6, 5, 6), "f16", "silu", False, params="f16")


@pytest.mark.parametrize("shape", [(2, 32, 40, 40, 8), (1, 512, 4, 4, 2), (3, 30, 33, 17, 5)])
def test_mean_far_from_zero(shape):
    """A mean of a thousand deviations: sums of squares would lose every digit of the variance."""
    check(shape, "f32", "identity", False, mean=1500.0)


def test_constant_groups_and_infinite_cells():
    x = torch.full((1, 8, 5, 5), 3.25, device="cuda").contiguous(memory_format=torch.channels_last)
    y, stats = F.group_norm_forward(x, 2, eps=1e-5)
    assert torch.equal(y, torch.zeros_like(y)) and torch.equal(stats[..., 0], torch.full((1, 2), 3.25, device="cuda"))
    x[0, 1, 2, 2] = math.inf  # in the first group: its cells have no mean, the other group is untouched
    y, _ = F.group_norm_forward(x, 2)
    assert torch.isnan(y[:, :4]).all() and torch.equal(y[:, 4:], torch.zeros_like(y[:, 4:]))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset,larger", [(0, 96), (8, 80), (1, 71), (3, 64)])
def test_channel_slices_are_read_and_written_in_place(offset, larger, dtype):
    c = 48

    def slice_of(t):
        big = torch.full((t.shape[0], larger, *t.shape[2:]), 7.0, dtype=t.dtype, device=t.device).contiguous(memory_format=torch.channels_last)
        big[:, offset:offset + c] = t
        return big[:, offset:offset + c]

    shape = (2, c, 9, 7, 12)
    x, y, got = check(shape, dtype, "silu", True, change=slice_of)
    dense, weight, bias, res, dy = tensors(shape, dtype, 0, True)
    out = torch.full((2, larger, 9, 7), 5.0, dtype=dense.dtype, device="cuda").contiguous(memory_format=torch.channels_last)
    F.group_norm(dense, 12, weight, bias, res, "silu", out=out[:, offset:offset + c])
    rest = torch.cat([out[:, :offset], out[:, offset + c:]], 1)
    assert torch.equal(rest, torch.full_like(rest, 5.0))
    close(out[:, offset:offset + c], y.double().cpu(), 1e-5 * y.double().cpu().abs() + 1e-6, dtype, "out")


def test_other_memory_orders_are_copied():
    x = torch.randn(2, 24, 6, 5, device="cuda")
    a = F.group_norm(x, 4)
    b = F.group_norm(x.contiguous(memory_format=torch.channels_last), 4)
    assert torch.equal(a, b) and a.is_contiguous(memory_format=torch.channels_last)
    wide = torch.randn(2, 24, 6, 10, device="cuda").contiguous(memory_format=torch.channels_last)[:, :, :, ::2]
    assert torch.equal(F.group_norm(wide, 4), F.group_norm(wide.contiguous(memory_format=torch.channels_last), 4))


def test_no_images():
    x = torch.empty(0, 8, 4, 4, device="cuda")
    m = F.GroupNormAct(2, 8).cuda()
    y = m(x.requires_grad_(True))
    y.sum().backward()
    assert y.shape == x.shape and torch.equal(m.weight.grad, torch.zeros(8, device="cuda"))


def test_autograd_and_module():
    """The module's gradients are those of the passes; operands that need none get none."""
    x, weight, bias, res, dy = tensors((2, 48, 7, 6, 6), "f32", 5, True)
    m = F.GroupNormAct(6, 48, "silu").cuda()
    with torch.no_grad():
        m.weight.copy_(weight)
        m.bias.copy_(bias)
    x.requires_grad_(True)
    res.requires_grad_(True)
    y = m(x, res)
    y.backward(dy)
    y2, stats = F.group_norm_forward(x, 6, weight, bias, res, "silu")
    gx, gw, gb, gr = F.group_norm_backward(x, stats, dy, 6, weight, bias, res, "silu")
    for a, b in ((y, y2), (x.grad, gx), (m.weight.grad, gw), (m.bias.grad, gb), (res.grad, gr)):
        assert torch.equal(a.detach(), b.detach())
    frozen = F.group_norm(x.detach(), 6, m.weight, None, None, "relu")
    frozen.sum().backward()
    with torch.no_grad():
        assert m(x, res).requires_grad is False
    plain = torch.nn.GroupNorm(6, 48).cuda()
    plain.load_state_dict(m.state_dict())


@pytest.mark.parametrize("name", F.ACTIVATIONS)
def test_gradients_against_differences(name):
    """Central differences of the forward pass along random directions.  With steps of 2^-7 the difference's own error is under 2e-4 of the
    direction's third-order term (of size ~ 10), the roundings of the sum of 600 results of size 1 add 600 * 2^-24 / 2^-7 = 5e-3."""
    shape = (2, 12, 5, 5, 3)
    x, weight, bias, res, dy = tensors(shape, "f32", 11, True)
    ref = Reference(x, 3, weight, bias, res, name, 1e-5)
    step = 2.0 ** -7
    g = torch.Generator().manual_seed(2)
    if name == "relu":  # away from the kink, further than the steps move z
        dy = torch.where(ref.z.abs().cuda() < 0.2, torch.zeros_like(dy), dy)
    _, stats = F.group_norm_forward(x, 3, weight, bias, res, name)
    grads = F.group_norm_backward(x, stats, dy, 3, weight, bias, res, name)
    operands = [x, weight, bias, res]
    for i, grad in enumerate(grads):
        v = torch.randn(grad.shape, generator=g).cuda()
        v = v / v.abs().max()
        value = []
        for sign in (1, -1):
            moved = list(operands)
            moved[i] = moved[i] + sign * step * v
            y = F.group_norm(moved[0], 3, moved[1], moved[2], moved[3], name)
            value.append(float((y.double() * dy.double()).sum()))
        slope_seen = (value[0] - value[1]) / (2 * step)
        slope_told = float((grad.double() * v.double()).sum())
        assert abs(slope_seen - slope_told) <= 1e-2 + 5e-3 * abs(slope_told), (name, i, slope_seen, slope_told)


def test_other_streams():
    x, weight, bias, res, dy = tensors((4, 64, 20, 20, 8), "bf16", 0, True)
    want, stats = F.group_norm_forward(x, 8, weight, bias, res, "silu")
    grads = F.group_norm_backward(x, stats, dy, 8, weight, bias, res, "silu")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            y, st = F.group_norm_forward(x, 8, weight, bias, res, "silu")
            got.append((y, F.group_norm_backward(x, st, dy, 8, weight, bias, res, "silu")))
    torch.cuda.synchronize()
    for y, gs in got:
        assert torch.equal(y, want) and all(torch.equal(a, b) for a, b in zip(gs, grads))


def test_an_image_of_more_than_two_to_the_31_bytes_and_a_tensor_of_more_elements():
    """Offsets beyond 32 bits: 3 images of 0.8 G elements; each image's groups are those of a small image repeated."""
    n, c, p = 3, 64, 12_500_000
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GiB")
    tile = torch.randn(1, 50, 50, c, device="cuda").to(torch.bfloat16)
    x = torch.empty(n, c, 2500, p // 2500, dtype=torch.bfloat16, device="cuda", memory_format=torch.channels_last)
    flat = x.permute(0, 2, 3, 1)
    for i in range(n):
        flat[i].view(-1, 50 * 50, c).copy_((tile.view(1, 2500, c).float() * (i + 1) + i).to(torch.bfloat16).expand(p // 2500, -1, -1))
    y, stats = F.group_norm_forward(x, 8, activation="silu")
    for i in range(n):
        small = flat[i].reshape(-1, c)[:2500].view(1, 50, 50, c).permute(0, 3, 1, 2)
        ref = Reference(small, 8, None, None, None, "silu", 1e-5)
        close(stats[i, :, 0], ref.mean[0, :, 0], (1e-4 / ref.rstd)[0, :, 0], "f32", "mean")  # (longer chains: 5000 terms a lane)
        for at in (0, p - 2500):
            got = y.permute(0, 2, 3, 1)[i].reshape(-1, c)[at:at + 2500].view(1, 50, 50, c).permute(0, 3, 1, 2)
            close(got, ref.y, 5 * ref.z_off + 1e-6, "bf16", "y")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(2, 64, 40, 40, 8), (1, 64, 60, 50, 32), (3, 48, 21, 20, 4), (2, 30, 30, 30, 6), (1, 256, 33, 31, 2)])
def test_work_groups_that_do_not_wait(shape, dtype):
    """Images of several chunks whose work-groups look for no other's sums (wait_polls = -1) compute them all themselves: the same bits."""
    x, weight, bias, res, dy = tensors(shape, dtype, 4, True)
    n, c, h, w, groups = shape
    want, stats = F.group_norm_forward(x, groups, weight, bias, res, "silu")
    grads = F.group_norm_backward(x, stats, dy, groups, weight, bias, res, "silu")
    for residual in (res, None):
        if residual is None:
            want, stats = F.group_norm_forward(x, groups, weight, bias, None, "silu")
            grads = F.group_norm_backward(x, stats, dy, groups, weight, bias, None, "silu")
        d = F._norm_operands(x, groups, weight, bias, residual, "silu", 1e-5, dy)[0]
        d.wait_polls = -1
        y, st, gx, gr = torch.empty_like(want), torch.empty_like(stats), torch.empty_like(x), torch.empty_like(x)
        gw, gb = torch.empty_like(weight), torch.empty_like(bias)
        stream = torch.cuda.current_stream().cuda_stream
        for backward in (False, True):
            size = bs.bs_group_norm_workspace_bytes(d, backward)
            ws = torch.full((size,), 255 if backward else 0, dtype=torch.uint8, device="cuda")  # (what it holds does not matter)
            r = residual.data_ptr() if residual is not None else 0
            if backward:
                bs.bs_group_norm_backward(d, x.data_ptr(), r, weight.data_ptr(), bias.data_ptr(), st.data_ptr(), dy.data_ptr(), gx.data_ptr(),
                                          gr.data_ptr(), gw.data_ptr(), gb.data_ptr(), ws.data_ptr(), size, stream)
            else:
                bs.bs_group_norm(d, x.data_ptr(), r, weight.data_ptr(), bias.data_ptr(), y.data_ptr(), st.data_ptr(), ws.data_ptr(), size, stream)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(st, stats) and torch.equal(gx, grads[0]) and torch.equal(gw, grads[1]) and torch.equal(gb, grads[2])
        if residual is not None:
            assert torch.equal(gr, grads[3])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(3, 256, 56, 56, 32), (2, 64, 112, 112, 32), (1, 96, 100, 75, 32), (1, 8, 90, 130, 8), (1, 64, 182, 181, 8), (2, 36, 50, 51, 4),
                                   (1, 1024, 20, 19, 1), (7, 512, 14, 14, 32), (1, 32, 300, 280, 4)])
def test_images_of_many_chunks(shape, dtype):
    check(shape, dtype, "silu", True, seed=6)
    check(shape, dtype, "gelu", False, seed=7)


def test_launches_one_after_the_other_share_a_workspace():
    """The second call finds the first one's words in the workspace and must not take them for its own."""
    shape, groups = (2, 64, 60, 60), 8
    xs = [torch.randn(shape, device="cuda").contiguous(memory_format=torch.channels_last) * (i + 1) for i in range(6)]
    want = [F.group_norm(x, groups) for x in xs]
    d = F._norm_operands(xs[0], groups, None, None, None, "identity", 1e-5)[0]
    size = bs.bs_group_norm_workspace_bytes(d, False)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    ys = [torch.empty_like(x) for x in xs]
    for x, y in zip(xs, ys):
        bs.bs_group_norm(d, x.data_ptr(), 0, 0, 0, y.data_ptr(), 0, ws.data_ptr(), size, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ys, want))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("polls", [0, -1])
def test_exchange_memory_is_zero_again(polls, dtype):
    """Calls through exchange memory, of several shapes one after the other, with and without waiting: the bits of calls through the workspace,
    and nothing is left in the memory."""
    memory = torch.zeros(bs.BS_GROUP_NORM_EXCHANGE_BYTES // 8, dtype=torch.int64, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    for i, shape in enumerate([(2, 64, 60, 60, 32), (5, 256, 56, 56, 8), (1, 48, 100, 90, 4), (3, 64, 112, 112, 32), (2, 64, 60, 60, 32)]):
        x, weight, bias, res, dy = tensors(shape, dtype, i, True)
        d = F._norm_operands(x, shape[4], weight, bias, res, "silu", 1e-5, dy)[0]
        results = []
        for exchange in (0, memory.data_ptr()):
            d.exchange, d.exchange_bytes, d.wait_polls = exchange, 8 * memory.numel() if exchange else 0, polls if exchange else 0
            y, gx, gr = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
            st, gw, gb = torch.empty(shape[0], shape[4], 2, device="cuda"), torch.empty_like(weight), torch.empty_like(bias)
            size = max(bs.bs_group_norm_workspace_bytes(d, b) for b in (False, True))
            ws = torch.empty(size, dtype=torch.uint8, device="cuda")
            bs.bs_group_norm(d, x.data_ptr(), res.data_ptr(), weight.data_ptr(), bias.data_ptr(), y.data_ptr(), st.data_ptr(), ws.data_ptr(), size, stream)
            bs.bs_group_norm_backward(d, x.data_ptr(), res.data_ptr(), weight.data_ptr(), bias.data_ptr(), st.data_ptr(), dy.data_ptr(), gx.data_ptr(),
                                      gr.data_ptr(), gw.data_ptr(), gb.data_ptr(), ws.data_ptr(), size, stream)
            torch.cuda.synchronize()
            assert not memory.any()
            results.append((y, st, gx, gr, gw, gb))
        assert all(torch.equal(a, b) for a, b in zip(*results))


def test_graph_replays():
    """A recorded forward and backward pass, replayed between eager calls on the same stream, each replay against the eager result."""
    shape = (4, 128, 40, 40, 32)
    x, weight, bias, res, dy = tensors(shape, "bf16", 2, True)
    args = (shape[4], weight, bias, res, "gelu")

    def step():
        y, stats = F.group_norm_forward(x, *args)
        return (y, *F.group_norm_backward(x, stats, dy, *args))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)).to(x.dtype))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(a, b) for a, b in zip(got, step())), i


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(2, 4096, 5, 5, 1), (1, 1536, 40, 30, 2), (2, 168, 62, 55, 8), (1, 2050, 9, 8, 1), (2, 22, 30, 31, 2), (1, 6000, 3, 4, 3), (3, 512, 9, 9, 512),
                                   (1, 24, 260, 250, 24)])
def test_wide_groups_and_many_groups(shape, dtype):
    """Groups wider than a work-group's lanes, groups of one channel, vectors that reach over groups, channels that divide by two only."""
    check(shape, dtype, "silu", True, seed=8)
    check(shape, dtype, "gelu", False, seed=9)


@pytest.mark.parametrize("shape,dtype", [((9, 288, 61, 63, 32), "f16"), ((3, 336, 99, 101, 12), "bf16"), ((5, 1216, 31, 29, 32), "f32"), ((40, 30, 90, 91, 6), "bf16"),
                                         ((6, 95, 170, 90, 5), "f32")])
def test_large_tensors_of_odd_groups(shape, dtype):
    """Blocks of channels that begin inside cache lines."""
    check(shape, dtype, "silu", True, seed=10)
    check(shape, dtype, "relu", False, seed=11)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 16, 700, 821, 4), (2, 7, 620, 401, 7), (1, 1030, 120, 121, 2), (1, 12, 500, 1001, 1), (1, 64, 640, 641, 32)])
def test_images_that_do_not_fit_the_registers(shape, dtype):
    """Images of more parts than a work-group joins: statistics first, then the tensor once more.  (Chains of pixels are up to four times as long.)"""
    print(f"[group norm] {shape} {dtype}", flush=True)
    x, weight, bias, res, dy = tensors(shape, dtype, 12, True)
    for residual, name in ((res, "silu"), (None, "gelu")):
        args = (shape[4], weight, bias, residual, name)
        ref = Reference(x, shape[4], weight, bias, residual, name, 1e-5)
        y, stats = F.group_norm_forward(x, *args)
        close(y, ref.y, 4 * 1.13 * ref.z_off + 2e-6 * ref.y.abs() + 1e-7, dtype, "y")
        got = F.group_norm_backward(x, stats, dy, *args)
        for g, (want, off), label in zip(got, ref.backward(dy), ("grad_x", "grad_weight", "grad_bias", "grad_residual")):
            if g is not None:
                close(g, want, 4 * off, "f32" if label in ("grad_weight", "grad_bias") else dtype, label)
        assert all(a is None or torch.equal(a, b) for a, b in zip(got, F.group_norm_backward(x, stats, dy, *args)))
