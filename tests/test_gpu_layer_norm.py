"""Layer normalisation behind an addition on the GPU, against its definition in 64 bits (tolerances: rows_reference)."""
import pytest
import torch

import rows_reference as ref
from paper_1804_08378_amd import brainslug as bs
from paper_1804_08378_amd import functional as F

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (2, 2), (3, 5), (5, 8), (3, 31), (2, 32), (5, 33), (4, 64), (7, 96), (33, 128), (3, 255), (2, 256), (9, 257), (1, 511), (2, 512), (3, 1000), (2, 1024),
          (1, 2047), (70, 2048), (3, 2049), (1, 4096), (2, 4099), (1, 8192), (2, 8200), (3, 16384), (1, 16389), (2, 32768), (1, 40001), (1, 70000), (1000, 17), (4097, 8),
          (300, 771), (2500, 64), (1, 300001)]


def operands(shape, dtype, seed, params="f32", mean=0.0, addend=True):
    g = torch.Generator().manual_seed(seed)
    dt, pt, n = ref.DTYPES[dtype], ref.DTYPES[params], shape[-1]
    make = lambda scale=1.0, shift=0.0: (torch.randn(shape, generator=g) * scale + shift).to(dt).cuda()
    return (make(1.5, mean), (torch.rand(n, generator=g) + 0.5).to(pt).cuda(), (torch.randn(n, generator=g) * 0.3).to(pt).cuda(), make(0.7) if addend else None,
            make(), make() if addend else None)


def check(x, weight, bias, addend, dy, dt, checkpoint, eps=1e-5):
    print(f"[layer norm] {tuple(x.shape)} {x.dtype} addend={addend is not None} checkpoint={checkpoint}", flush=True)
    want = ref.Norm(x, weight, bias, addend, eps, checkpoint)
    r = F.layer_norm_forward(x, weight, bias, addend, eps, checkpoint)
    torch.cuda.synchronize()
    ref.close(r.y, want.y, want.y_off, "y")
    assert (r.total is None) == (addend is None) and (addend is None or torch.equal(r.total.cpu(), want.total))
    ref.close(r.stats[..., 0], want.mean[..., 0], (want.mean_off / want.rstd)[..., 0], "mean")
    ref.close(r.stats[..., 1], want.rstd[..., 0], (want.rstd_off * want.rstd)[..., 0], "rstd")
    assert (r.kept is None) == (not checkpoint)
    if checkpoint:
        codes, exponents = ref.pack8(want.total)
        assert torch.equal(r.kept.codes.cpu(), codes) and torch.equal(r.kept.exponents.cpu(), exponents)
    args = (r.kept if checkpoint else x if addend is None else r.total, r.stats, dy, weight, bias, dt)
    got = F.layer_norm_backward(*args)
    torch.cuda.synchronize()
    for g, (w, off), label in zip(got, want.backward(dy, dt), ("grad_x", "grad_weight", "grad_bias")):
        if g is not None:
            ref.close(g, w, off, label)
    assert (got[1] is None) == (weight is None) and (got[2] is None) == (bias is None)
    assert all(a is None or torch.equal(a, b) for a, b in zip(got, F.layer_norm_backward(*args))), "equal calls give equal bits"
    alone = F.layer_norm(x, weight, bias, addend, eps)
    assert torch.equal(alone if addend is None else alone[0], r.y)
    return r, got


@pytest.mark.parametrize("dtype", list(ref.DTYPES))
@pytest.mark.parametrize("shape", SHAPES)
def test_rows(shape, dtype):
    x, w, b, a, dy, dt = operands(shape, dtype, 1)
    check(x, w, b, None, dy, None, False)
    check(x, w, b, a, dy, dt, True)
    check(x, w, b, a, dy, None, False)
    check(x, None, None, None, dy, dt, True)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_parameters_of_the_rows_type(dtype):
    for shape in ((3, 77), (50, 1024), (2, 5000), (1, 20000)):
        x, w, b, a, dy, dt = operands(shape, dtype, 2, params=dtype)
        check(x, w, b, a, dy, dt, False)
        check(x, w, b, None, dy, None, True)
        check(x, w, None, None, dy, None, False)
        check(x, None, b, None, dy, None, False)


@pytest.mark.parametrize("dtype", list(ref.DTYPES))
def test_a_mean_far_from_zero(dtype):
    for shape in ((5, 40), (4, 1000), (2, 9000), (1, 33000)):
        x, w, b, _, dy, _ = operands(shape, dtype, 3, mean=40.0, addend=False)
        check(x, w, b, None, dy, None, False)
        check(x, w, b, None, dy, None, True)


@pytest.mark.parametrize("eps", [0.0, 1e-12, 1.0])
def test_eps(eps):
    x, w, b, a, dy, dt = operands((6, 200), "f32", 4)
    check(x, w, b, a, dy, dt, False, eps)


def test_sizes_of_numbers():
    """Rows of very small and very large numbers, whose squares float32 holds."""
    for scale in (1e-15, 1e-6, 1e6, 1e15):
        x, w, b, _, dy, _ = operands((4, 300), "f32", 5, addend=False)
        check(x * scale, w, b, None, dy, None, False, 0.0)


def test_constant_rows():
    """Deviations of 0: xh is 0, y the bias; the gradient of x is (u - mean u) / sqrt(eps)."""
    x, w, b, _, dy, _ = operands((3, 130), "f32", 6, addend=False)
    x = torch.full_like(x, 3.0)
    r = F.layer_norm_forward(x, w, b)
    assert torch.equal(r.y, b.expand(3, -1))
    want = ref.Norm(x, w, b, None, 1e-5, False)
    (dx, off), _, _ = want.backward(dy)
    ref.close(F.layer_norm_backward(x, r.stats, dy, w, b)[0], dx, off, "grad_x")


@pytest.mark.parametrize("features", [17, 300, 3001, 20001])
@pytest.mark.parametrize("addend", [False, True])
def test_rows_that_are_not_numbers_keep_to_themselves(features, addend):
    x, w, b, a, dy, dt = operands((6, features), "bf16", 7)
    a, dt = (a, dt) if addend else (None, None)
    bad = x.clone()
    bad[1, 3], bad[3, 0], bad[4, features - 1] = float("nan"), float("inf"), float("-inf")
    fine = [0, 2, 5]
    for checkpoint in (False, True):
        r, q = F.layer_norm_forward(bad, w, b, a, checkpoint=checkpoint), F.layer_norm_forward(x, w, b, a, checkpoint=checkpoint)
        assert torch.equal(r.y[fine], q.y[fine]) and r.y[[1, 3, 4]].isnan().all()
        kept = [s.kept if checkpoint else v if a is None else s.total for s, v in ((r, bad), (q, x))]
        g, h = F.layer_norm_backward(kept[0], r.stats, dy, w, b, dt), F.layer_norm_backward(kept[1], q.stats, dy, w, b, dt)
        assert torch.equal(g[0][fine], h[0][fine]) and g[0][[1, 3, 4]].isnan().all() and torch.equal(g[2], h[2])


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_strides_and_alignment(dtype):
    x, _, _, a, dy, dt = operands((8, 640), dtype, 8)
    g = torch.Generator().manual_seed(9)
    cuts = [lambda t: t[:, 3:100], lambda t: t[:, 1:34], lambda t: t[1:, :64], lambda t: t[2:3, 5:9], lambda t: t[::2, 7:], lambda t: t[:, ::2], lambda t: t.t()[:, :5],
            lambda t: t[0], lambda t: t.view(2, 4, 640)[:, :, 2:377], lambda t: t.view(2, 4, 640).transpose(0, 1), lambda t: t[:3].expand(2, 3, 640),
            lambda t: t.view(2, 4, 16, 40).contiguous(memory_format=torch.channels_last).permute(0, 2, 3, 1), lambda t: t[3, 17:18]]
    for i, cut in enumerate(cuts):
        for checkpoint in (False, True):
            n = cut(x).shape[-1]
            buffer = torch.randn(2, n + 3, generator=g).cuda()
            w, b = buffer[0, 3:], buffer[1, 1:n + 1]  # parameters begin anywhere
            # each operand with strides of its own
            other = cuts[i] if checkpoint else lambda t: cut(t).contiguous()
            check(cut(x), w, b, other(a), cut(dy), other(dt), checkpoint)


def test_wanted_gradients():
    x, w, b, a, dy, dt = operands((40, 333), "bf16", 10)
    r = F.layer_norm_forward(x, w, b, a)
    full = F.layer_norm_backward(r.total, r.stats, dy, w, b, dt)
    for need in [(True, False, False), (False, True, False), (False, False, True), (False, True, True), (True, True, False), (False, False, False)]:
        got = F.layer_norm_backward(r.total, r.stats, dy, w, b, dt, need)
        for g, f, wanted in zip(got, full, need):
            assert (g is not None) == wanted and (g is None or torch.equal(g, f))


def test_no_rows():
    x, w = torch.zeros(0, 7, device="cuda"), torch.ones(7, device="cuda")
    r = F.layer_norm_forward(x, w, w, x, checkpoint=True)
    assert r.y.shape == r.total.shape == x.shape and r.stats.shape == (0, 2) and r.kept.codes.shape == x.shape and r.kept.exponents.shape == (0, 1)
    for kept in (r.total, r.kept):
        gx, gw, gb = F.layer_norm_backward(kept, r.stats, x, w, w, x)
        assert gx.shape == x.shape and torch.equal(gw, torch.zeros(7, device="cuda")) and torch.equal(gb, gw)
    y, total = F.layer_norm(torch.zeros(3, 0, 7, device="cuda", requires_grad=True), w, w, torch.zeros(3, 0, 7, device="cuda"))
    y.sum().backward()


def test_many_rows():
    """More rows than work-groups walk over at once; sums over half a million rows."""
    x, w, b, _, dy, _ = operands((500001, 12), "f32", 11, addend=False)
    check(x, w, b, None, dy, None, False)


# rows for every number of lanes that one is spread over, several for each work-group, and lengths that leave some of the lanes without columns
MANY = [(70001, 23), (40001, 64), (33333, 40), (20001, 100), (9001, 200), (9001, 256), (4501, 391), (5001, 1000), (2601, 2048), (1401, 4001), (701, 8200), (601, 16384), (517, 12345),
        (601, 20000), (301, 32768), (291, 40002)]


@pytest.mark.parametrize("checkpoint", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", MANY)
def test_sums_over_many_rows(shape, dtype, checkpoint):
    x, w, b, a, dy, dt = operands(shape, dtype, 16)
    check(x, w, b, a if checkpoint else None, dy, dt if checkpoint else None, checkpoint)


def test_large_tensors():
    """Rows behind the first 2^32 bytes and 2^31 elements."""
    n = 8192
    x = torch.zeros((1 << 31) // n + 5, n, dtype=torch.bfloat16, device="cuda")
    dy = torch.zeros_like(x)
    rows = [0, 262143, x.shape[0] - 1]
    for row in rows:
        g = torch.Generator().manual_seed(row)
        x[row], dy[row] = torch.randn(n, generator=g).bfloat16().cuda(), torch.randn(n, generator=g).bfloat16().cuda()
    w, b = torch.rand(n).cuda() + 0.5, torch.randn(n).cuda()
    want = ref.Norm(x[rows], w, b, None, 1e-5, True)
    r = F.layer_norm_forward(x, w, b, checkpoint=True)
    ref.close(r.y[rows], want.y, want.y_off, "y")
    grads = F.layer_norm_backward(r.kept, r.stats, dy, w, b)
    (dx, off), (dw, dw_off), (db, db_off) = want.backward(dy[rows])
    ref.close(grads[0][rows], dx, off, "grad_x")
    ref.close(grads[1], dw, dw_off, "grad_weight")
    ref.close(grads[2], db, db_off, "grad_bias")
    del x, dy, r, grads
    torch.cuda.empty_cache()


def test_rows_in_the_middle_of_memory():
    """The C entries leave what is beside a strided tensor as it was, and take results and operands that lie in one buffer."""
    x, w, b, a, dy, dt = operands((7, 90), "bf16", 12)
    r = F.layer_norm_forward(x, w, b, a)
    gx = F.layer_norm_backward(r.total, r.stats, dy, w, b, dt)[0]
    joint = torch.full((7, 300), 5.0, dtype=torch.bfloat16, device="cuda")
    stats = torch.empty(7, 2, device="cuda")
    d = bs.bs_layer_norm_desc()
    d.rows, d.features, d.eps, d.dtype, d.param_dtype = 7, 90, 1e-5, bs.BS_BF16, bs.BS_F32
    d.y_stride = d.total_stride = d.grad_x_stride = 300
    stream = torch.cuda.current_stream().cuda_stream
    bs.bs_layer_norm(d, x.data_ptr(), a.data_ptr(), w.data_ptr(), b.data_ptr(), joint[:, 3:].data_ptr(), joint[:, 101:].data_ptr(), stats.data_ptr(), 0, 0, stream)
    d.x_stride = 300
    bs.bs_layer_norm_backward(d, joint[:, 101:].data_ptr(), 0, 0, stats.data_ptr(), w.data_ptr(), dy.data_ptr(), dt.data_ptr(), joint[:, 200:].data_ptr(), 0, 0, 0, 0, stream)
    assert torch.equal(joint[:, 3:93], r.y) and torch.equal(joint[:, 101:191], r.total) and torch.equal(joint[:, 200:290], gx)
    joint[:, 3:93] = joint[:, 101:191] = joint[:, 200:290] = 5.0
    assert (joint == 5).all()


# ------------------------------------------------------------------------------------------------ autograd
@pytest.mark.parametrize("checkpoint", [False, True])
def test_autograd(checkpoint):
    for shape, addend in (((4, 6, 50), True), ((30, 200), False), ((60,), True)):
        x, w, b, a, dy, dt = operands(shape, "f32", 13)
        a, dt = (a, dt) if addend else (None, None)
        leaves = [t.requires_grad_(True) for t in (x, w, b, a) if t is not None]
        out = F.layer_norm(x, w, b, a, checkpoint=checkpoint)
        y, total = out if addend else (out, None)
        want = ref.Norm(x, w, b, a, 1e-5, checkpoint)
        expected = want.backward(dy, dt)
        grads = torch.autograd.grad([t for t in (y, total) if t is not None], leaves, [t for t in (dy, dt) if t is not None], retain_graph=True)
        for g, (v, off), label in zip(grads, (*expected, expected[0]), ("x", "weight", "bias", "addend")):
            ref.close(g, v, off, label)
        if addend:  # one result's gradient alone
            (dx, off), _, _ = want.backward(dy)
            ref.close(torch.autograd.grad(y, a, dy, retain_graph=True)[0], dx, off, "y alone")
            assert torch.equal(torch.autograd.grad(total, x, dt, retain_graph=True)[0], dt)


def test_gradients_against_differences():
    """Central differences of the float32 forward pass, summed in 64 bits: steps of h = 2^-6 along a direction of size 1 leave an error of h^2 and
    roundings of 2^-24 sqrt(elements) / h, together under 1e-3 of gradients of size 1."""
    x, w, b, a, dy, dt = operands((5, 48), "f32", 14)
    leaves = [t.requires_grad_(True) for t in (x, w, b, a)]
    y, total = F.layer_norm(x, w, b, a)
    grads = torch.autograd.grad([y, total], leaves, [dy, dt])
    g = torch.Generator().manual_seed(15)
    value = lambda v: sum(float((p.double() * q.double()).sum()) for p, q in zip(F.layer_norm(*v), (dy, dt)))
    with torch.no_grad():
        for i, leaf in enumerate(leaves):
            e = torch.randn(leaf.shape, generator=g).cuda()
            e /= e.norm()
            h = 2.0 ** -6
            moved = [[t + s * h * e if j == i else t for j, t in enumerate(leaves)] for s in (1, -1)]
            diff = (value(moved[0]) - value(moved[1])) / (2 * h)
            assert abs(diff - float((grads[i].double() * e.double()).sum())) <= 1e-3 * (1 + float(grads[i].norm())), i


def test_module():
    m = F.LayerNorm(100, eps=1e-6, checkpoint=True).cuda()
    plain = torch.nn.LayerNorm(100, eps=1e-6)
    plain.load_state_dict({k: v.cpu() for k, v in m.state_dict().items()})
    x = torch.randn(3, 4, 100)
    assert float((m(x.cuda()).cpu() - plain(x)).detach().abs().max()) <= 1e-5  # values of a few units, some 40 roundings
    y, total = m(x.cuda(), x.cuda())
    assert torch.equal(total.cpu(), x + x) and y.requires_grad
    with pytest.raises(ValueError, match="features"):
        m(x[..., :99].cuda())
    assert F.LayerNorm(8, elementwise_affine=False).cuda()(x[..., :8].cuda()).shape == (3, 4, 8) and F.LayerNorm(8, bias=False).bias is None
    assert "checkpoint=True" in repr(m)


@pytest.mark.parametrize("dtype", list(ref.DTYPES))
@pytest.mark.parametrize("n", [5, 8, 100, 515, 4096, 16389, 40001])
def test_the_total_of_no_addend(n, dtype):
    """The C entry writes t where it is wanted, with an addend or without: then it is x.  Rows shorter than a vector, in registers, over memory."""
    x = torch.randn(3, n, dtype=ref.DTYPES[dtype], device="cuda")
    buffers = torch.full((2, 3, n + 16), 7.0, dtype=x.dtype, device="cuda")
    y, total = buffers[0, :, 8:8 + n], buffers[1, :, 8:8 + n]
    d = bs.bs_layer_norm_desc()
    d.rows, d.features, d.eps, d.dtype, d.param_dtype = 3, n, 1e-5, {"f32": bs.BS_F32, "bf16": bs.BS_BF16, "f16": bs.BS_F16}[dtype], bs.BS_F32
    d.y_stride = d.total_stride = n + 16
    bs.bs_layer_norm(d, x.data_ptr(), 0, 0, 0, y.data_ptr(), total.data_ptr(), 0, 0, 0, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(total, x) and torch.equal(y, F.layer_norm(x))
    assert (buffers[:, :, :8] == 7).all() and (buffers[:, :, 8 + n:] == 7).all()
