"""What the group-normalisation and log-probability entry points refuse, without a GPU: nothing is launched, no pointer is followed."""
import ctypes as C

import pytest
import torch

from paper_1804_08378_amd import brainslug as bs
from paper_1804_08378_amd import functional as F

NULL, SHAPE, PARAM, UNSUPPORTED, ALIGN, WORKSPACE, ALIAS = 1, 2, 3, 4, 7, 8, 12


def norm_desc(shape=(2, 32, 6, 5), groups=8, dtype=bs.BS_F32, param_dtype=bs.BS_F32, activation=bs.BS_ACT_SILU, eps=1e-5, **strides):
    d = bs.bs_group_norm_desc()
    d.shape[:] = shape
    d.groups, d.dtype, d.param_dtype, d.activation, d.eps = groups, dtype, param_dtype, activation, eps
    for k, v in strides.items():
        setattr(d, k, v)
    return d


def head_desc(rows=4, classes=100, dtype=bs.BS_F32, target_bytes=8, top=0, **more):
    d = bs.bs_log_probs_desc()
    d.rows, d.classes, d.dtype, d.target_bytes, d.top, d.ignore_index = rows, classes, dtype, target_bytes, top, -100
    for k, v in more.items():
        setattr(d, k, v)
    return d


def status(fn, *args):
    with pytest.raises(bs.BrainSlugError) as e:
        fn(*args)
    return e.value.status


# addresses that stand for buffers: 1 MiB apart, never followed
X, R, W, B, Y, S, WS, DY, DX, DR, DW, DB = (0x10000000 + i * 0x100000 for i in range(12))
BIG = 1 << 20


def forward(d, x=X, r=0, w=W, b=B, y=Y, s=S, ws=WS, n=BIG):
    return status(bs.bs_group_norm, d, x, r, w, b, y, s, ws, n, 0)


def backward(d, x=X, r=0, w=W, b=B, s=S, dy=DY, dx=DX, dr=0, dw=DW, db=DB, ws=WS, n=BIG):
    return status(bs.bs_group_norm_backward, d, x, r, w, b, s, dy, dx, dr, dw, db, ws, n, 0)


def test_group_norm_refusals():
    for call in (forward, backward):
        assert call(norm_desc((0, 32, 6, 5))) == SHAPE and call(norm_desc((2, 32, 0, 5))) == SHAPE
        assert call(norm_desc(groups=0)) == PARAM and call(norm_desc(groups=5)) == PARAM
        assert call(norm_desc(eps=-1.0)) == PARAM and call(norm_desc(eps=float("nan"))) == PARAM
        assert call(norm_desc(dtype=3)) == UNSUPPORTED and call(norm_desc(activation=4)) == UNSUPPORTED
        assert call(norm_desc(param_dtype=bs.BS_F16)) == UNSUPPORTED
        assert call(norm_desc((1, 1 << 20, 1 << 10, 2), 1)) == UNSUPPORTED  # 2^31 elements in an image
        assert call(norm_desc((1 << 20, 32, 1, 1), 32)) == UNSUPPORTED      # 2^25 groups
        assert call(norm_desc((1, 1 << 40, 1, 1), 1)) == UNSUPPORTED
        assert call(norm_desc(x_stride=31)) == SHAPE
        assert call(norm_desc(), x=0) == NULL
        assert call(norm_desc(), x=X + 2) == ALIGN and call(norm_desc(), w=W + 1) == ALIGN and call(norm_desc(), ws=WS + 8) == ALIGN
        assert call(norm_desc(), n=0) == WORKSPACE and call(norm_desc(), ws=0) == WORKSPACE
        assert call(norm_desc(), ws=X) == ALIAS
    need = bs.bs_group_norm_workspace_bytes(norm_desc(), False)
    assert 0 < need < BIG and forward(norm_desc(), n=need - 1) == WORKSPACE
    assert forward(norm_desc(), y=0) == NULL and forward(norm_desc(), y=X) == ALIAS and forward(norm_desc(), r=Y) == ALIAS
    assert forward(norm_desc(), s=Y) == ALIAS and forward(norm_desc(), s=W) == ALIAS
    assert backward(norm_desc(), s=0) == NULL and backward(norm_desc(), dy=0) == NULL
    assert backward(norm_desc(), dx=DY) == ALIAS and backward(norm_desc(), dr=DX) == ALIAS and backward(norm_desc(), dw=W) == ALIAS and backward(norm_desc(), dx=S) == ALIAS
    # overlapping channel slices of one buffer, next to each other they are none
    assert forward(norm_desc(x_stride=64, y_stride=64), y=X + 31 * 4) == ALIAS
    assert bs.bs_group_norm_workspace_bytes(norm_desc(groups=0), False) == 0
    lib = bs.load()
    assert lib.bs_group_norm(None, *[None] * 7, 0, None) == NULL and lib.bs_group_norm_backward(None, *[None] * 11, 0, None) == NULL
    assert lib.bs_group_norm_workspace_bytes(None, 0) == 0


@pytest.mark.parametrize("shape,groups", [((1, 1, 1, 1), 1), ((64, 256, 56, 56), 32), ((1, 771, 400, 300), 3), ((128, 2048, 7, 7), 32), ((1, 4096, 1, 1), 1),
                                          ((1 << 19, 32, 1, 1), 32), ((1, 8, 16000, 16000), 2)])
def test_group_norm_workspaces_stay_small(shape, groups):
    """Partial sums: at most a sixteenth of the tensor, or 4 MiB."""
    d = norm_desc(shape, groups, bs.BS_BF16)
    tensor = 2 * shape[0] * shape[1] * shape[2] * shape[3]
    for bwd in (False, True):
        n = bs.bs_group_norm_workspace_bytes(d, bwd)
        assert 0 < n <= max(4 << 20, tensor // 16 + 16 * shape[0] * max(groups, shape[1])), (n, tensor)


def test_group_norm_takes_many_small_images():
    """Launches count lanes in 32 bits: channel blocks grow where the images alone are millions."""
    for shape, groups in (((1 << 20, 1024, 1, 1), 16), ((1 << 22, 256, 1, 1), 4), ((1 << 22, 511, 1, 1), 1), ((1 << 21, 64, 2, 2), 8)):
        for dtype in (bs.BS_F32, bs.BS_F16):
            assert bs.bs_group_norm_workspace_bytes(norm_desc(shape, groups, dtype), False) > 0
    assert forward(norm_desc(((1 << 22) + 1, 8, 1, 1), 1)) == UNSUPPORTED


def head(d, x=X, t=Y, lp=S, e=WS, lse=DY, tl=0, ti=0, ws=0, n=0):
    return status(bs.bs_log_probs, d, x, t, lp, e, lse, tl, ti, ws, n, 0)


def head_backward(d, x=X, t=Y, lse=DY, e=WS, g=DW, h=DB, dx=DX):
    return status(bs.bs_log_probs_backward, d, x, t, lse, e, g, h, dx, 0)


def test_log_probs_refusals():
    for call in (head, head_backward):
        assert call(head_desc(rows=-1)) == SHAPE and call(head_desc(classes=0)) == SHAPE and call(head_desc(row_stride=99)) == SHAPE
        assert call(head_desc(grad_row_stride=99)) == SHAPE
        assert call(head_desc(dtype=5)) == UNSUPPORTED and call(head_desc(classes=(1 << 30) + 1)) == UNSUPPORTED and call(head_desc(rows=(1 << 23) + 1)) == UNSUPPORTED
        assert call(head_desc(target_bytes=2)) == PARAM and call(head_desc(top=33)) == PARAM and call(head_desc(top=-1)) == PARAM
        assert call(head_desc(classes=10, top=11)) == PARAM
        assert call(head_desc(), x=0) == NULL and call(head_desc(), x=X + 2) == ALIGN and call(head_desc(), t=Y + 4) == ALIGN
    assert head(head_desc(), t=0) == NULL and head(head_desc(top=3)) == NULL and head(head_desc(), lp=X) == ALIAS and head(head_desc(), e=S) == ALIAS
    assert head(head_desc(top=3), tl=R, ti=R) == ALIAS
    assert head_backward(head_desc(), lse=0) == NULL and head_backward(head_desc(), e=0) == NULL and head_backward(head_desc(), t=0) == NULL
    assert head_backward(head_desc(), dx=0) == NULL and head_backward(head_desc(), dx=X + 4) == ALIAS
    assert head_backward(head_desc(grad_row_stride=128), dx=X) == ALIAS and head_backward(head_desc(), dx=DY) == ALIAS
    lib = bs.load()
    assert lib.bs_log_probs(None, *[None] * 8, 0, None) == NULL and lib.bs_log_probs_backward(None, *[None] * 8) == NULL
    assert lib.bs_log_probs(C.byref(head_desc(rows=0)), *[None] * 8, 0, None) == 0  # no rows: nothing to do


def test_functions_refuse_what_they_cannot_take():
    x = torch.zeros(2, 8, 3, 3)
    with pytest.raises(RuntimeError, match="GPU"):
        F.group_norm(x, 2)
    with pytest.raises(RuntimeError, match="GPU"):
        F.log_probs(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="activation"):
        F.GroupNormAct(2, 8, "tanh")


def test_pixel_strides():
    """Which tensors are read in place: brute force over the addresses of every element."""
    base = torch.zeros(3, 5, 4, 12).permute(0, 3, 1, 2)  # channels last, 12 channels
    for t in (base, base[:, 2:9], base[:, :1], base[:1, :, :1], base[:, :, :1, :1], base[:, :, 1:3], base[:, :, :, :2], base.contiguous(), base[1:, 3:],
              base[:1, 4:8, :1, :1], base[::2], torch.zeros(1, 1, 4, 4), torch.zeros(2, 1, 3, 3)):
        n, c, h, w = t.shape
        sn, sc, sh, sw = t.stride()
        offsets = [i * sn + y * sh + z * sw + k * sc for i in range(n) for y in range(h) for z in range(w) for k in range(c)]
        step = F._pixel_stride(t)
        if step is not None:
            assert offsets == [p * step + k for p in range(n * h * w) for k in range(c)], (t.shape, t.stride())
        else:
            steps = {offsets[c * (p + 1)] - offsets[c * p] for p in range(n * h * w - 1)}
            assert len(steps) > 1 or min(steps) < c or (c > 1 and sc != 1), (t.shape, t.stride())


@pytest.mark.gpu
def test_native_and_python_calls_agree(monkeypatch):
    """The native calls take the plain case; without them the Python code makes the same call of the library."""
    g = torch.Generator().manual_seed(0)
    x, res, dy = (torch.randn(3, 24, 6, 5, generator=g).cuda().contiguous(memory_format=torch.channels_last) for _ in range(3))
    w, b = torch.rand(24, generator=g).cuda(), torch.randn(24, generator=g).cuda()
    logits, t, gl, ge = torch.randn(7, 300, generator=g).cuda(), torch.randint(0, 300, (7,), generator=g).cuda(), torch.randn(7, generator=g).cuda(), torch.randn(7, generator=g).cuda()

    def everything():
        y, stats = F.group_norm_forward(x, 4, w, b, res, "gelu")
        r = F.log_probs_forward(logits, t, 6)
        return [y, stats, F.group_norm(x, 4, w, None), *F.group_norm_backward(x, stats, dy, 4, w, b, res, "gelu", need=(True, False, True, True)),
                *r, F.log_probs_backward(logits, t, r.lse, r.entropy, gl, None), F.log_probs_backward(logits, t, r.lse, r.entropy, gl, ge)]

    assert F._native_calls(), "the native calls are built"
    native = everything()
    monkeypatch.setattr(F, "_native", False)
    for a, c in zip(native, everything()):
        assert (a is None and c is None) or torch.equal(a, c)
    monkeypatch.undo()
    with pytest.raises(ValueError, match="residual"):
        F.group_norm(x, 4, w, b, res[:, :8])
    with pytest.raises(bs.BrainSlugError) as e:
        F.group_norm(x, 5, w, b)
    assert e.value.status == PARAM
    with pytest.raises(bs.BrainSlugError) as e:
        F.log_probs(logits, t, 33)
    assert e.value.status == PARAM
    with pytest.raises(TypeError):
        F.log_probs(logits.double(), t)
    with pytest.raises(ValueError, match="targets"):
        F.log_probs(logits, t[:3])
