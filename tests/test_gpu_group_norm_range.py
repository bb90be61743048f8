"""Group normalisation whose activations get arguments far from zero: the exponential at the ends of its range."""
import pytest
import torch

from paper_1804_08378_amd import functional as F
from test_gpu_group_norm import DTYPES, Reference, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["silu", "gelu", "identity", "relu"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 16, 41, 40, 4), (2, 60, 30, 31, 12), (1, 16, 700, 821, 4)])
def test_arguments_from_minus_120_to_120(shape, dtype, name):
    """The residual operand moves the activation's argument over the range where exp(-z) overflows and where it vanishes, -111 .. -88 densest."""
    n, c, h, w, groups = shape
    print(f"[group norm] {shape} {dtype} {name}", flush=True)
    g = torch.Generator().manual_seed(7)
    dt = DTYPES[dtype]
    cl = lambda t: t.to(dt).cuda().permute(0, 3, 1, 2)
    x, dy = cl(torch.randn(n, h, w, c, generator=g)), cl(torch.randn(n, h, w, c, generator=g))
    cells = h * w * c
    sweep = torch.cat([torch.linspace(-120, 120, cells // 2), torch.linspace(-113, -86, cells - cells // 2)])
    res = cl(sweep[torch.randperm(cells, generator=g)].view(1, h, w, c).expand(n, h, w, c).contiguous())
    weight, bias = torch.rand(c, generator=g).cuda() + 0.5, torch.randn(c, generator=g).cuda() * 0.3
    ref = Reference(x, groups, weight, bias, res, name, 1e-5)
    if name == "relu":  # next to the kink either gradient is right: none is asked for there
        dy = torch.where(ref.z.abs().cuda() <= 2 * ref.z_off.cuda() + 1e-6, torch.zeros_like(dy), dy)
    args = (groups, weight, bias, res, name)
    y, stats = F.group_norm_forward(x, *args)
    chains = 4 if cells > 1 << 20 else 1  # (chains of pixels are up to four times as long)
    close(y, ref.y, chains * 1.13 * ref.z_off + 2e-6 * ref.y.abs() + 1e-7, dtype, "y")
    got = F.group_norm_backward(x, stats, dy, *args)
    for grad, (want, off), label in zip(got, ref.backward(dy), ("grad_x", "grad_weight", "grad_bias", "grad_residual")):
        close(grad, want, chains * off, "f32" if label in ("grad_weight", "grad_bias") else dtype, label)
