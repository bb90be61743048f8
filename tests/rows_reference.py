"""Layer normalisation, activations and the 8-bit form by their definitions, in 64 bits on the CPU, with what the tests' tolerances need.

Tolerances.  With u = 2^-24: float32 sums here run over chains of at most a few hundred terms (elements of a lane, then lanes, then parts of the
rows), so a sum is off by less than 300 u = 2e-5 of the sum of its terms' magnitudes, a mean by 2e-5 deviations and 4 u of its own size (the last
roundings), results by that times the factors behind it.  Results are rounded once: half a unit in the last place, 2^-24, 2^-8 or 2^-11 of the
value, and in binary16 half of its smallest step, 2^-25.  The 8-bit form is exact: whole numbers of a power of two.
"""
import math

import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROUNDING = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
U, SUMS = 2.0 ** -24, 2e-5
BLOCK = 32


def cpu(t):
    return None if t is None else t.detach().cpu().double().contiguous()


def close(got, want, off, label):
    """`got`, on the GPU and of its own type, against `want` +- `off`, rounded."""
    dtype, got = got.dtype, got.detach().cpu().double()
    assert got.shape == want.shape, (label, got.shape, want.shape)
    bound = off + ROUNDING[dtype] * 1.01 * (want.abs() + off) + (2.0 ** -25 if dtype == torch.float16 else 1e-37)
    bad = ~((got - want).abs() <= bound) & ~((got == want) | (got.isnan() & want.isnan()))
    assert not bad.any(), (label, int(bad.sum()), float(((got - want).abs() / bound)[bad][0]), got[bad][0], want[bad][0])


# ------------------------------------------------------------------------------------------------ 8 bits
def pack8(x):
    """(codes, exponents) of rows of any of the types, from numbers: x = m * 2^k, 1/2 <= m < 1."""
    largest = 142 if x.dtype == torch.float16 else 254
    rows = cpu(x).reshape(-1, x.shape[-1])
    n = rows.shape[1]
    blocks = -(-n // BLOCK)
    v = torch.zeros(rows.shape[0], blocks * BLOCK, dtype=torch.float64)
    v[:, :n] = rows
    v = v.view(-1, blocks, BLOCK)
    top = torch.where(v.isfinite(), v.abs(), 0.0).amax(2)
    m, k = torch.frexp(top)
    e = torch.where(m * 128 >= 126.5, k + 1, k) + 126  # 128 steps are the power of two above the largest: 2^(E - 133) * 128 = 2^k
    e = torch.where(top < 2.0 ** -126, (top >= 125 * 2.0 ** -133).to(e.dtype), e).clamp(0, largest)  # subnormal: the formula's border is 125 steps
    step = torch.ldexp(torch.ones_like(top), e - 133)[:, :, None]
    codes = torch.round(v / step).clamp(-126, 126)
    codes = torch.where(v == math.inf, 127.0, torch.where(v == -math.inf, -127.0, torch.where(v.isnan(), -128.0, codes)))
    codes = codes.reshape(rows.shape[0], -1)[:, :n].to(torch.int8)
    return codes.reshape(x.shape), e.to(torch.uint8).reshape(*x.shape[:-1], blocks)


def unpack8(codes, exponents):
    """The values that codes and exponents stand for, in 64 bits."""
    c = codes.cpu().double()
    e = exponents.cpu().to(torch.int32).repeat_interleave(BLOCK, -1)[..., :c.shape[-1]]
    v = torch.ldexp(c, e - 133)
    return torch.where(c == 127, math.inf, torch.where(c == -127, -math.inf, torch.where(c == -128, math.nan, v)))


def held(x):
    return unpack8(*pack8(x))


# ------------------------------------------------------------------------------------------------ activations
def activation(name, z):
    return {"identity": lambda v: v, "relu": lambda v: torch.where(v > 0, v, 0.0), "silu": lambda v: v * torch.sigmoid(v),
            "gelu": lambda v: 0.5 * v * torch.erfc(-v / math.sqrt(2))}[name](z)


def slope(name, z):
    s = torch.sigmoid(z)
    return {"identity": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(), "silu": lambda: s * (1 + z * (1 - s)),
            "gelu": lambda: 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)}[name]()


# ------------------------------------------------------------------------------------------------ layer normalisation
class Norm:
    """t = round(x + addend) normalised over its last dimension; `checkpoint`: the backward pass at t's values in 8 bits."""

    def __init__(self, x, weight, bias, addend, eps, checkpoint):
        # the sum of two float32 numbers is rounded to float32 first (a no-op for float32 tensors), then to their type
        self.total = x.detach().cpu() if addend is None else (x.detach().cpu().float() + addend.detach().cpu().float()).to(x.dtype)
        t, n = self.total.double(), x.shape[-1]
        self.weight = torch.ones(n).double() if weight is None else cpu(weight)
        bias = torch.zeros(n).double() if bias is None else cpu(bias)
        self.mean = t.mean(-1, keepdim=True)
        var = ((t - self.mean) ** 2).mean(-1, keepdim=True)
        self.rstd = 1 / torch.sqrt(var + eps)
        xh = (t - self.mean) * self.rstd
        self.y = xh * self.weight + bias
        # how far the mean may be off, in deviations, and the reciprocal deviation, relative
        self.mean_off = SUMS + 4 * U * self.mean.abs() * self.rstd
        self.rstd_off = 2 * SUMS + 4 * U
        off = self.mean_off + self.rstd_off * xh.abs()
        self.y_off = off * self.weight.abs() + 4 * U * (self.y.abs() + bias.abs())
        t = held(self.total) if checkpoint else t
        self.xh = (t - self.mean) * self.rstd
        self.xh_off = self.mean_off + self.rstd_off * self.xh.abs() + 4 * U * (t.abs() * self.rstd)

    def backward(self, dy, dt=None):
        dy, dt = cpu(dy), cpu(dt)
        u = dy * self.weight
        xh, x_off = self.xh, self.xh_off
        m1, m2 = u.mean(-1, keepdim=True), (u * xh).mean(-1, keepdim=True)
        dx = self.rstd * (u - m1 - xh * m2)
        u_off = 2 * U * u.abs()
        m1_off = u_off.mean(-1, keepdim=True) + SUMS * u.abs().mean(-1, keepdim=True)
        m2_off = (u_off * xh.abs() + u.abs() * x_off).mean(-1, keepdim=True) + SUMS * (u * xh).abs().mean(-1, keepdim=True)
        off = self.rstd * (u_off + m1_off + xh.abs() * m2_off + x_off * m2.abs() + (self.rstd_off + 8 * U) * (u.abs() + m1.abs() + (xh * m2).abs()))
        if dt is not None:
            dx, off = dx + dt, off + 4 * U * (dx.abs() + dt.abs())
        flat = lambda v: v.reshape(-1, v.shape[-1])
        dw, dw_off = flat(dy * xh).sum(0), flat(dy.abs() * x_off).sum(0) + SUMS * flat(dy * xh).abs().sum(0)
        return (dx, off), (dw, dw_off), (flat(dy).sum(0), SUMS * flat(dy).abs().sum(0))
