"""What training a network from scratch needs beside its stacks, on torch tensors: group normalisation with a residual operand and an
activation (channels last), the log probabilities at a classifier's end, layer normalisation behind an addition, activations with a gate, each
with its gradients, and what the backward passes need held in 8 bits.

`group_norm`, `log_probs`, `layer_norm` and `activate` are differentiable functions; `GroupNormAct` and `LayerNorm` are the normalisations as
modules.  The `_forward` / `_backward` pairs are the single passes, for programs that keep their own tape.  `pack8` / `unpack8` hold a tensor in 8
bits; `checkpoints_in_8_bits` holds what autograd keeps for any layer so.  Everything runs on the current stream of the tensors' device through the
C ABI (`bs_group_norm`, `bs_log_probs`, `bs_layer_norm`, `bs_activate`, `bs_pack8` in include/brainslug.h); there is no fallback: tensors the library cannot take raise.  What overrides
torch's functions overrides these too: `torch.fx` records a call of one of them as one node, so `optimize_graph` and `capture` take models with them.
"""
from __future__ import annotations

import collections
import ctypes as C
import operator
from typing import NamedTuple, Optional, Tuple

import torch
from torch import nn
from torch.autograd import forward_ad
from torch.overrides import handle_torch_function, has_torch_function_variadic

from . import brainslug as bs

__all__ = ["group_norm", "group_norm_forward", "group_norm_backward", "GroupNormAct", "log_probs", "log_probs_forward", "log_probs_backward",
           "LogProbs", "layer_norm", "layer_norm_forward", "layer_norm_backward", "LayerNormed", "LayerNorm", "activate", "activate_forward",
           "activate_backward", "Activated", "pack8", "unpack8", "Packed8", "checkpoints_in_8_bits", "ACTIVATIONS"]

ACTIVATIONS = {"identity": bs.BS_ACT_IDENTITY, "relu": bs.BS_ACT_RELU, "silu": bs.BS_ACT_SILU, "gelu": bs.BS_ACT_GELU}
_DTYPES = {torch.float32: bs.BS_F32, torch.bfloat16: bs.BS_BF16, torch.float16: bs.BS_F16}


_native = None  # the native calls (csrc/bs_torch.cpp), False: not built for this torch; None: not looked for yet


def _native_calls():
    """Every one of them takes the plain case -- tensors (no subclasses) that are read in place, on one device, without modes, forward-mode
    derivatives or tracing -- and returns None for any other, which the Python code hands on, takes or refuses."""
    global _native
    if _native is None:
        with bs._native_lock:
            if _native is None:
                module, lib = bs._torch_calls(), bs.load()
                if module is not None:
                    names = ("bs_group_norm_workspace_bytes", "bs_group_norm", "bs_group_norm_backward", "bs_log_probs_workspace_bytes", "bs_log_probs",
                             "bs_log_probs_backward", "bs_layer_norm", "bs_layer_norm_workspace_bytes", "bs_layer_norm_backward", "bs_activate",
                             "bs_activate_backward", "bs_pack8", "bs_unpack8")
                    module.set_operators(tuple(C.cast(getattr(lib, n), C.c_void_p).value for n in names))
                _native = module or False
    return _native


def _dtype(t: torch.Tensor, what: str) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what}: float32, bfloat16 and float16 tensors, not {t.dtype}")
    return code


def _integer(v, what: str, bits: int = 32) -> int:
    """Fields of the C descriptions cut numbers off without a word."""
    v = operator.index(v)
    if not -1 << bits - 1 <= v < 1 << bits - 1:
        raise ValueError(f"{what}: {v} does not fit {bits} bits")
    return v


def _on_gpu(t: torch.Tensor, what: str) -> None:
    if not t.is_cuda:
        raise RuntimeError(f"{what} needs tensors on the GPU")


def _refuse_recorders(what: str, *tensors: Optional[torch.Tensor]) -> None:
    """Results are written through pointers: whoever records or derives operations on tensors would see an empty tensor and nothing else."""
    if torch.jit.is_tracing():
        raise RuntimeError(f"{what}: torch.jit.trace records calls of the differentiable functions, not the single passes, nor calls with out")
    if any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise NotImplementedError(f"{what} has no forward-mode derivatives")


def _ptr(t: Optional[torch.Tensor]) -> int:
    return t.data_ptr() if t is not None else 0


def _workspace(n: int, like: torch.Tensor) -> Optional[torch.Tensor]:
    """Of the call's own: torch's allocator hands the memory on to later work of the same stream only."""
    return torch.empty(n, dtype=torch.uint8, device=like.device) if n else None


# ------------------------------------------------------------------------------------------------ group normalisation
def _pixel_stride(t: torch.Tensor) -> Optional[int]:
    """Elements from a pixel to the next of a 4-D tensor whose channels are contiguous in every pixel and whose pixels follow each other
    (channels last, or a channel slice of such a tensor), else None."""
    n, c, h, w = t.shape
    sn, sc, sh, sw = t.stride()
    step = sw if w > 1 else sh if h > 1 else sn if n > 1 else c
    if step >= c and (c == 1 or sc == 1) and (w == 1 or sw == step) and (h == 1 or sh == w * step) and (n == 1 or sn == h * w * step):
        return int(step)
    return None


def _readable(t: torch.Tensor) -> Tuple[torch.Tensor, int]:
    """`t` and its pixel stride; a copy in channels-last order where it cannot be read in place."""
    t = t.resolve_neg()
    step = _pixel_stride(t)
    if step is None:
        t = t.contiguous(memory_format=torch.channels_last)
        step = t.shape[1]
    return t, step


def _norm_operands(x, groups, weight, bias, residual, activation, eps, grad=None):
    """Checked operands and the call's description."""
    _on_gpu(x, "group_norm")
    if x.dim() != 4:
        raise ValueError("group_norm needs a 4-D tensor (N, C, H, W)")
    if activation not in ACTIVATIONS:
        raise ValueError(f"group_norm: activation {activation!r}, not one of {', '.join(ACTIVATIONS)}")
    d = bs.bs_group_norm_desc()
    d.dtype = _dtype(x, "group_norm")
    d.groups, d.activation, d.eps = _integer(groups, "group_norm: groups"), ACTIVATIONS[activation], float(eps)
    d.shape[:] = x.shape
    d.param_dtype = bs.BS_F32
    params = [p for p in (weight, bias) if p is not None]
    if params:
        d.param_dtype = _dtype(params[0], "group_norm")
    for p in params:
        if tuple(p.shape) != (x.shape[1],) or not p.is_contiguous() or p.is_neg() or p.device != x.device:
            raise ValueError("group_norm: weight and bias hold one element a channel, contiguous (no negated view), on x's device")
        if p.dtype not in (torch.float32, x.dtype) or p.dtype != params[0].dtype:
            raise TypeError("group_norm: weight and bias are both float32 or both of x's type")
    for t, name in ((residual, "residual"), (grad, "grad")):
        if t is not None and (t.shape != x.shape or t.dtype != x.dtype or t.device != x.device):
            raise ValueError(f"group_norm: {name} must have x's shape, type and device (no broadcasting)")
    x, d.x_stride = _readable(x)
    if residual is not None:
        residual, d.residual_stride = _readable(residual)
    if grad is not None:
        grad, d.grad_y_stride = _readable(grad)
    return d, x, residual, grad


def _run_norm(x, groups, weight, bias, residual, activation, eps, out, keep_stats, recorded=False):
    """`recorded`: called by the node that a recorder sees."""
    native, act = _native_calls(), ACTIVATIONS.get(activation)
    if native and out is None and act is not None:
        done = native.group_norm(x, groups, weight, bias, residual, act, eps, keep_stats)
        if done is not None:
            return done if keep_stats else (done, None)
    if not recorded:
        if has_torch_function_variadic(x, weight, bias, residual):  # (group_norm has looked already)
            return handle_torch_function(group_norm_forward, (x, weight, bias, residual), x, groups, weight, bias, residual, activation, eps, out)
        if torch.jit.is_tracing() and not keep_stats and out is None:
            return _GroupNorm.apply(x, weight, bias, residual, groups, activation, eps), None
        _refuse_recorders("group_norm", x, weight, bias, residual)
    d, x, residual, _ = _norm_operands(x, groups, weight, bias, residual, activation, eps)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device, memory_format=torch.channels_last)
    else:
        step = _pixel_stride(out)
        if out.shape != x.shape or out.dtype != x.dtype or out.device != x.device or step is None or out.is_neg():
            raise ValueError("group_norm: out must have x's shape, type and device, channels last or a channel slice of such a tensor")
        d.y_stride = step
        torch.autograd.graph.increment_version(out)  # (written through its pointer, which autograd does not see)
    stats = torch.empty((x.shape[0], max(1, min(d.groups, x.shape[1])), 2), dtype=torch.float32, device=x.device) if keep_stats else None
    if x.numel() == 0 and x.shape[0] == 0:
        return out, stats  # no images
    n = bs.bs_group_norm_workspace_bytes(d, False)
    ws = _workspace(n, x)
    with torch.cuda.device(x.device):
        bs.bs_group_norm(d, x.data_ptr(), _ptr(residual), _ptr(weight), _ptr(bias), out.data_ptr(), _ptr(stats), _ptr(ws), n,
                         torch.cuda.current_stream(x.device).cuda_stream)
    return out, stats


def group_norm_forward(x, groups: int, weight=None, bias=None, residual=None, activation: str = "identity", eps: float = 1e-5,
                       out: Optional[torch.Tensor] = None):
    """`(y, stats)`: the forward pass and, N x groups x 2 float32, the means and reciprocal deviations that `group_norm_backward` needs.
    `x` and `residual` are channels last, or channel slices of such tensors (read in place; other memory orders are copied first); `y` is
    channels last, or written to `out`."""
    with torch.no_grad():
        return _run_norm(x, groups, weight, bias, residual, activation, eps, out, True)


def group_norm_backward(x, stats, grad, groups: int, weight=None, bias=None, residual=None, activation: str = "identity", eps: float = 1e-5,
                        need=(True, True, True, True)):
    """`(grad_x, grad_weight, grad_bias, grad_residual)` from the gradient `grad` of `group_norm_forward`'s result; `need` says which of
    them are wanted (those of absent operands are None)."""
    native, act = _native_calls(), ACTIVATIONS.get(activation)
    if native and act is not None:
        done = native.group_norm_backward(x, stats, grad, groups, weight, bias, residual, act, eps, need[0] | need[1] << 1 | need[2] << 2 | need[3] << 3)
        if done is not None:
            return done
    if has_torch_function_variadic(x, stats, grad, weight, bias, residual):
        return handle_torch_function(group_norm_backward, (x, stats, grad, weight, bias, residual), x, stats, grad, groups, weight, bias, residual,
                                     activation, eps, need)
    _refuse_recorders("group_norm_backward", x, stats, grad, weight, bias, residual)
    with torch.no_grad():
        d, x, residual, grad = _norm_operands(x, groups, weight, bias, residual, activation, eps, grad)
        if tuple(stats.shape) != (x.shape[0], groups, 2) or stats.dtype != torch.float32 or not stats.is_contiguous() or stats.device != x.device:
            raise ValueError("group_norm_backward: stats must be those of group_norm_forward")

        def like(wanted, t):
            return torch.empty(t.shape, dtype=t.dtype, device=t.device, memory_format=torch.channels_last if t.dim() == 4 else torch.contiguous_format) \
                if wanted and t is not None else None

        gx, gw, gb, gr = like(need[0], x), like(need[1], weight), like(need[2], bias), like(need[3], residual)
        if x.shape[0] == 0:
            for g in (gw, gb):
                if g is not None:
                    g.zero_()
            return gx, gw, gb, gr
        n = bs.bs_group_norm_workspace_bytes(d, True)
        ws = _workspace(n, x)
        with torch.cuda.device(x.device):
            bs.bs_group_norm_backward(d, x.data_ptr(), _ptr(residual), _ptr(weight), _ptr(bias), stats.data_ptr(), grad.data_ptr(), _ptr(gx), _ptr(gr),
                                      _ptr(gw), _ptr(gb), _ptr(ws), n, torch.cuda.current_stream(x.device).cuda_stream)
        return gx, gw, gb, gr


class _GroupNorm(torch.autograd.Function):
    """One node of the graph: keeps the operands and the statistics, no intermediate tensor."""

    @staticmethod
    def forward(ctx, x, weight, bias, residual, groups, activation, eps):
        y, stats = _run_norm(x, groups, weight, bias, residual, activation, eps, None, True, recorded=True)
        ctx.save_for_backward(x, weight, bias, residual, stats)
        ctx.args = groups, activation, eps
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        x, weight, bias, residual, stats = ctx.saved_tensors
        groups, activation, eps = ctx.args
        return (*group_norm_backward(x, stats, grad, groups, weight, bias, residual, activation, eps, ctx.needs_input_grad[:4]), None, None, None)


def group_norm(x, groups: int, weight=None, bias=None, residual=None, activation: str = "identity", eps: float = 1e-5, out: Optional[torch.Tensor] = None):
    """act(group_norm(x) * weight + bias + residual), channels last; differentiable in every tensor.  See `group_norm_forward`; `out` is
    for calls that autograd does not record."""
    if has_torch_function_variadic(x, weight, bias, residual):
        return handle_torch_function(group_norm, (x, weight, bias, residual), x, groups, weight, bias, residual, activation, eps, out)
    if torch.is_grad_enabled() and (x.requires_grad or (weight is not None and weight.requires_grad) or (bias is not None and bias.requires_grad) or
                                    (residual is not None and residual.requires_grad)):
        if out is not None:
            raise RuntimeError("group_norm: out is for calls that autograd does not record")
        return _GroupNorm.apply(x, weight, bias, residual, groups, activation, eps)
    return _run_norm(x, groups, weight, bias, residual, activation, eps, out, False)[0]


class GroupNormAct(nn.GroupNorm):
    """`nn.GroupNorm` (same parameters, same state dict) with an activation behind it and an optional residual operand in front of the
    activation: `m(x)`, `m(x, residual)`.  Unlike it, x is 4-D, the parameters are contiguous, and the result is channels last whatever x's
    memory order (other orders than channels last are copied first)."""

    def __init__(self, num_groups: int, num_channels: int, activation: str = "relu", eps: float = 1e-5, affine: bool = True, device=None, dtype=None):
        super().__init__(num_groups, num_channels, eps, affine, device=device, dtype=dtype)
        if activation not in ACTIVATIONS:
            raise ValueError(f"GroupNormAct: activation {activation!r}, not one of {', '.join(ACTIVATIONS)}")
        self.activation = activation

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        return group_norm(x, self.num_groups, self.weight, self.bias, residual, self.activation, self.eps)

    def extra_repr(self) -> str:
        return super().extra_repr() + f", activation={self.activation!r}"


# ------------------------------------------------------------------------------------------------ log probabilities
class LogProbs(NamedTuple):
    """Per row: log probability of the given class (None without targets), entropy, top alternatives, most probable first (None for top = 0),
    and the logarithm of the sum of exponentials, float64, that `log_probs_backward` needs."""
    logp: Optional[torch.Tensor]
    entropy: torch.Tensor
    top_logp: Optional[torch.Tensor]
    top_index: Optional[torch.Tensor]
    lse: torch.Tensor


def _head_operands(logits, targets, top, ignore_index):
    _on_gpu(logits, "log_probs")
    if logits.dim() != 2:
        raise ValueError("log_probs needs rows of logits: a 2-D tensor")
    d = bs.bs_log_probs_desc()
    d.dtype = _dtype(logits, "log_probs")
    d.rows, d.classes = logits.shape
    if targets is not None:
        if tuple(targets.shape) != (logits.shape[0],) or targets.dtype not in (torch.int64, torch.int32) or targets.device != logits.device:
            raise ValueError("log_probs: targets hold one int64 or int32 class a row, on the logits' device")
        targets = targets.contiguous()
    d.target_bytes = 4 if targets is not None and targets.dtype == torch.int32 else 8
    d.ignore_index, d.top, d.lse_bytes = _integer(ignore_index, "log_probs: ignore_index", 64), _integer(top, "log_probs: top"), 8
    return d, targets


def _row_stride(t: torch.Tensor) -> Optional[int]:
    rows, classes = t.shape
    if (classes <= 1 or t.stride(1) == 1) and (rows <= 1 or t.stride(0) >= classes):
        return int(t.stride(0)) if rows > 1 else classes
    return None


def _readable_rows(t: torch.Tensor) -> Tuple[torch.Tensor, int]:
    t = t.resolve_neg()
    step = _row_stride(t)
    return (t, step) if step is not None else (t.contiguous(), t.shape[1])


def log_probs_forward(logits, targets=None, top: int = 0, ignore_index: int = -100) -> LogProbs:
    """Log probabilities of `targets`, entropy and `top` best classes of every row of `logits` (rows x classes; rows may lie further apart
    than they are long).  What masked classes, empty rows and ignored targets give stands at bs_log_probs in include/brainslug.h."""
    return _run_log_probs(logits, targets, top, ignore_index)


def _run_log_probs(logits, targets, top, ignore_index, recorded=False, traced=False) -> LogProbs:
    """`recorded`: called by the node that a recorder sees; `traced`: make that node where torch.jit.trace records."""
    native = _native_calls()
    if native:
        done = native.log_probs(logits, targets, top, ignore_index)
        if done is not None:
            return LogProbs(*done)
    if not recorded:
        if has_torch_function_variadic(logits, targets):  # (log_probs has looked already)
            return handle_torch_function(log_probs_forward, (logits, targets), logits, targets, top, ignore_index)
        if traced and torch.jit.is_tracing():
            return LogProbs(*_LogProbs.apply(logits, targets, top, ignore_index))
        _refuse_recorders("log_probs", logits)
    with torch.no_grad():
        d, targets = _head_operands(logits, targets, top, ignore_index)
        logits, d.row_stride = _readable_rows(logits)
        rows, dev = logits.shape[0], logits.device
        f32 = dict(dtype=torch.float32, device=dev)
        logp = torch.empty(rows, **f32) if targets is not None else None
        entropy, lse = torch.empty(rows, **f32), torch.empty(rows, dtype=torch.float64, device=dev)
        top_logp = torch.empty((rows, top), **f32) if top else None
        top_index = torch.empty((rows, top), dtype=torch.int32, device=dev) if top else None
        n = bs.bs_log_probs_workspace_bytes(d)
        ws = _workspace(n, logits)
        with torch.cuda.device(dev):
            bs.bs_log_probs(d, logits.data_ptr(), _ptr(targets), _ptr(logp), entropy.data_ptr(), lse.data_ptr(), _ptr(top_logp), _ptr(top_index),
                            _ptr(ws), n, torch.cuda.current_stream(dev).cuda_stream)
        return LogProbs(logp, entropy, top_logp, top_index, lse)


def log_probs_backward(logits, targets, lse, entropy, grad_logp=None, grad_entropy=None, ignore_index: int = -100,
                       out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient with respect to the logits from those of `logp` and `entropy` (a float a row; None: zero).  `lse` as `log_probs_forward` gives
    it; rounded to float32 it is taken too, and probabilities are off by that rounding.  `out=logits` writes the gradient over the logits."""
    native = _native_calls()
    if native and out is None:
        done = native.log_probs_backward(logits, targets, lse, entropy, grad_logp, grad_entropy, ignore_index)
        if done is not None:
            return done
    if has_torch_function_variadic(logits, targets, lse, entropy, grad_logp, grad_entropy):
        return handle_torch_function(log_probs_backward, (logits, targets, lse, entropy, grad_logp, grad_entropy), logits, targets, lse, entropy,
                                     grad_logp, grad_entropy, ignore_index, out)
    _refuse_recorders("log_probs_backward", logits, lse, entropy, grad_logp, grad_entropy)
    with torch.no_grad():
        d, targets = _head_operands(logits, targets, 0, ignore_index)
        rows = logits.shape[0]
        given = []
        for t in (lse, entropy, grad_logp, grad_entropy):
            if t is not None and (tuple(t.shape) != (rows,) or t.device != logits.device or
                                  not (t.dtype == torch.float32 or (t is lse and t.dtype == torch.float64))):
                raise ValueError("log_probs_backward: lse, entropy and their gradients hold one float32 (lse: or float64) a row, on the logits' device")
            given.append(t.resolve_neg().contiguous() if t is not None else None)
        lse, entropy, grad_logp, grad_entropy = given
        d.lse_bytes = lse.element_size()
        if out is None:
            out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        elif out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device or _row_stride(out) is None or out.is_neg():
            raise ValueError("log_probs_backward: out must have the logits' shape, type and device, its classes contiguous")
        else:
            torch.autograd.graph.increment_version(out)  # (written through its pointer, which autograd does not see)
        d.grad_row_stride = _row_stride(out)
        logits, d.row_stride = _readable_rows(logits)
        with torch.cuda.device(logits.device):
            bs.bs_log_probs_backward(d, logits.data_ptr(), _ptr(targets), lse.data_ptr(), _ptr(entropy), _ptr(grad_logp), _ptr(grad_entropy),
                                     out.data_ptr(), torch.cuda.current_stream(logits.device).cuda_stream)
        return out


class _LogProbs(torch.autograd.Function):
    """Keeps the logits, the targets and two floats a row.  Gradients flow through logp and entropy; the alternatives are answers."""

    @staticmethod
    def forward(ctx, logits, targets, top, ignore_index):
        r = _run_log_probs(logits, targets, top, ignore_index, recorded=True)
        ctx.save_for_backward(logits, targets, r.lse, r.entropy)
        ctx.ignore_index = ignore_index
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*[t for t in (r.top_logp, r.top_index, r.lse) if t is not None])
        return tuple(r)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_logp, grad_entropy, *_):
        logits, targets, lse, entropy = ctx.saved_tensors
        if grad_logp is None and grad_entropy is None:
            return None, None, None, None
        return log_probs_backward(logits, targets, lse, entropy, grad_logp, grad_entropy, ctx.ignore_index), None, None, None


def log_probs(logits, targets=None, top: int = 0, ignore_index: int = -100) -> LogProbs:
    """`log_probs_forward`, differentiable in `logp` and `entropy`: a cross entropy is `-log_probs(logits, targets).logp.mean()`."""
    if has_torch_function_variadic(logits, targets):
        return handle_torch_function(log_probs, (logits, targets), logits, targets, top, ignore_index)
    if torch.is_grad_enabled() and logits.requires_grad:
        return LogProbs(*_LogProbs.apply(logits, targets, top, ignore_index))
    return _run_log_probs(logits, targets, top, ignore_index, traced=True)


# ------------------------------------------------------------------------------------------------ rows
def _rows(t: torch.Tensor) -> Optional[Tuple[int, int]]:
    """Rows (all dimensions but the last) of a tensor whose rows are contiguous and follow each other at one distance, and that distance; else
    None.  Nothing reads a tensor without elements."""
    columns = t.shape[-1]
    if t.numel() == 0:
        return t.numel() // max(1, columns), columns
    if columns > 1 and t.stride(-1) != 1:
        return None
    rows, step = 1, None
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size > 1:
            if step is not None and stride != rows * step:
                return None
            step = stride if step is None else step
            rows *= size
    step = columns if step is None else step
    return (rows, step) if step >= columns else None


def _readable_rows_of(t: Optional[torch.Tensor]) -> Tuple[Optional[torch.Tensor], int]:
    """`t` and the distance of its rows; a copy where it cannot be read in place."""
    if t is None:
        return None, 0
    t = t.resolve_neg()
    found = _rows(t)
    if found is None:
        t = t.contiguous()
        found = _rows(t)
    return t, found[1]


def _row_operand(x: torch.Tensor, what: str) -> None:
    _on_gpu(x, what)
    if x.dim() < 1:
        raise ValueError(f"{what} needs rows: a tensor of one dimension at least")


def _alike(t: Optional[torch.Tensor], x: torch.Tensor, what: str) -> None:
    if t is not None and (t.shape != x.shape or t.dtype != x.dtype or t.device != x.device):
        raise ValueError(f"{what} must have the other operand's shape, type and device (no broadcasting)")


class Packed8(NamedTuple):
    """Rows in 8 bits (bs_pack8 in include/brainslug.h): `codes`, int8, of the rows' shape, `exponents`, uint8, one for every 32 neighbouring
    elements of a row."""
    codes: torch.Tensor
    exponents: torch.Tensor


def _empty_packed(x: torch.Tensor) -> Packed8:
    columns = x.shape[-1]
    return Packed8(torch.empty(x.shape, dtype=torch.int8, device=x.device),
                   torch.empty((*x.shape[:-1], -(-columns // bs.BS_PACK8_BLOCK)), dtype=torch.uint8, device=x.device))


def _packed_operand(p, what: str) -> Packed8:
    codes, exponents = p
    _row_operand(codes, what)
    if codes.dtype != torch.int8 or exponents.dtype != torch.uint8 or codes.device != exponents.device or \
            tuple(exponents.shape) != (*codes.shape[:-1], -(-codes.shape[-1] // bs.BS_PACK8_BLOCK)):
        raise ValueError(f"{what}: int8 codes and uint8 exponents, one for every 32 of a row, on one device, as pack8 gives them")
    return Packed8(codes.contiguous(), exponents.contiguous())


def _parts(t) -> tuple:
    """The tensors of an operand that is one tensor or a Packed8 (or None)."""
    return tuple(t) if isinstance(t, tuple) else (t,)


def _stream(t: torch.Tensor) -> int:
    return torch.cuda.current_stream(t.device).cuda_stream


# ------------------------------------------------------------------------------------------------ 8 bits
def _pack8_desc(x: torch.Tensor, dtype: int, step: int):
    d = bs.bs_pack8_desc()
    d.rows, d.columns = x.numel() // max(1, x.shape[-1]), x.shape[-1]
    d.x_stride, d.dtype = step, dtype
    return d


def pack8(x) -> Packed8:
    """`x` in 8 bits, 33 bytes for 32 elements of a row (its last dimension): whole numbers of a step, the power of two by which the largest of the
    32 has 63 to 126 steps.  Elements are off by half a step at most, under 0.8 % of that largest one; infinities and NaN stay."""
    native = _native_calls()
    if native:
        done = native.pack8(x)
        if done is not None:
            return Packed8(*done)
    if has_torch_function_variadic(x):
        return handle_torch_function(pack8, (x,), x)
    _refuse_recorders("pack8", x)
    with torch.no_grad():
        _row_operand(x, "pack8")
        dtype = _dtype(x, "pack8")
        x, step = _readable_rows_of(x)
        out = _empty_packed(x)
        with torch.cuda.device(x.device):
            bs.bs_pack8(_pack8_desc(x, dtype, step), x.data_ptr(), out.codes.data_ptr(), out.exponents.data_ptr(), _stream(x))
        return out


def unpack8(packed, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """The values that `packed` (a Packed8) stands for, rounded to `dtype`; types that `pack8` takes hold those of their own tensors exactly."""
    native, code = _native_calls(), _DTYPES.get(dtype)
    if native and code is not None and isinstance(packed, tuple):
        done = native.unpack8(*packed, code)
        if done is not None:
            return done
    if has_torch_function_variadic(*_parts(packed)):
        return handle_torch_function(unpack8, _parts(packed), packed, dtype)
    _refuse_recorders("unpack8")
    with torch.no_grad():
        codes, exponents = _packed_operand(packed, "unpack8")
        if code is None:
            raise TypeError(f"unpack8: float32, bfloat16 and float16 tensors, not {dtype}")
        out = torch.empty(codes.shape, dtype=dtype, device=codes.device)
        with torch.cuda.device(codes.device):
            bs.bs_unpack8(_pack8_desc(out, code, out.shape[-1]), codes.data_ptr(), exponents.data_ptr(), out.data_ptr(), _stream(codes))
        return out


def _dense_order(t: torch.Tensor) -> Optional[Tuple[int, ...]]:
    """The order of dimensions in which a tensor is one block of memory without gaps, else None."""
    order = tuple(sorted(range(t.dim()), key=lambda i: (t.stride(i), t.shape[i]), reverse=True))
    step = 1
    for i in reversed(order):
        if t.shape[i] > 1:
            if t.stride(i) != step:
                return None
            step *= t.shape[i]
    return order


def _autocasts() -> int:
    """How many autocast blocks the thread is in."""
    n = torch.autocast_increment_nesting() - 1
    torch.autocast_decrement_nesting()
    return n


class _Statistics:
    """Which of the tensors that autograd keeps, one after another, are statistics: factors of a gradient's formula that have to fit its other operands,
    where a value next to them makes another formula of it.  As far as they can be told:
    - tensors without a gradient (attention's log sums, layer normalisation's statistics; masks and constants too),
    - the second, third ... result of one of torch's own operations that is no view of its operand (group normalisation's mean and deviation),
    - tensors whose sizes are another one's with dimensions taken out, one of the last that were kept (log sums and norms along a dimension).
    What is taken for one and is none (the second of two stacked operands) only stays as precise as it was."""

    def __init__(self):
        self._sizes = collections.deque(maxlen=16)  # of the last tensors, without ones

    def begin(self) -> None:
        self._sizes.clear()

    def found(self, t: torch.Tensor) -> bool:
        if not t.requires_grad:
            return True
        sizes = tuple(t.shape)
        if 1 in sizes:
            sizes = tuple(n for n in sizes if n != 1)
        of_another, dims = False, len(sizes)
        for other in self._sizes:
            if len(other) > dims and _left_of(sizes, other):
                of_another = True
                break
        self._sizes.append(sizes)
        return of_another or (t.output_nr > 0 and not t._is_view() and not isinstance(t.grad_fn, torch.autograd.function.BackwardCFunction))


def _left_of(sizes: Tuple[int, ...], other: Tuple[int, ...]) -> bool:
    """Are `sizes` what is left of `other` when some are taken out?"""
    rest = iter(other)
    return all(n in rest for n in sizes)


class checkpoints_in_8_bits(torch.autograd.graph.saved_tensors_hooks):
    """`with checkpoints_in_8_bits(model): y = model(x)`: what autograd keeps for the backward pass in the block -- convolutions' and linear layers'
    inputs, the operands of stacks and of the functions here -- is held by `pack8` and brought back when the backward pass asks for it, so that the
    gradients are those at the values in 8 bits.

    Held so are tensors on the GPU of `pack8`'s types and sizes that have a gradient, with at least `least` elements and two dimensions, more than two
    of them in the last, dense in memory (any order of dimensions).  The others stay as they are, and so do the parameters and buffers that
    `model` (a module, or an iterable of tensors) has where the block begins, and any `nn.Parameter`, which are in use anyway; changed in place before the
    backward pass, they are refused there, as without the block.  A tensor that several nodes keep is held once for each, 1.03 bytes
    an element and node against the 2 or 4 that it takes as it is, so that the input of three projections in 16 bits takes more than without the block (nothing
    is looked up by the tensor that it was made of, whose numbers may change without a trace, by a graph's replay for one).  Under autocast, whose copies
    of the weights could not be told from activations, and where an autocast begins inside the block, it refuses.

    What is exact in 16 bits is not so in 8: an element is off by 0.8 % of the largest of 32 neighbours in memory at most.  A ReLU's gradient then takes
    the other side for elements that close to 0, the largest of a pooling window is another one where two are that close; logits lose it from their
    probabilities (keep the loss outside of the block), and numbers next to masks of the type's lowest value all they are.

    Statistics stay as they are as far as they can be told: what has no gradient (attention's log sums, constants, masks), the further results of torch's
    operations (a group normalisation's mean and deviation), and tensors whose sizes are those of one of the last sixteen with dimensions taken out (log
    sums and norms along a dimension).  A statistic that a program computes by itself, with a gradient and in sizes of its own, is held as any operand, and
    so are weights computed from parameters (casts, parametrisations).  Attention takes the exponential of its operands' products: the larger the scores, the
    coarser its gradients at operands in 8 bits."""

    def __init__(self, model, least: int = 1 << 14):
        self._model = model if isinstance(model, nn.Module) else list(model)
        # what the hooks read: not self, as graphs hold the hooks and a model may hold its graph
        self._autocasts, self._memory, self._statistics = [0], set(), _Statistics()  # _memory: where the model's tensors are
        autocasts, memory, statistics = self._autocasts, self._memory, self._statistics
        least = _integer(least, "checkpoints_in_8_bits: least", 64)

        def held(t):
            """What stands for `t` in 8 bits; None: it stays as it is."""
            kind = type(t)
            if torch.jit.is_tracing() or not t.is_cuda or not (kind is torch.Tensor or kind is nn.Parameter) or t.dtype not in _DTYPES or \
                    t.layout != torch.strided or t.dim() < 2 or t.numel() < max(1, least):  # (what is that small is no statistic's operand either)
                return None
            if statistics.found(t) or t.shape[-1] <= 2 or kind is nn.Parameter or t.untyped_storage().data_ptr() in memory:
                return None
            base = t._base
            if base is not None and isinstance(base, nn.Parameter):  # (made or moved inside the block)
                return None
            order = _dense_order(t)
            if order is None:
                return None
            t = t.detach()
            shape = [t.shape[i] for i in order]
            columns, inner = 1, len(shape)  # rows of as many dimensions as a call takes
            while inner and columns * shape[inner - 1] <= 1 << 30:
                inner -= 1
                columns *= shape[inner]
            if t.numel() // columns * -(-columns // bs.BS_PACK8_BLOCK) > 1 << 28:
                return None
            return pack8(t.permute(order).reshape(-1, columns)), t.dtype, order, shape

        def pack(t):
            if _autocasts() > autocasts[0]:  # (inside an operation autocast itself reads as switched off)
                raise RuntimeError("checkpoints_in_8_bits: no autocast inside the block")
            # (Another tensor of the same memory and versions: the very result of a node that keeps it would keep that node alive, which no collector sees.
            # Versions: where hooks are set, torch itself compares none.)
            return held(t) or (t.detach(), t._version)

        def unpack(kept):
            if len(kept) == 2:
                t, version = kept
                if t._version != version:
                    raise RuntimeError("one of the variables needed for gradient computation has been modified by an inplace operation: a tensor that "
                                       f"checkpoints_in_8_bits kept as it is, {tuple(t.shape)}, is at version {t._version}; expected version {version} instead")
                return t
            packed, dtype, order, shape = kept
            back = sorted(range(len(order)), key=order.__getitem__)
            return unpack8(packed, dtype).view(shape).permute(back)

        super().__init__(pack, unpack)

    def __enter__(self):
        if torch.is_autocast_enabled("cuda"):
            raise RuntimeError("checkpoints_in_8_bits: not under autocast")
        self._autocasts[0] = _autocasts()
        self._statistics.begin()
        tensors = (*self._model.parameters(), *self._model.buffers()) if isinstance(self._model, nn.Module) else self._model
        self._memory.clear()  # (a model that was moved or cast since has other memory)
        self._memory.update(t.untyped_storage().data_ptr() for t in tensors if not nn.parameter.is_lazy(t) and t.layout == torch.strided)
        return super().__enter__()


# ------------------------------------------------------------------------------------------------ layer normalisation
class LayerNormed(NamedTuple):
    """`y`; the sum `total` that was normalised (None without an addend); per row mean and reciprocal deviation, float32; what was normalised in 8
    bits (None: not asked for)."""
    y: torch.Tensor
    total: Optional[torch.Tensor]
    stats: Optional[torch.Tensor]
    kept: Optional[Packed8]


def _row_params(params, like: torch.Tensor, dtype: int) -> int:
    code = bs.BS_F32
    given = [p for p in params if p is not None]
    for p in given:
        if tuple(p.shape) != (like.shape[-1],) or not p.is_contiguous() or p.is_neg() or p.device != like.device:
            raise ValueError("layer_norm: weight and bias hold one element a feature, contiguous (no negated view), on the rows' device")
        code = _dtype(p, "layer_norm")
        if code not in (bs.BS_F32, dtype) or p.dtype != given[0].dtype:
            raise TypeError("layer_norm: weight and bias are both float32 or both of the rows' type")
    return code


def _layer_norm_desc(like: torch.Tensor, dtype: int, weight, bias, eps: float):
    d = bs.bs_layer_norm_desc()
    d.rows, d.features = like.numel() // max(1, like.shape[-1]), like.shape[-1]
    d.dtype, d.param_dtype, d.eps = dtype, _row_params((weight, bias), like, dtype), float(eps)
    return d


def _run_layer_norm(x, weight, bias, addend, eps, checkpoint, keep_stats, recorded=False) -> LayerNormed:
    """`recorded`: called by the node that a recorder sees."""
    native = _native_calls()
    if native:
        done = native.layer_norm(x, weight, bias, addend, eps, checkpoint, keep_stats)
        if done is not None:
            return LayerNormed(*done[:3], Packed8(*done[3:]) if checkpoint else None)
    if not recorded:
        if has_torch_function_variadic(x, weight, bias, addend):  # (layer_norm has looked already)
            return handle_torch_function(layer_norm_forward, (x, weight, bias, addend), x, weight, bias, addend, eps, checkpoint)
        if torch.jit.is_tracing() and not keep_stats:
            r = _LayerNorm.apply(x, weight, bias, addend, eps, checkpoint)
            return LayerNormed(*(r if addend is not None else (r, None)), None, None)
        _refuse_recorders("layer_norm", x, weight, bias, addend)
    with torch.no_grad():
        _row_operand(x, "layer_norm")
        _alike(addend, x, "layer_norm: addend")
        d = _layer_norm_desc(x, _dtype(x, "layer_norm"), weight, bias, eps)
        x, d.x_stride = _readable_rows_of(x)
        addend, d.addend_stride = _readable_rows_of(addend)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        total = torch.empty(x.shape, dtype=x.dtype, device=x.device) if addend is not None else None
        stats = torch.empty((*x.shape[:-1], 2), dtype=torch.float32, device=x.device) if keep_stats else None
        kept = _empty_packed(x) if checkpoint else None
        with torch.cuda.device(x.device):
            bs.bs_layer_norm(d, x.data_ptr(), _ptr(addend), _ptr(weight), _ptr(bias), y.data_ptr(), _ptr(total), _ptr(stats),
                             *((0, 0) if kept is None else (kept.codes.data_ptr(), kept.exponents.data_ptr())), _stream(x))
        return LayerNormed(y, total, stats, kept)


def layer_norm_forward(x, weight=None, bias=None, addend=None, eps: float = 1e-5, checkpoint: bool = False) -> LayerNormed:
    """Rows (the last dimension of `x`) plus those of `addend`, the sum `total` rounded to x's type, normalised: (total - mean) / sqrt(var + eps) *
    weight + bias, and what `layer_norm_backward` needs; `checkpoint`: that too in 8 bits, `kept`.  Rows may lie further apart than they are long
    (other memory orders are copied first)."""
    return _run_layer_norm(x, weight, bias, addend, eps, checkpoint, True)


def layer_norm_backward(x, stats, grad, weight=None, bias=None, grad_total=None, need=(True, True, True)):
    """`(grad_x, grad_weight, grad_bias)`: from what was normalised -- `x`, or `total` where there was an addend, or `kept` -- its `stats`, the gradient
    `grad` of y and `grad_total` of total (None: zero).  grad_x is the gradient of x and of the addend alike; `need` says which are wanted (those of
    absent parameters are None)."""
    native = _native_calls()
    if native:
        done = native.layer_norm_backward(*(x if isinstance(x, tuple) else (x, None)), stats, grad, weight, bias, grad_total, need[0] | need[1] << 1 | need[2] << 2)
        if done is not None:
            return done
    tensors = (*_parts(x), stats, grad, weight, bias, grad_total)
    if has_torch_function_variadic(*tensors):
        return handle_torch_function(layer_norm_backward, tensors, x, stats, grad, weight, bias, grad_total, need)
    _refuse_recorders("layer_norm_backward", *tensors)
    with torch.no_grad():
        _row_operand(grad, "layer_norm_backward")
        held = _packed_operand(x, "layer_norm_backward") if isinstance(x, tuple) else None
        if held is None:
            _alike(x, grad, "layer_norm_backward: x")
        elif held.codes.shape != grad.shape or held.codes.device != grad.device:
            raise ValueError("layer_norm_backward: the codes must have the gradient's shape and device")
        _alike(grad_total, grad, "layer_norm_backward: grad_total")
        if tuple(stats.shape) != (*grad.shape[:-1], 2) or stats.dtype != torch.float32 or stats.device != grad.device:
            raise ValueError("layer_norm_backward: stats must be those of layer_norm_forward")
        stats = stats.contiguous()
        d = _layer_norm_desc(grad, _dtype(grad, "layer_norm_backward"), weight, bias, 0.0)
        if held is None:
            x, d.x_stride = _readable_rows_of(x)
        grad, d.grad_y_stride = _readable_rows_of(grad)
        grad_total, d.grad_total_stride = _readable_rows_of(grad_total)
        gx = torch.empty(grad.shape, dtype=grad.dtype, device=grad.device) if need[0] else None
        gw, gb = (torch.empty(p.shape, dtype=p.dtype, device=p.device) if wanted and p is not None else None for wanted, p in zip(need[1:], (weight, bias)))
        n = bs.bs_layer_norm_workspace_bytes(d) if gw is not None or gb is not None else 0
        ws = _workspace(n, grad)
        with torch.cuda.device(grad.device):
            bs.bs_layer_norm_backward(d, _ptr(x) if held is None else 0, *((0, 0) if held is None else (held.codes.data_ptr(), held.exponents.data_ptr())),
                                      stats.data_ptr(), _ptr(weight), grad.data_ptr(), _ptr(grad_total), _ptr(gx), _ptr(gw), _ptr(gb), _ptr(ws), n,
                                      _stream(grad))
        return gx, gw, gb


class _LayerNorm(torch.autograd.Function):
    """Keeps what was normalised, as it is or in 8 bits, the statistics and the parameters."""

    @staticmethod
    def forward(ctx, x, weight, bias, addend, eps, checkpoint):
        r = _run_layer_norm(x, weight, bias, addend, eps, checkpoint, True, recorded=True)
        kept = r.kept if checkpoint else (x if addend is None else r.total, None)
        ctx.save_for_backward(*kept, r.stats, weight, bias)
        ctx.set_materialize_grads(False)
        return r.y if addend is None else (r.y, r.total)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad, grad_total=None):
        kept, exponents, stats, weight, bias = ctx.saved_tensors
        need = ctx.needs_input_grad
        if grad is None:
            return grad_total, None, None, grad_total if need[3] else None, None, None
        gx, gw, gb = layer_norm_backward(kept if exponents is None else Packed8(kept, exponents), stats, grad, weight, bias, grad_total,
                                         (need[0] or need[3], need[1], need[2]))
        return gx if need[0] else None, gw, gb, gx if need[3] else None, None, None


def layer_norm(x, weight=None, bias=None, addend=None, eps: float = 1e-5, checkpoint: bool = False):
    """The rows of `x` normalised, weight and bias per feature; with an `addend` `(y, total)`: the rows of total = x + addend normalised, and total,
    which a residual network adds to next.  Differentiable in every tensor.  `checkpoint`: autograd keeps the normalised rows in 8 bits instead of
    in their own type, and the gradients are those at the values these stand for.  See `layer_norm_forward`."""
    if has_torch_function_variadic(x, weight, bias, addend):
        return handle_torch_function(layer_norm, (x, weight, bias, addend), x, weight, bias, addend, eps, checkpoint)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, weight, bias, addend)):
        return _LayerNorm.apply(x, weight, bias, addend, eps, checkpoint)
    r = _run_layer_norm(x, weight, bias, addend, eps, False, False)
    return r.y if addend is None else (r.y, r.total)


class LayerNorm(nn.LayerNorm):
    """`nn.LayerNorm` over the last dimension (same parameters, same state dict) with an optional addition in front: `m(x)`, or
    `y, total = m(x, addend)`.  `checkpoint`: what its backward pass needs is kept in 8 bits."""

    def __init__(self, features: int, eps: float = 1e-5, elementwise_affine: bool = True, bias: bool = True, checkpoint: bool = False, device=None, dtype=None):
        super().__init__(_integer(features, "LayerNorm: features", 64), eps, elementwise_affine, bias, device=device, dtype=dtype)
        self.checkpoint = checkpoint

    def forward(self, x: torch.Tensor, addend: Optional[torch.Tensor] = None):
        if isinstance(x, torch.Tensor) and x.shape[-1] != self.normalized_shape[0]:  # (not what stands for one where a recorder looks)
            raise ValueError(f"LayerNorm: rows of {x.shape[-1]} features, not {self.normalized_shape[0]}")
        return layer_norm(x, self.weight, self.bias, addend, self.eps, self.checkpoint)

    def extra_repr(self) -> str:
        return super().extra_repr() + f", checkpoint={self.checkpoint}"


# ------------------------------------------------------------------------------------------------ activations
class Activated(NamedTuple):
    """`y`; x and gate in 8 bits (None: not asked for, no gate)."""
    y: torch.Tensor
    x: Optional[Packed8]
    gate: Optional[Packed8]


def _activate_desc(like: torch.Tensor, dtype: int, activation: str):
    if activation not in ACTIVATIONS:
        raise ValueError(f"activate: activation {activation!r}, not one of {', '.join(ACTIVATIONS)}")
    d = bs.bs_activate_desc()
    d.rows, d.columns = like.numel() // max(1, like.shape[-1]), like.shape[-1]
    d.dtype, d.activation = dtype, ACTIVATIONS[activation]
    return d


def _run_activate(x, activation, gate, checkpoint, recorded=False, traced=False) -> Activated:
    """`recorded`: called by the node that a recorder sees; `traced`: make that node where torch.jit.trace records."""
    native, act = _native_calls(), ACTIVATIONS.get(activation)
    if native and act is not None:
        done = native.activate(x, act, gate, checkpoint)
        if done is not None:
            return Activated(done[0], Packed8(*done[1:3]) if checkpoint else None, Packed8(*done[3:]) if checkpoint and gate is not None else None)
    if not recorded:
        if has_torch_function_variadic(x, gate):  # (activate has looked already)
            return handle_torch_function(activate_forward, (x, gate), x, activation, gate, checkpoint)
        if traced and torch.jit.is_tracing():
            return Activated(_Activate.apply(x, gate, activation, checkpoint), None, None)
        _refuse_recorders("activate", x, gate)
    with torch.no_grad():
        _row_operand(x, "activate")
        _alike(gate, x, "activate: gate")
        d = _activate_desc(x, _dtype(x, "activate"), activation)
        x, d.x_stride = _readable_rows_of(x)
        gate, d.gate_stride = _readable_rows_of(gate)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        held = tuple(_empty_packed(x) if checkpoint and t is not None else None for t in (x, gate))
        with torch.cuda.device(x.device):
            bs.bs_activate(d, x.data_ptr(), _ptr(gate), y.data_ptr(), *(_ptr(t) for h in held for t in (h or (None, None))), _stream(x))
        return Activated(y, *held)


def activate_forward(x, activation: str = "silu", gate=None, checkpoint: bool = False) -> Activated:
    """act(x) * gate, or act(x); `checkpoint`: x and gate too in 8 bits.  A ReLU of NaN is 0, where torch's is NaN.  Rows (the last dimension) of either
    operand may lie further apart than they are long, as in the halves of one product's result (other memory orders are copied first)."""
    return _run_activate(x, activation, gate, checkpoint)


def activate_backward(x, grad, activation: str = "silu", gate=None, need=(True, True)):
    """`(grad_x, grad_gate)` from the gradient `grad` of `activate_forward`'s result; x and gate both as they were or both in 8 bits (Packed8).
    `need` says which are wanted (that of an absent gate is None)."""
    native, act = _native_calls(), ACTIVATIONS.get(activation)
    if native and act is not None:
        done = native.activate_backward(*(x if isinstance(x, tuple) else (x, None)), grad, act, *(gate if isinstance(gate, tuple) else (gate, None)),
                                        need[0] | need[1] << 1)
        if done is not None:
            return done
    tensors = (*_parts(x), grad, *_parts(gate))
    if has_torch_function_variadic(*tensors):
        return handle_torch_function(activate_backward, tensors, x, grad, activation, gate, need)
    _refuse_recorders("activate_backward", *tensors)
    with torch.no_grad():
        _row_operand(grad, "activate_backward")
        d = _activate_desc(grad, _dtype(grad, "activate_backward"), activation)
        held = isinstance(x, tuple)
        if gate is not None and isinstance(gate, tuple) != held:
            raise ValueError("activate_backward: x and gate both as tensors or both in 8 bits")
        if held:
            x, gate = (_packed_operand(t, "activate_backward") if t is not None else None for t in (x, gate))
            if any(t is not None and (t.codes.shape != grad.shape or t.codes.device != grad.device) for t in (x, gate)):
                raise ValueError("activate_backward: the codes must have the gradient's shape and device")
            pointers = [0, *(_ptr(t) for t in x), 0, *(_ptr(t) for t in gate or (None, None))]
        else:
            _alike(x, grad, "activate_backward: x")
            _alike(gate, grad, "activate_backward: gate")
            x, d.x_stride = _readable_rows_of(x)
            gate, d.gate_stride = _readable_rows_of(gate)
            pointers = [x.data_ptr(), 0, 0, _ptr(gate), 0, 0]
        grad, d.grad_y_stride = _readable_rows_of(grad)
        gx = torch.empty(grad.shape, dtype=grad.dtype, device=grad.device) if need[0] else None
        gg = torch.empty(grad.shape, dtype=grad.dtype, device=grad.device) if need[1] and gate is not None else None
        with torch.cuda.device(grad.device):
            bs.bs_activate_backward(d, *pointers, grad.data_ptr(), _ptr(gx), _ptr(gg), _stream(grad))
        return gx, gg


class _Activate(torch.autograd.Function):
    """Keeps x and gate, as they are or in 8 bits."""

    @staticmethod
    def forward(ctx, x, gate, activation, checkpoint):
        r = _run_activate(x, activation, gate, checkpoint, recorded=True)
        kept = (*r.x, *(r.gate or (None, None))) if checkpoint else (x, None, gate, None)
        ctx.save_for_backward(*kept)
        ctx.activation = activation
        return r.y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        x, x_exponents, gate, gate_exponents = ctx.saved_tensors
        if x_exponents is not None:
            x, gate = Packed8(x, x_exponents), None if gate is None else Packed8(gate, gate_exponents)
        return (*activate_backward(x, grad, ctx.activation, gate, ctx.needs_input_grad[:2]), None, None)


def activate(x, activation: str = "silu", gate=None, checkpoint: bool = False):
    """act(x) * gate, or act(x) without a gate; differentiable in both.  `checkpoint`: autograd keeps x and gate in 8 bits instead of in their own
    type, and the gradients are those at the values these stand for.  See `activate_forward`."""
    if has_torch_function_variadic(x, gate):
        return handle_torch_function(activate, (x, gate), x, activation, gate, checkpoint)
    if torch.is_grad_enabled() and (x.requires_grad or (gate is not None and gate.requires_grad)):
        return _Activate.apply(x, gate, activation, checkpoint)
    return _run_activate(x, activation, gate, False, traced=True).y
