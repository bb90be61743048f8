"""What training a network from scratch needs beside its stacks, on torch tensors: group normalisation with a residual operand and an
activation (channels last), and the log probabilities at a classifier's end, both with their gradients.

`group_norm` and `log_probs` are differentiable functions; `GroupNormAct` is the normalisation as a module.  The `_forward` / `_backward`
pairs are the single passes, for programs that keep their own tape.  Everything runs on the current stream of the tensors' device through the
C ABI (`bs_group_norm`, `bs_log_probs` in include/brainslug.h); there is no fallback: tensors the library cannot take raise.  What overrides
torch's functions overrides these too: `torch.fx` records a call of one of them as one node, so `optimize_graph` and `capture` take models with them.
"""
from __future__ import annotations

import ctypes as C
import operator
from typing import NamedTuple, Optional, Tuple

import torch
from torch import nn
from torch.autograd import forward_ad
from torch.overrides import handle_torch_function, has_torch_function_variadic

from . import brainslug as bs

__all__ = ["group_norm", "group_norm_forward", "group_norm_backward", "GroupNormAct", "log_probs", "log_probs_forward", "log_probs_backward",
           "LogProbs", "ACTIVATIONS"]

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
                             "bs_log_probs_backward")
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
        raise RuntimeError(f"{what}: torch.jit.trace records calls of group_norm and log_probs, not the single passes, nor calls with out")
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
        if tuple(p.shape) != (x.shape[1],) or not p.is_contiguous() or p.device != x.device:
            raise ValueError("group_norm: weight and bias hold one element a channel, contiguous, on x's device")
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
        if out.shape != x.shape or out.dtype != x.dtype or out.device != x.device or step is None:
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
            given.append(t.contiguous() if t is not None else None)
        lse, entropy, grad_logp, grad_entropy = given
        d.lse_bytes = lse.element_size()
        if out is None:
            out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        elif out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device or _row_stride(out) is None:
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
