"""Group normalisation with an activation (channels last) and log probabilities of given classes, as cases to be measured.

`group_norm`: x of N images with C channels in G groups, channels contiguous in memory; normalised over each image's group, weight and bias
per channel, an optional residual operand added, then the activation.  `log_probs`: rows of logits; the log probability of each row's given
class, the entropy of the row's distribution and its top alternatives.  Mode "run" is a forward pass, mode "train" a forward and a backward
pass that returns the result and every gradient.

A case of group_norm: op, n, c, h, w, groups, act, residual, dtype, mode.  A case of log_probs: op, rows, classes, top, dtype, mode.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
IGNORED = -100  # a row without a given class


def _norm(name, shape, groups, act, dtype="f32", mode="run", residual=False):
    n, c, h, w = shape
    case = {"op": "group_norm", "n": n, "c": c, "h": h, "w": w, "groups": groups, "act": act, "residual": residual, "dtype": dtype, "mode": mode}
    return {"name": name, **case} if name else case


def _head(name, rows, classes, top, dtype="f32", mode="run"):
    case = {"op": "log_probs", "rows": rows, "classes": classes, "top": top, "dtype": dtype, "mode": mode}
    return {"name": name, **case} if name else case


def listed():
    return [
        # one small image: serving a request, a call whose time is its launches
        _norm("norm_run_tiny_f32", (1, 16, 32, 32), 4, "relu"),
        # the end of a residual block, batch 64, 16-bit: the commonest call of a residual network
        _norm("norm_run_tail_bf16", (64, 256, 56, 56), 32, "relu", "bf16", residual=True),
        # a middle stage of a network that is served in small batches
        _norm("norm_run_mid_f16", (8, 512, 28, 28), 32, "silu", "f16"),
        # the first stage in training, float32: two channels in a group, long planes, the most bytes of all
        _norm("norm_train_stem_f32", (64, 64, 112, 112), 32, "silu", "f32", "train"),
        # the end of a residual block in training, 16-bit
        _norm("norm_train_tail_bf16", (64, 256, 56, 56), 32, "silu", "bf16", "train", residual=True),
        # odd planes, groups of five channels: scaled networks
        _norm("norm_train_odd_f16", (5, 60, 37, 29), 12, "gelu", "f16", "train"),
        # the last stage of a network, a small batch in training: short sums, many channels
        _norm("norm_train_last_bf16", (4, 2048, 7, 7), 32, "silu", "bf16", "train"),
        # one row over a large vocabulary: the answer of one decoding step
        _head("head_run_token_bf16", 1, 131072, 20, "bf16"),
        # a batch of images over a classifier's 1000 classes
        _head("head_run_classes_f32", 256, 1000, 5),
        # scoring a text: many rows, a vocabulary of odd size, so that rows begin anywhere
        _head("head_run_odd_f16", 777, 50021, 20, "f16"),
        # the loss of a training step over a large batch of rows
        _head("head_train_bf16", 8192, 32000, 0, "bf16", "train"),
        # the same in float32 at odd sizes, with the row's best classes
        _head("head_train_odd_f32", 1001, 10007, 5, "f32", "train"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    mode, dtype = rng.choice(["run", "train"]), rng.choice(list(DTYPES))
    if rng.random() < 0.5:
        groups = rng.choice([1, 2, 4, 8, 16, 32, 32, 32, 3, 12])
        per = _log(rng, 1, 64) if rng.random() < 0.4 else 2 ** rng.randint(0, 6)  # channels of a group
        per = max(1, min(per, 2048 // groups))
        h = _log(rng, 1, 160)
        w = h if rng.random() < 0.6 else _log(rng, 1, 160)
        if per * h * w < 16:  # the gradient through the statistics of a few cells is a difference of nearly equal numbers
            h = w = 4
        n = max(1, min(_log(rng, 1, 64), (48 << 20) // (groups * per * h * w)))
        # a ReLU's gradient jumps at 0, where a rounding decides: in training the smooth activations
        act = rng.choice(["identity", "silu", "gelu"] + ["relu"] * (2 * (mode == "run")))
        return _norm(None, (n, groups * per, h, w), groups, act, dtype, mode, rng.random() < 0.4)
    classes = _log(rng, 10, 160000)
    rows = max(1, min(_log(rng, 1, 8192), (200 << 20) // classes))
    return _head(None, rows, classes, min(classes // 2, rng.choice([0, 1, 5, 20, 32])), dtype, mode)


def _generator(case, seed):
    return torch.Generator(device="cuda").manual_seed(seed * 1000003 + 17)


def _norm_tensors(case, seed):
    """x with a mean and a spread of its own in every channel, as behind a convolution; weight near 1, bias near 0."""
    g, dt = _generator(case, seed), DTYPES[case["dtype"]]
    n, c, h, w = case["n"], case["c"], case["h"], case["w"]

    def make(scale=None, shift=None):
        t = torch.randn(n, h, w, c, generator=g, device="cuda")
        if scale is not None:
            t = t.mul_(scale).add_(shift)
        return t.to(dt).permute(0, 3, 1, 2)

    x = make(torch.rand(c, generator=g, device="cuda") + 0.5, torch.randn(c, generator=g, device="cuda") * 0.5)
    weight = torch.rand(c, generator=g, device="cuda") + 0.5
    bias = torch.randn(c, generator=g, device="cuda") * 0.1
    return {"x": x, "weight": weight, "bias": bias, "residual": make() if case["residual"] else None, "grad": make() if case["mode"] == "train" else None}


def _head_tensors(case, seed):
    """Logits with some clear favourites; the last few columns pad the vocabulary and are masked; a few rows have no given class."""
    g, dt = _generator(case, seed), DTYPES[case["dtype"]]
    rows, classes = case["rows"], case["classes"]
    logits = torch.randn(rows, classes, generator=g, device="cuda").mul_(2.5)
    targets = torch.randint(0, classes - classes // 50, (rows,), generator=g, device="cuda")
    known = torch.rand(rows, generator=g, device="cuda")
    bonus = torch.rand(rows, 1, generator=g, device="cuda") * 12
    logits.scatter_add_(1, targets[:, None], bonus)
    logits = logits.to(dt)
    if classes >= 50:
        logits[:, classes - classes // 50:] = -math.inf
    targets = torch.where(known < 0.05, IGNORED, targets) if rows > 1 else targets
    out = {"logits": logits, "targets": targets, "grad_logp": None, "grad_entropy": None}
    if case["mode"] == "train":
        out["grad_logp"] = torch.rand(rows, generator=g, device="cuda").add_(0.5).mul_(-1)
        out["grad_entropy"] = torch.randn(rows, generator=g, device="cuda") * 0.1
    return out


def prepare(case, seed):
    return {"case": case, **(_norm_tensors if case["op"] == "group_norm" else _head_tensors)(case, seed)}


# ------------------------------------------------------------------------------------------------ plain forms
def _activation(act, z):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return z * 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(act, z):
    """Derivative of the activation."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return (z > 0).float() if act == "relu" else torch.ones_like(z)


def _plain_norm(s):
    case = s["case"]
    n, c, h, w = case["n"], case["c"], case["h"], case["w"]
    shape = (n, h * w, case["groups"], c // case["groups"])

    def rows(t):  # pixels x groups x channels of a group, in 32 bits
        return t.permute(0, 2, 3, 1).float().reshape(shape)

    def back(t):
        return t.reshape(n, h, w, c).to(DTYPES[case["dtype"]]).permute(0, 3, 1, 2)

    weight, bias = s["weight"].view(shape[2:]), s["bias"].view(shape[2:])
    x = rows(s["x"])
    d = x - x.mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt((d * d).mean((1, 3), keepdim=True) + EPS)
    xh = d * rstd
    z = xh * weight + bias
    if s["residual"] is not None:
        z = z + rows(s["residual"])
    y = back(_activation(case["act"], z))
    if case["mode"] == "run":
        return {"y": y}
    dz = rows(s["grad"]) * _slope(case["act"], z)
    dxh = dz * weight
    dx = rstd * (dxh - dxh.mean((1, 3), keepdim=True) - xh * (dxh * xh).mean((1, 3), keepdim=True))
    out = {"y": y, "grad_x": back(dx), "grad_weight": (dz * xh).sum((0, 1)).view(c), "grad_bias": dz.sum((0, 1)).view(c)}
    return {**out, "grad_residual": back(dz)} if s["residual"] is not None else out


def _plain_head(s):
    case = s["case"]
    logits, targets = s["logits"].float(), s["targets"]
    d = logits - logits.amax(1, keepdim=True)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    logp = d - torch.log(total)
    p = e / total
    plogp = torch.where(p > 0, p * logp, 0.0)
    entropy = -plogp.sum(1)
    given = targets != IGNORED
    at = torch.where(given, targets, 0)[:, None]
    out = {"logp": torch.where(given, logp.gather(1, at)[:, 0], 0.0), "entropy": entropy}
    if case["top"]:
        # one number a class that orders by value and then by the lower index: the bits of a float, ordered like integers, above the index
        bits = (logits + 0.0).view(torch.int32).long()
        bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
        key = bits * 2 ** 20 + torch.arange(case["classes"] - 1, -1, -1, device=logits.device)
        index = case["classes"] - 1 - torch.topk(key, case["top"], 1).values % 2 ** 20
        out.update(top_logp=logp.gather(1, index), top_index=index.int())
    if case["mode"] == "train":
        g, h = torch.where(given, s["grad_logp"], 0.0)[:, None], s["grad_entropy"][:, None]
        grad = -g * p - h * (plogp + p * entropy[:, None])
        grad.scatter_add_(1, at, g)
        out["grad_logits"] = grad.to(DTYPES[case["dtype"]])
    return out


# ------------------------------------------------------------------------------------------------ the framework's operators
def _own_norm(s):
    from paper_1804_08378_amd import functional as F

    case = s["case"]
    args = (s["weight"], s["bias"], s["residual"], case["act"], EPS)
    if case["mode"] == "run":
        return {"y": F.group_norm(s["x"], case["groups"], *args)}
    y, stats = F.group_norm_forward(s["x"], case["groups"], *args)
    gx, gw, gb, gr = F.group_norm_backward(s["x"], stats, s["grad"], case["groups"], *args)
    out = {"y": y, "grad_x": gx, "grad_weight": gw, "grad_bias": gb}
    return {**out, "grad_residual": gr} if s["residual"] is not None else out


def _own_head(s):
    from paper_1804_08378_amd import functional as F

    case = s["case"]
    r = F.log_probs_forward(s["logits"], s["targets"], top=case["top"], ignore_index=IGNORED)
    out = {"logp": r.logp, "entropy": r.entropy}
    if case["top"]:
        out.update(top_logp=r.top_logp, top_index=r.top_index)
    if case["mode"] == "train":
        out["grad_logits"] = F.log_probs_backward(s["logits"], s["targets"], r.lse, r.entropy, s["grad_logp"], s["grad_entropy"], ignore_index=IGNORED)
    return out


def run(state):
    if state["case"]["op"] == "group_norm":
        return _own_norm(state) if own else _plain_norm(state)
    return _own_head(state) if own else _plain_head(state)


def work(case):
    """Inputs read once, results written once.  Operations per element: statistics 4, normalisation and affine 4, activation 4, residual 1;
    the backward pass about twice that.  Logits: maximum, difference, exponential, two sums; the gradient 6 more."""
    es, train = ES[case["dtype"]], case["mode"] == "train"
    if case["op"] == "group_norm":
        cells, c, r = case["n"] * case["c"] * case["h"] * case["w"], case["c"], int(case["residual"])
        tensors = (4 + 2 * r) if train else (2 + r)
        return {"bytes": cells * es * tensors + c * 4 * (4 if train else 2), "flops": cells * ((12 + r) * (3 if train else 1))}
    rows, classes, top = case["rows"], case["classes"], case["top"]
    moved = rows * classes * es * (2 if train else 1) + rows * (8 + 8 + 8 * top + (8 if train else 0))
    return {"bytes": moved, "flops": rows * classes * (12 if train else 6)}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_norm(case, s):
    train = case["mode"] == "train"
    leaves = {k: s[k].double().contiguous().requires_grad_(train) for k in ("x", "weight", "bias", "residual") if s[k] is not None}
    with torch.set_grad_enabled(train):
        x = leaves["x"].reshape(case["n"], case["groups"], -1)
        var, mean = torch.var_mean(x, 2, correction=0, keepdim=True)
        z = ((x - mean) / (var + EPS).sqrt()).view_as(leaves["x"]) * leaves["weight"].view(1, -1, 1, 1) + leaves["bias"].view(1, -1, 1, 1)
        z = z + leaves["residual"] if case["residual"] else z
        y = {"identity": lambda v: v, "relu": lambda v: v.clamp(min=0), "silu": lambda v: v * torch.sigmoid(v),
             "gelu": lambda v: v * torch.special.ndtr(v)}[case["act"]](z)
    if not train:
        return {"y": y}
    grads = torch.autograd.grad(y, list(leaves.values()), s["grad"].double().contiguous())
    names = {"x": "grad_x", "weight": "grad_weight", "bias": "grad_bias", "residual": "grad_residual"}
    return {"y": y.detach(), **{names[k]: v for k, v in zip(leaves, grads)}}


def _exact_head(case, s):
    train = case["mode"] == "train"
    logits = s["logits"].double().requires_grad_(train)
    given = s["targets"] != IGNORED
    with torch.set_grad_enabled(train):
        logp = logits - torch.logsumexp(logits, 1, keepdim=True)
        finite = torch.isfinite(logp)
        entropy = -(torch.exp(logp) * torch.where(finite, logp, 0.0)).sum(1)
        mine = logp.gather(1, s["targets"].clamp(min=0)[:, None])[:, 0]
        mine = torch.where(given, mine, 0.0)
    out = {"logp": mine.detach(), "entropy": entropy.detach()}
    if case["top"]:
        values, index = torch.sort(logp.detach(), dim=1, descending=True, stable=True)
        out.update(top_logp=values[:, :case["top"]], top_index=index[:, :case["top"]].int())
    if train:
        out["grad_logits"] = torch.autograd.grad([mine, entropy], logits, [s["grad_logp"].double(), s["grad_entropy"].double()])[0]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_norm(case, s) if case["op"] == "group_norm" else _exact_head(case, s)
