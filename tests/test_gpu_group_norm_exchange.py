"""The memory that the parts of an image hand sums through: calls one behind the other, those whose work-groups wait and those whose do not."""
import ctypes

import pytest
import torch

from paper_1804_08378_amd import brainslug as bs
from paper_1804_08378_amd import functional as F
from test_gpu_group_norm import DTYPES, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(2, 64, 60, 60, 32), (5, 256, 56, 56, 8), (1, 96, 100, 75, 32)])
def test_calls_follow_each_other_through_one_memory(shape, dtype):
    """Three tensors in turn, forward and backward, every second call without waiting, none waited for by the host: no word of one call is
    taken by the next, and nothing is left at the end."""
    memory = torch.zeros(bs.BS_GROUP_NORM_EXCHANGE_BYTES // 8, dtype=torch.int64, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    n, c, h, w, groups = shape
    sets, want = [], []
    for seed in range(3):
        x, weight, bias, res, dy = tensors(shape, dtype, seed, True, mean=0.5 * seed)
        d = F._norm_operands(x, groups, weight, bias, res, "silu", 1e-5, dy)[0]
        d.exchange, d.exchange_bytes = memory.data_ptr(), 8 * memory.numel()
        size = max(bs.bs_group_norm_workspace_bytes(d, b) for b in (False, True))
        sets.append((d, x, weight, bias, res, dy, torch.empty(size, dtype=torch.uint8, device="cuda"), size))
        y, stats = F.group_norm_forward(x, groups, weight, bias, res, "silu")
        gx, gw, gb, gr = F.group_norm_backward(x, stats, dy, groups, weight, bias, res, "silu")
        want.append((y, stats, gx, gr, gw, gb))
    outs = []
    for i in range(24):
        d, x, weight, bias, res, dy, ws, size = sets[i % 3]
        out = [torch.empty_like(t) for t in want[i % 3]]
        y, st, gx, gr, gw, gb = (t.data_ptr() for t in out)
        d.wait_polls = -1 if i % 2 else 0
        bs.bs_group_norm(d, x.data_ptr(), res.data_ptr(), weight.data_ptr(), bias.data_ptr(), y, st, ws.data_ptr(), size, stream)
        d.wait_polls = -1 if i // 2 % 2 else 0
        bs.bs_group_norm_backward(d, x.data_ptr(), res.data_ptr(), weight.data_ptr(), bias.data_ptr(), st, dy.data_ptr(), gx, gr, gw, gb,
                                  ws.data_ptr(), size, stream)
        outs.append(out)
    torch.cuda.synchronize()
    assert not memory.any()
    for i, out in enumerate(outs):
        assert all(torch.equal(a, b) for a, b in zip(out, want[i % 3])), i


def test_streams_that_torch_did_not_make():
    """A handle from elsewhere keeps no memory: it may stand for several streams, or for another one tomorrow.  Results are the same bits."""
    hip = ctypes.CDLL("libamdhip64.so")
    x, weight, bias, res, dy = tensors((2, 64, 60, 60, 8), "bf16", 0, True)
    args = (8, weight, bias, res, "silu")

    def both():
        y, stats = F.group_norm_forward(x, *args)
        return (y, stats, *F.group_norm_backward(x, stats, dy, *args))

    want = both()
    torch.cuda.synchronize()
    handles, kept = [], []
    for _ in range(3):
        handle = ctypes.c_void_p()
        assert hip.hipStreamCreate(ctypes.byref(handle)) == 0
        handles.append(handle)
        before = torch.cuda.memory_allocated()
        with torch.cuda.stream(torch.cuda.ExternalStream(handle.value)):
            got = both()
            torch.cuda.current_stream().synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del got
        kept.append(torch.cuda.memory_allocated() - before)
    for handle in handles:
        assert hip.hipStreamDestroy(handle) == 0
    assert kept == [0, 0, 0]


def test_streams_of_torch_keep_the_memory_once():
    """The default stream and a stream of torch's pool, called again: nothing more is kept."""
    x = tensors((2, 64, 60, 60, 8), "bf16", 0, False)[0]
    for stream in (torch.cuda.default_stream(), torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            F.group_norm(x, 8)
            before = torch.cuda.memory_allocated()
            F.group_norm(x, 8)
            assert torch.cuda.memory_allocated() == before
    torch.cuda.synchronize()
