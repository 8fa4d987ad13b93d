"""The most tokens and the largest grids of the experts' calls."""
import ctypes as C

import pytest
import torch

import paper_2412_14590_amd as mx
from paper_2412_14590_amd import binding


def test_grids_that_cannot_be_launched_are_refused():
    # 1024 experts with a row each, 2^23 channels: 2^26 tiles.  (Refused: nothing is launched, whether there is a GPU or not.)
    e, L, address = binding._Epilogue(None, None, 0, 0), mx.lib(), 0x10000000
    d = binding._desc(1024, 128, 1 << 23, 0)
    y = 0x7f0000000000
    assert L.mixllm_experts_linear(C.byref(d), 1024, address, address, address, address, address, 1, C.byref(e), y, None) == -2
    assert L.mixllm_experts_linear_fp16(C.byref(d), 1024, address, address, address, address, 1, C.byref(e), y, address, 1 << 24, None) == -2


@pytest.mark.gpu
@pytest.mark.parametrize("T", [(1 << 23) + 3, 1 << 24])
def test_the_sum_of_the_most_tokens(T):
    """Each token's row is that of its index modulo 2000, the residual its index modulo 7: halves of whole numbers, exact in fp16."""
    y = torch.arange(2000, device="cuda").half()[:, None].contiguous()
    slots = torch.arange(T, device="cuda").remainder(2000).int()[:, None].contiguous()
    route = mx.Route(None, torch.full((T, 1), 0.5, device="cuda"), None, None, slots)
    residual = torch.arange(T, device="cuda").remainder(7).half()[:, None].contiguous()
    want = slots.half() * 0.5
    assert torch.equal(mx.experts_combine(y, route), want)
    assert torch.equal(mx.experts_combine(y, route, residual), want + residual)
