"""Operators next to the linear, without a GPU: results may lie on the residual, on nothing else that a call reads; and grids beyond a
launch."""
import ctypes as C

import pytest

import paper_2412_14590_amd as mx
from paper_2412_14590_amd import binding

FAKE = 0x100000   # never dereferenced: without a GPU a call that passes the checks ends in EHIP
W = 0x90000000    # weights, lists, workspace: apart from the rest
EINVAL, EHIP = -1, -4


def epilogue(M, N, gated, x, y, residual, codes, K=256):
    e = binding._Epilogue(None, residual, 0, gated)
    d = binding._desc(M, K, N, 8)
    L = mx.lib()
    if codes:
        return L.mixllm_mixed_linear_epilogue(C.byref(d), x, W, W, W, W, W, W, W, C.byref(e), y, None, 0, None)
    return L.mixllm_mixed_linear_fp16_epilogue(C.byref(d), x, W, W, W, W, W, W, C.byref(e), y, W, 1 << 28, None)


@pytest.mark.parametrize("M", [1, 4, 16, 40, 300])   # one kernel, and quantizer and linear
@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("codes", [False, True])
def test_epilogues_refuse_results_on_their_operands(M, gated, codes):
    N, K = 256, 256
    xb, yb = M * K * (1 if codes else 2), M * (N // 2 if gated else N) * 2
    call = lambda x=W, y=FAKE, residual=None: epilogue(M, N, gated, x, y, residual, codes, K)
    assert call(x=FAKE) == EINVAL                                     # K = N, in place
    assert call(x=FAKE, residual=FAKE) == EINVAL
    assert call(x=FAKE + yb - 16) == EINVAL and call(x=FAKE - xb + 16) == EINVAL
    assert call(x=FAKE + yb) == EHIP and call(x=FAKE - xb) == EHIP    # side by side
    assert call(residual=FAKE) == EHIP                                # added to in place
    assert call(residual=FAKE + 16) == EINVAL and call(residual=FAKE - 16) == EINVAL
    assert call(residual=FAKE + yb) == EHIP and call(residual=FAKE - yb) == EHIP
    assert call(x=FAKE + yb, residual=FAKE + yb) == EHIP              # the activations as the residual, results elsewhere


@pytest.mark.parametrize("M,gather", [(1, 4), (8, 0), (300, 2)])
@pytest.mark.parametrize("gated", [0, 1])
def test_experts_refuse_results_on_their_activations(M, gather, gated):
    N, K = 256, 256
    e, d, L = binding._Epilogue(None, None, 0, gated), binding._desc(M, K, N, 8), mx.lib()
    yb = M * max(gather, 1) * (N // 2 if gated else N) * 2
    for size, call in ((2, lambda x, xs=W: L.mixllm_experts_linear_fp16(C.byref(d), 4, W, x, W, W, gather, C.byref(e), FAKE, W, 1 << 28, None)),
                       (1, lambda x, xs=W: L.mixllm_experts_linear(C.byref(d), 4, W, x, xs, W, W, gather, C.byref(e), FAKE, None))):
        assert call(FAKE) == EINVAL and call(FAKE + yb - 16) == EINVAL and call(FAKE - M * K * size + 16) == EINVAL
        assert call(FAKE + yb) == EHIP and call(FAKE - M * K * size) == EHIP
    assert call(W, FAKE) == EINVAL


def test_sums_refuse_results_on_their_operands():
    T, k, N, places = 4, 2, 64, 8
    row = 2 * N
    f = lambda y=W, w=W, s=W, r=None: mx.lib().mixllm_experts_combine(T, k, N, places, y, w, s, r, FAKE, None)
    assert f() == f(r=FAKE) == f(y=FAKE + T * row) == f(y=FAKE - places * row) == f(r=FAKE + T * row) == EHIP
    for bad in (dict(y=FAKE), dict(y=FAKE + (T - 1) * row), dict(y=FAKE - (places - 1) * row), dict(w=FAKE + 4), dict(s=FAKE - 4), dict(r=FAKE + 16)):
        assert f(**bad) == EINVAL, bad


def test_grids_that_cannot_be_launched_are_refused():
    # 1024 experts with a row each, 2^23 channels: 2^26 tiles
    e, L, address = binding._Epilogue(None, None, 0, 0), mx.lib(), W
    d = binding._desc(1024, 128, 1 << 23, 0)
    y = 0x7f0000000000
    assert L.mixllm_experts_linear(C.byref(d), 1024, address, address, address, address, address, 1, C.byref(e), y, None) == -2
    assert L.mixllm_experts_linear_fp16(C.byref(d), 1024, address, address, address, address, 1, C.byref(e), y, address, 1 << 24, None) == -2
