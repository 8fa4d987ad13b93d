"""Results of the operators next to the linear are of the type that the operand's own new_empty makes."""
import pytest
import torch
from torch.overrides import TorchFunctionMode

import paper_2412_14590_amd as mx
from paper_2412_14590_amd import synth

pytestmark = pytest.mark.gpu


class Tagged(torch.Tensor):
    """A tensor subclass: its methods' results are of its type."""


class Seen(TorchFunctionMode):
    count = 0

    def __torch_function__(self, func, types, args=(), kwargs=None):
        self.count += func is torch.Tensor.new_empty
        return func(*args, **(kwargs or {}))


@pytest.mark.parametrize("T", [3, 40])
def test_results_come_from_the_operands_own_new_empty(T):
    layer = lambda N, K: mx.quantize_weights(torch.from_numpy(synth.make_w(N, K, 0.02, 1, N)).cuda(), [2, 3])
    PL, up, down = layer(64, 256), mx.pack_experts([layer(256, 256)] * 3), mx.pack_experts([layer(64, 128)] * 3)
    x, logits = torch.from_numpy(synth.make_x(T, 256, 1)).cuda(), torch.randn((T, 3), device="cuda")

    def results(kind):
        X, l = x.as_subclass(kind), logits.as_subclass(kind)
        r = mx.route_experts(l, 2)
        xq, xs = mx.quantize_activations(X)
        h = mx.experts_linear_fp16(X, up, r, activation="silu", gated=True)
        y = mx.experts_linear_fp16(h, down, r, gather=False)
        return [r.ids, r.weights, r.offsets, r.rows, r.slots, mx.linear_fp16_epilogue(X, PL, activation="relu"), mx.mixed_linear_epilogue(xq, xs, PL),
                h, mx.experts_linear(xq, xs, up, r, gated=True), y, mx.experts_combine(y, r), mx.experts_mlp(X, r, up, down)]

    want = results(torch.Tensor)
    got = results(Tagged)
    assert all(type(t) is torch.Tensor for t in want) and all(type(t) is Tagged for t in got)
    for a, b in zip(want, got):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b.as_subclass(torch.Tensor))
    with Seen() as mode:
        results(torch.Tensor)
    assert mode.count >= 15
