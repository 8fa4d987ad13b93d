"""The table of experts holds device addresses: what they point to stays, and there is one for every expert."""
import gc
import weakref

import pytest
import torch

import paper_2412_14590_amd as mx
from paper_2412_14590_amd import binding, synth


def test_a_table_without_an_entry_for_every_expert_is_refused(monkeypatch):
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    u8 = lambda n: torch.zeros(n, dtype=torch.uint8)
    L = binding.PackedLayer(256, 64, 8, 256, u8(16 * 256), u8(64 * 128), u8(32), u8(64 * 16), u8(64 * 4), torch.zeros(64, dtype=torch.int32))
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    route = mx.Route(i32(4, 2), torch.zeros((4, 2)), i32(4), i32(8), i32(4, 2))
    x = torch.zeros((4, 256), dtype=torch.float16)
    for table in (u8(2 * 64), None):
        E = mx.PackedExperts(256, 64, 256, [L] * 3, table, 8)
        with pytest.raises(AssertionError, match="table"):
            mx.experts_linear_fp16(x, E, route)
        with pytest.raises(AssertionError, match="table"):
            mx.experts_linear(x.to(torch.int8), torch.zeros((4, 1), dtype=torch.float16), E, route)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 40])
def test_layers_that_get_other_tensors_leave_packed_experts_as_they_were(T):
    """Reloading weights into the PackedLayer objects: the experts keep the tensors that their table names."""
    K, N, E = 256, 64, 3
    layers = [mx.quantize_weights(torch.from_numpy(synth.make_w(N, K, 0.02, 1, e)).cuda(), [2, 3, 10, 11][: 2 * (e % 3)]) for e in range(E)]
    PE = mx.pack_experts(layers)
    x = torch.from_numpy(synth.make_x(T, K, 0)).cuda()
    route = mx.route_experts(torch.randn((T, E), device="cuda"), 2)
    want = mx.experts_linear_fp16(x, PE, route, activation="silu", gated=True)
    names = ("w4", "w8", "s4", "s8", "z4", "perm")
    alive = [weakref.ref(getattr(L, n)) for L in layers for n in names]
    for L in layers:
        for n in names:
            setattr(L, n, torch.zeros(1, dtype=torch.uint8, device="cuda"))
    del L
    gc.collect()
    assert all(r() is not None for r in alive)
    assert torch.equal(mx.experts_linear_fp16(x, PE, route, activation="silu", gated=True), want)
    assert PE.E == E and all(getattr(L, n) is r() for (L, n), r in zip(((L, n) for L in PE.layers for n in names), alive))
    PE.layers[0].w4 = None                                        # ... and one replaced in there, too
    gc.collect()
    assert all(r() is not None for r in alive)
    del PE, layers
    gc.collect()
    assert all(r() is None for r in alive)                        # nothing else holds them
