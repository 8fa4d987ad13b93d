"""The experts' products for a token or a few, on sizes at which the kernel's blocks go through full rounds of tiles, change from
one batch of rounds to the next, take more chunks than a list holds, and scan more than 512 experts.  Each case says how much of
that it reaches, and checks it."""
import numpy as np
import pytest
import torch

import paper_2412_14590_amd as mx
from oracle import ref
from paper_2412_14590_amd import synth
from test_operators import check, epilogue64, ids_of, lists_of, route_of, sums64
from util import G, dev, pack_from_oracle

pytestmark = pytest.mark.gpu
WAVES, BATCH, LIST = 8, 4, 64   # tiles of a round and block, rounds of a batch, chunks of a list


def random_layer(K, N, n8, grouped8, seed):
    """A layer of random codes and scales in an order of random pairs."""
    rng = np.random.default_rng(seed)
    p = rng.permutation(N // 2)
    perm = np.stack([2 * p, 2 * p + 1], 1).reshape(-1).astype(np.int32)
    ng, n4 = K // G, N - n8
    scale = lambda *s: (rng.random(s) * 2e-3 + 1e-3).astype(np.float16)
    return ref.QuantizedLayer(N, K, G, G if grouped8 else K, perm, rng.integers(-127, 128, (n8, K), dtype=np.int8), scale(n8, ng if grouped8 else 1) / np.float16(8),
                              rng.integers(0, 16, (n4, K), dtype=np.uint8), scale(n4, ng), rng.integers(0, 16, (n4, ng), dtype=np.uint8))


def rounds_of(counts, layers, N):
    """Full rounds of either part's blocks (8-bit, 4-bit), from the rows of every expert."""
    tiles = lambda n: (n + 15) // 16
    U8 = sum(tiles(c) * tiles(L.n8) for c, L in zip(counts, layers))
    U4 = sum(tiles(c) * tiles(N - L.n8) for c, L in zip(counts, layers))
    B = torch.cuda.get_device_properties(0).multi_processor_count
    nb8 = 0 if U8 == 0 else min(max(int(2.0 * U8 * B / (2.0 * U8 + U4) + 0.5), 1), B)
    nb8 = min(nb8, B - 1) if U4 else nb8
    return (U8 // (WAVES * nb8) if nb8 else 0), (U4 // (WAVES * (B - nb8)) if B > nb8 else 0)


# tokens, experts, k, K, N, shares of 8-bit channels, rounds of the 8-bit and of the 4-bit part (at least).  (With one scale a row
# more than eight rows of a short K are the tiled kernel's: such cases are here for the scales per group.)
CASES = {
    "rounds and a rest": (2, 8, 4, 128, 16002, (0.1, 0.0, 0.3), (1, 1)),
    "... of many rows": (8, 6, 4, 128, 16002, (0.1, 0.0, 0.3), (1, 1)),
    "a change of batch": (1, 8, 8, 128, 40002, (0.1, 0.0, 0.3, 1.0, 0.2), (5, 5)),
    "... of many rows, too": (16, 16, 8, 128, 16002, (0.1, 0.0, 0.3, 1.0, 0.2), (5, 5)),
    "three row tiles": (60, 3, 2, 128, 16002, (0.2, 0.05, 0.4), (2, 4)),
    "ragged groups": (4, 8, 2, 640, 16002, (0.5, 0.0, 1.0), (1, 1)),
    "many rows of a long K": (4, 20, 8, 4096, 2050, (0.1, 0.4), (0, 0)),
    "two lists of chunks": (1, 32, 32, 16256, 4112, (0.2, 0.0), (2, 4)),
    "one part only": (1, 8, 8, 128, 40002, (0.0,), (0, 5)),
    "the other part only": (1, 8, 8, 256, 22002, (1.0,), (5, 0)),
    "more than 512 experts": (4, 700, 2, 128, 34, (0.1, 0.0, 1.0, 0.5), (0, 0)),
    "1024 experts": (2, 1024, 4, 128, 66, (0.3, 1.0), (0, 0)),
    "1024 experts, many rows": (5, 1024, 20, 128, 66, (0.3, 1.0), (0, 0)),
}


@pytest.mark.parametrize("act_grouped,w8_grouped", [(False, False), (True, True), (False, True), (True, False)])
@pytest.mark.parametrize("name", list(CASES))
def test_every_turn_of_the_loop(name, act_grouped, w8_grouped):
    T, E, k, K, N, shares, least = CASES[name]
    rng = np.random.default_rng(len(name) + 2 * act_grouped + w8_grouped)
    kinds = [random_layer(K, N, 2 * int(s * N / 2), w8_grouped, i) for i, s in enumerate(shares)]
    packed = [pack_from_oracle(L) for L in kinds]
    which = np.arange(E) % len(kinds)
    layers = [kinds[i] for i in which]
    PE = mx.pack_experts([packed[i] for i in which])
    ids = ids_of("some", T, E, k, rng)
    if E > 512:
        ids[0, :2] = 511, E - 1                              # either side of a pass, and the last
        ids[1, :2] = 512, 0
        ids = np.stack([np.concatenate([row[:2], [e for e in rng.permutation(E) if e not in row[:2]][:k - 2]]) for row in ids]).astype(np.int32)
    offsets, rows, _ = lists_of(ids, E)
    counts = np.diff(offsets)
    got = rounds_of(counts, layers, N)
    assert got[0] >= least[0] and got[1] >= least[1], got
    if name == "two lists of chunks":
        assert min(got[0], BATCH) * (K + 511) // 512 >= LIST - 1 and min(got[1], BATCH) * (K // 512) > LIST
    route, places = route_of(ids, E, T, k), T * k
    assert places <= 128 and T * K <= 16384                   # the one-kernel form
    for gather, gated in ((True, True), (False, False)):
        if (T if gather else places) * K > 16384:
            continue                                          # (the tiled kernel's)
        x = synth.make_x(T if gather else places, K, gather)
        xq, xs = ref.quantize_act(x, G if act_grouped else None)
        bias = (rng.standard_normal((E, N)) * 0.5).astype(np.float16)
        No = N // 2 if gated else N
        area = torch.full((places * No + 4096,), 7.0, dtype=torch.float16, device="cuda")
        out = area[2048:2048 + places * No].view(places, No)
        act = "silu" if gated else "relu"
        mx.experts_linear_fp16(dev(x), PE, route, dev(bias), act, gated=gated, gather=gather, act_group=G if act_grouped else None, out=out)
        y = out.cpu().numpy()
        assert (y != 7).any(axis=1).all() and bool((area[:2048] == 7).all()) and bool((area[2048 + places * No:] == 7).all())
        for e in rng.permutation(np.nonzero(counts)[0])[:24 if K < 1024 else 10]:
            at = np.arange(offsets[e], offsets[e + 1])
            src = rows[at] // k if gather else at
            z, dz = sums64(xq[src], xs[src], layers[e])
            check(y[at], *epilogue64(z, dz, bias[e], act, gated, None), (name, gather, "expert", e))
