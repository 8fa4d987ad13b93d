"""The router's weights are formed in 64 bits and rounded once, whatever is asked for."""
import pytest
import torch

from test_operators import check_route

pytestmark = pytest.mark.gpu

# half a step of fp32, and room for the 64-bit arithmetic of both sides (some 2^-45)
ONE_ROUNDING = 2.0 ** -24 * (1 + 2.0 ** -20)


# one launch and two; a wave and 16 lanes a token, one to sixteen experts a lane
@pytest.mark.parametrize("T,E,k", [(1, 64, 4), (16, 1024, 8), (300, 100, 6), (500, 256, 8), (64, 900, 5), (2100, 64, 6), (4200, 128, 8), (8200, 250, 8)])
@pytest.mark.parametrize("kw", [dict(renormalize=False), dict(), dict(score="sigmoid", renormalize=False), dict(bias=True, renormalize=False)],
                         ids=["softmax", "renormalized", "sigmoid", "bias"])
def test_weights_are_rounded_once(T, E, k, kw):
    gen = torch.Generator(device="cuda").manual_seed(T + E)
    logits = 2 * torch.randn((T, E), generator=gen, device="cuda")
    kw = dict(kw)
    if kw.pop("bias", False):
        kw["bias"] = 0.1 * torch.randn(E, generator=gen, device="cuda")
    check_route(logits, k, tol=ONE_ROUNDING, **kw)
