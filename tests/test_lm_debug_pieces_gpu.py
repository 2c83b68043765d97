"""The head loss backward in pieces of rows and of the vocabulary, with the sums behind the targets'
entries, through the LOCA_DEBUG build between poisoned guard bands."""

import pytest
import test_lm_debug_gpu as debug
import torch

pytestmark = pytest.mark.gpu
lc = debug.lc  # the fixture


def _backward(lc, mk, N, d, V, dw, masked):
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    H = torch.randn((N, d), generator=g, device="cuda").to(torch.bfloat16)
    W = (torch.randn((V, d), generator=g, device="cuda") / d ** 0.5).to(torch.bfloat16)
    y = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    y[torch.rand((N,), generator=g, device="cuda") < masked] = -1
    loss, lse = torch.empty((N,), device="cuda"), torch.empty((N,), device="cuda")
    lc.loca_head_loss(H, W, y, loss, lse=lse)
    o = {"dH": mk.empty((N, d), torch.bfloat16)}
    if dw:
        o["dW"] = mk.empty((V, d), torch.bfloat16)
    ws = mk.empty((lc.head_loss_backward_workspace_size(N, V, d, True, dw),), torch.uint8)
    lc.loca_head_loss_backward(H, W, y, lse, dH=o["dH"], dW=o.get("dW"), workspace=ws)
    mk.check("loca_head_loss_backward")
    return o


@pytest.mark.parametrize("N,d,V,dw,masked", [
    (9000, 72, 70001, False, 0.3),            # two pieces of the rows
    (9000, 72, 70001, False, 0.9),            # the second without a live row
    (100, 8, (1 << 21) + 300, False, 0.1),    # up to 128 tokens, two pieces of the vocabulary
    (300, 8, (1 << 21) + 300, False, 0.1),
    (11500, 8, 190001, True, 0.1),            # dW: two pieces of the vocabulary
    (17, 200, 65, True, 0.0),
    (300, 200, 1, True, 0.0),
])
def test_pieces_stay_inside(lc, N, d, V, dw, masked):
    lc.use_debug_library(False)
    ref = _backward(lc, debug.Guarded(lc), N, d, V, dw, masked)
    lc.use_debug_library(True)
    assert lc.loca_debug_build()
    got = _backward(lc, debug.Guarded(lc), N, d, V, dw, masked)
    lc.use_debug_library(False)
    for k in ref:
        assert torch.equal(ref[k], got[k]), k
