"""Gradients of the head loss for positions that the model predicts almost surely, row by row.

dZ of such a target is p - 1, a difference of nearly equal numbers: the row's whole gradient is as small
as 1 - p, and a norm over all rows does not see it.  Each row of ``dH`` (and each row of ``dW``) is
therefore held to its own terms.  Bound, fixed before the first run: every logit and normaliser is within
2e-5 (1 + max |z|) (the head loss's own tests derive it), so every p is off by at most twice that,
relatively, and so is the sum of the others' p that the target's entry consists of; dZ and the gradient
are each rounded to bf16, whose unit roundoff is 2^-8 (8 significant bits).  A row of dH is then within
(2^-7 + 4e-5 (1 + max |z|)) sum_v |dZ_nv| |W_v| of its value, a row of dW within the same of
sum_n |dZ_nv| |H_n|.
"""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lc():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_03020_gb300 import _build

    _build.build()
    from paper_2608_03020_gb300 import loca

    loca.lib()
    return loca


def _inputs(N, d, V, level, decades, seed=0):
    """Hidden states along their target's row, as far as 1 - p comes out over that many decades below about
    0.1, and a direction common to all rows that moves every logit by `level`."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + N + 3 * d + 5 * V)
    common = torch.randn((d,), generator=g, device="cuda")
    common /= common.norm()
    W = 2.0 / d ** 0.5 * torch.randn((V, d), generator=g, device="cuda")
    W -= (W @ common)[:, None] * common
    y = torch.randint(0, V, (N,), generator=g, device="cuda")
    unit = W[y] / W[y].square().sum(1, keepdim=True)
    # the others' logits have a variance of far^2 / d: 1 - p is about V exp(far^2 / 2 d - far)
    sure = math.log(V) + 2.0 + 2.3 * decades * torch.rand((N, 1), generator=g, device="cuda")
    far = d * (1.0 - torch.sqrt(1.0 - 2.0 * sure / d))
    H = (far * unit + level / 4.0 * common).to(torch.bfloat16)
    W = (W + 4.0 * common).to(torch.bfloat16)
    y = y.to(torch.int32)
    y[5::7] = -1
    w = torch.rand((N,), generator=g, device="cuda") + 0.5
    return H, W, y, w


def _check(lc, H, W, y, w, least, dw, rows=1000):
    N, d = H.shape
    V = W.shape[0]
    loss, lse = torch.empty((N,), device="cuda"), torch.empty((N,), device="cuda")
    dH = torch.full((N, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    dW = torch.full((V, d), float("nan"), dtype=torch.bfloat16, device="cuda") if dw else None
    lc.loca_head_loss(H, W, y, loss, lse=lse, w=w)
    lc.loca_head_loss_backward(H, W, y, lse, dH=dH, dW=dW, w=w)
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0
    Wd, live = W.double(), torch.nonzero(y >= 0)[:, 0]
    size_w = Wd.norm(dim=1)
    want_w, size = torch.zeros((V, d), dtype=torch.float64, device="cuda") if dw else None, torch.zeros_like(size_w)
    unsure, worst, zmax = [], [], 0.0
    for r in live.split(rows):
        Hr, yr = H[r].double(), y[r].long()
        z = Hr @ Wd.T
        zmax = max(zmax, float(z.abs().max()))
        at = torch.arange(len(r), device="cuda")
        dz = torch.softmax(z, 1)
        dz[at, yr] = 0.0
        others = dz.sum(1)
        dz[at, yr] = -others  # p - 1, without the cancellation
        unsure.append(others)
        dz *= w[r].double()[:, None]
        off = (dH[r].double() - dz @ Wd).norm(dim=1)
        worst.append(off / (dz.abs() @ size_w))
        if dw:
            want_w += dz.T @ Hr
            size += dz.abs().T @ Hr.norm(dim=1)
    unsure, worst = torch.cat(unsure), torch.cat(worst)
    assert N == 1 or float(unsure.min()) < least < 0.03 < float(unsure.max()), (float(unsure.min()), float(unsure.max()))
    tol = 2.0 ** -7 + 4e-5 * (1.0 + zmax)
    i = int(worst.argmax())
    assert float(worst[i]) <= tol, ("dH", float(worst[i]), tol, "1 - p", float(unsure[i]), "of", float((worst > tol).float().mean()))
    assert torch.all(dH[y < 0] == 0)
    if dw:
        ratio = (dW.double() - want_w).norm(dim=1) / size
        i = int(ratio.argmax())
        assert float(ratio[i]) <= tol, ("dW", float(ratio[i]), tol)


# dZ's logits have to be the sums that went into lse: where they restarted at other places, the difference
# grew with the logits and with d
@pytest.mark.parametrize("N,d,V,level,dw", [(2000, 5120, 32000, 200.0, True), (600, 2048, 49152, 200.0, False),
                                            (100, 5120, 32000, 200.0, True), (400, 8192, 4099, 100.0, False)])
def test_large_logits_of_fairly_sure_rows(lc, N, d, V, level, dw):
    _check(lc, *_inputs(N, d, V, level, 1.0), 0.02, dw)


# p - 1 of a target is a difference of nearly equal numbers
@pytest.mark.parametrize("N,d,V,level,dw", [
    (2000, 5120, 32000, 30.0, True),      # many tokens, a long k
    (600, 2048, 49152, 30.0, False),
    (100, 5120, 32000, 30.0, True),       # up to 128 tokens
    (1, 896, 5003, 0.0, True),
    (777, 896, 32003, 0.0, True),
    (9000, 104, 70001, 10.0, False),      # pieces of the rows
    (3000, 104, 200000, 10.0, True),
    (11500, 104, 190001, 10.0, True),     # pieces of the vocabulary
    (130, 104, (1 << 21) + 300, 0.0, False),
])
def test_rows_over_four_decades_of_certainty(lc, N, d, V, level, dw):
    _check(lc, *_inputs(N, d, V, level, 4.0), 1e-4, dw, rows=max(1, int(3e8 / V)))
