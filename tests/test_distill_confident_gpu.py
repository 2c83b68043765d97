"""Gradients of distillation where teacher and student agree on one word almost surely, position by position.

With q and p of that word nearly one its entry of dZ, tau (p - q), is a difference of nearly equal numbers, and the
position's whole gradient is as small as 1 - p and 1 - q; a norm over all positions does not see it.  Each row of
``dH`` (and of ``dW``) is therefore held to its own terms.  In exact arithmetic the word's entry is
tau (sum of the others' q - sum of the others' p).  Bound, fixed before the first run: every scaled logit and
normaliser is within 2e-5 (1 + max |z|) / tau (derived in the operator's own tests), so every p and every sum of the
others' p is off by at most twice that, relatively; q comes from logits of at most 32 in size (after the division by
tau), two roundings of 2^-24 of them, the logarithm and the exponential of some ulp: 2^-17 of it; dZ and the gradient
are each rounded to bf16 (2^-8).  A row of dH is then within
  (2^-7 |dZ| + c p + 2^-17 q) |W|, summed over the words with the agreed word's p and q replaced by the others' sums,
  c = 4e-5 (1 + max |z|) / tau,
of its value, a row of dW within the same with |H|, summed over the positions.
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


def _inputs(N, d, V, K, level, decades, tau, seed=0):
    """Hidden states along the agreed word's row, as far as 1 - p comes out over that many decades below about 0.1, a
    direction common to all positions that moves every logit by `level` (and lse with it), and teachers whose 1 - q
    spans the same decades, apart from 1 - p by up to a factor of three."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + N + 3 * d + 5 * V + 7 * K)
    common = torch.randn((d,), generator=g, device="cuda")
    common /= common.norm()
    W = 2.0 / d ** 0.5 * torch.randn((V, d), generator=g, device="cuda")
    W -= (W @ common)[:, None] * common
    y = torch.randint(0, V, (N,), generator=g, device="cuda")
    unit = W[y] / W[y].square().sum(1, keepdim=True)
    # the others' scaled logits have a variance of far^2 / d: 1 - p is about V exp(far^2 / 2 d - far)
    below = 2.3 * decades * torch.rand((N, 1), generator=g, device="cuda")
    sure = math.log(V) + 2.0 + below
    far = d * (1.0 - torch.sqrt(1.0 - 2.0 * sure / d))
    H = (tau * far * unit + level / 4.0 * common).to(torch.bfloat16)
    W = (W + 4.0 * common).to(torch.bfloat16)
    # the agreed word at a place of its own among the K, the others' shares some e^-(2 + below) together
    idx = torch.randint(0, V, (N, K), generator=g, device="cuda")
    t = torch.randn((N, K), generator=g, device="cuda") - math.log(max(K - 1, 1))
    own = 2.0 + below + 2.2 * (torch.rand((N, 1), generator=g, device="cuda") - 0.5)
    at = torch.randint(0, K, (N, 1), generator=g, device="cuda")
    idx.scatter_(1, at, y[:, None])
    t.scatter_(1, at, own)
    t = tau * (t - 3.0)
    idx[5::7] = -1
    w = torch.rand((N,), generator=g, device="cuda") + 0.5
    return H, W, idx.to(torch.int32).contiguous(), t.contiguous(), y, w


def _check(lc, H, W, idx, t, y, w, tau, least, dw, rows=1000):
    N, d = H.shape
    V, K = W.shape[0], idx.shape[1]
    assert float(t.abs().max()) / tau <= 32.0
    loss, lse = torch.empty((N,), device="cuda"), torch.empty((N,), device="cuda")
    dH = torch.full((N, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    dW = torch.full((V, d), float("nan"), dtype=torch.bfloat16, device="cuda") if dw else None
    lc.loca_head_distill(H, W, idx, t, loss, lse=lse, w=w, tau=tau)
    lc.loca_head_distill_backward(H, W, idx, t, lse, dH=dH, dW=dW, w=w, tau=tau)
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0
    Wd, live = W.double(), torch.nonzero(idx[:, 0] >= 0)[:, 0]
    size_w = Wd.norm(dim=1)
    want_w, room_w = torch.zeros((V, d), dtype=torch.float64, device="cuda") if dw else None, torch.zeros_like(size_w)
    zmax = 0.0
    for r in live.split(rows):
        zmax = max(zmax, float((H[r].double() @ Wd.T).abs().max()))
    c = 4e-5 * (1.0 + zmax) / tau
    unsure, worst = [], []
    for r in live.split(rows):
        Hr, yr = H[r].double(), y[r].long()
        n = torch.arange(len(r), device="cuda")
        p = torch.softmax(Hr @ Wd.T / tau, 1)
        share = torch.softmax(t[r].double() / tau, 1)
        q = torch.zeros_like(p).scatter_add_(1, idx[r].long(), share)
        p[n, yr], q[n, yr] = 0.0, 0.0
        others_p, others_q = p.sum(1), q.sum(1)
        dz = p - q
        dz[n, yr] = others_q - others_p  # without the cancellation
        p[n, yr], q[n, yr] = others_p, others_q
        wr = w[r].double()[:, None] * tau
        dz *= wr
        room = 2.0 ** -7 * dz.abs() + wr * (c * p + 2.0 ** -17 * q)
        unsure.append(others_p)
        worst.append((dH[r].double() - dz @ Wd).norm(dim=1) / (room @ size_w))
        if dw:
            want_w += dz.T @ Hr
            room_w += room.T @ Hr.norm(dim=1)
    unsure, worst = torch.cat(unsure), torch.cat(worst)
    assert N <= 2 or float(unsure.min()) < least < 0.03 < float(unsure.max()), (float(unsure.min()), float(unsure.max()))
    i = int(worst.argmax())
    assert float(worst[i]) <= 1.0, ("dH", float(worst[i]), "1 - p", float(unsure[i]), "of", float((worst > 1.0).float().mean()))
    assert torch.all(dH[idx[:, 0] < 0] == 0)
    if dw:
        ratio = (dW.double() - want_w).norm(dim=1) / room_w.clamp(min=1e-300)
        i = int(ratio.argmax())
        assert float(ratio[i]) <= 1.0, ("dW", float(ratio[i]), i)


@pytest.mark.parametrize("N,d,V,K,level,tau,dw", [
    (2000, 5120, 32000, 8, 30.0, 1.0, True),      # many positions, a long k
    (600, 2048, 49152, 64, 30.0, 1.0, False),
    (777, 896, 32003, 5, 30.0, 2.0, True),
    (300, 896, 5003, 200, 0.0, 1.0, True),        # more words than go against all columns at once
    (100, 5120, 32000, 16, 30.0, 1.0, True),      # up to 128 positions
    (100, 896, 4099, 120, 30.0, 1.0, True),       # of them, rows with several words in a half tile
    (63, 896, 20011, 6, 30.0, 1.5, True),         # dZ in two parts
    (40, 896, 2003, 100, 30.0, 1.0, True),
    (1, 896, 5003, 4, 0.0, 1.0, True),
    (500, 896, 20011, 1, 30.0, 1.0, True),        # the word alone: q is one
    (9000, 104, 70001, 4, 10.0, 1.0, False),      # pieces of the rows
    (11500, 104, 190001, 4, 10.0, 1.0, True),     # pieces of the vocabulary
    (130, 104, (1 << 21) + 300, 3, 0.0, 1.0, False),
    (20, 104, (1 << 21) + 300, 3, 0.0, 1.0, False),
])
def test_positions_over_four_decades_of_certainty(lc, N, d, V, K, level, tau, dw):
    # (1 - p cannot come out below what bf16 hidden states resolve; 20 positions do not reach the last decade)
    _check(lc, *_inputs(N, d, V, K, level, 4.0, tau), tau, 1e-4 if N > 100 else 1e-2, dw, rows=max(1, int(3e8 / V)))
