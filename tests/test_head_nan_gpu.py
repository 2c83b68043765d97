"""A NaN among the logits of a position reaches its loss and normaliser, wherever its column stands
among the columns that one thread reduces."""

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


# the last column alone in its half tile (V = 128 m + 1), with others, the only one; up to 128 tokens
# and more.  Columns beside it may be -inf: zero times infinity must not hide it either
@pytest.mark.parametrize("N", [3, 300])
@pytest.mark.parametrize("V,at", [(1, 0), (257, 256), (385, 384), (32001, 32000), (300, 299), (300, 5)])
@pytest.mark.parametrize("low", [False, True])
def test_nan_in_one_column(lc, N, V, at, low):
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    d = 64
    H = torch.randn((N, d), generator=g, device="cuda").abs().to(torch.bfloat16)
    W = torch.randn((V, d), generator=g, device="cuda").to(torch.bfloat16)
    y = torch.zeros((N,), dtype=torch.int32, device="cuda")
    y[1] = -1
    if low:  # every other logit of the half tile -inf
        first = at // 128 * 128
        W[max(first, 1):first + 128] = float("-inf")
    W[at, 3] = float("nan")
    loss, lse = torch.zeros((N,), device="cuda"), torch.zeros((N,), device="cuda")
    dH = torch.zeros((N, d), dtype=torch.bfloat16, device="cuda")
    lc.loca_head_loss(H, W, y, loss, lse=lse)
    lc.loca_head_loss_backward(H, W, y, lse, dH=dH)
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0
    live = y >= 0
    assert torch.isnan(loss[live]).all() and torch.isnan(lse[live]).all() and torch.isnan(dH[live].float()).all()
    assert loss[1] == 0 and lse[1] == 0 and torch.all(dH[1] == 0)


def test_columns_of_minus_infinity_count_for_nothing(lc):
    N, d, V = 200, 64, 700
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    H = torch.randn((N, d), generator=g, device="cuda").abs().to(torch.bfloat16)
    W = torch.randn((V, d), generator=g, device="cuda").to(torch.bfloat16)
    y = torch.randint(0, 256, (N,), generator=g, device="cuda", dtype=torch.int32)
    loss, want = torch.empty((N,), device="cuda"), torch.empty((N,), device="cuda")
    lc.loca_head_loss(H, W[:256].contiguous(), y, want)
    W[256:] = float("-inf")
    lc.loca_head_loss(H, W, y, loss)
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0
    # the same 256 logits, whose partial sums stand in the same two tiles' halves
    assert float((loss - want).abs().max()) <= 4e-6 * float(1.0 + want.abs().max())
