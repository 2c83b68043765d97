"""Outputs that share memory with an input that is still read are refused; rows side by side in one
buffer, and the overlaps that do no harm, are not."""

import ctypes

import pytest
import torch

P = ctypes.c_void_p
BIG = 1 << 40
BASE = 1 << 20  # addresses that are never used: the calls are refused


@pytest.fixture(scope="module")
def L():
    if torch.cuda.is_available():
        pytest.skip("made-up addresses stay away from a GPU")
    from paper_2608_03020_gb300 import _build
    from paper_2608_03020_gb300 import loca

    _build.build()
    return loca.lib()


def _other(i):
    return P((1 << 32) + i * (1 << 24))


# 10 rows of 64 channels in, 72 out; (offset in bytes, pitch in elements) of Y against X at pitch 64 or 144
@pytest.mark.parametrize("ldx,off,ldy", [
    (64, 0, 72), (64, 1264, 72), (64, -1424, 72), (144, 0, 144), (144, 112, 144), (144, 144 * 2 - 128, 144),
    (144, -288 * 9 - 128, 144), (144, 288 * 9 + 112, 144), (144, 128, 152), (64, 16, 200),
])
def test_apply_refuses_y_over_x(L, ldx, off, ldy):
    rc = L.loca_adapter_apply(P(BASE), ldx, 10, 64, _other(0), 72, _other(1), 2, 4, _other(2), P(BASE + off), ldy,
                              _other(3), BIG, None)
    assert rc == 1 and b"overlap" in L.loca_last_error_string()


@pytest.mark.parametrize("over", ["X with dA", "X with dB", "dY", "dY and no gradient of the adapters"])
def test_backward_refuses_dx_over_its_inputs(L, over):
    X, dY = P(BASE), P(BASE + (1 << 16))
    dX = P(BASE + 64) if over.startswith("X") else P(BASE + (1 << 16) + 1024)
    dA = _other(4) if over in ("X with dA", "dY") else None
    dB = _other(5) if over == "X with dB" else None
    rc = L.loca_adapter_backward(X, 64, dY, 72, 10, 64, _other(0), 72, _other(1), 2, 4, _other(2), dX, 64, dA, dB, 0,
                                 _other(3), BIG, None)
    assert rc == 1 and b"overlap" in L.loca_last_error_string()


@pytest.mark.parametrize("off,ld", [(128, 64), (-128, 64), (0, 72), (16, 64)])
def test_head_backward_refuses_dh_across_h(L, off, ld):
    rc = L.loca_head_loss_backward(P(BASE), 64, 10, 64, _other(0), 100, _other(1), None, _other(2), None,
                                   ctypes.c_float(1.0), P(BASE + off), ld, None, _other(3), BIG, None)
    assert rc == 1 and b"overlap" in L.loca_last_error_string()


@pytest.mark.gpu
def test_what_does_no_harm_is_taken():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_03020_gb300 import _build

    _build.build()
    from paper_2608_03020_gb300 import loca as lc

    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    N, d, o, k, n, V = 700, 128, 200, 8, 3, 999
    X, dY, W = rn(N, d).to(torch.bfloat16), rn(N, o).to(torch.bfloat16), (rn(o, d) / 11).to(torch.bfloat16)
    A, B = rn(n, d, k), rn(n, o, k)
    ad = lc.AdapterSet(n, d, o, k).pack(A, B)
    plan = lc.AdapterPlan(torch.randint(-1, n, (N,), generator=g, device="cuda", dtype=torch.int32), n)
    Y, dX = torch.empty_like(dY), torch.empty_like(X)
    lc.loca_adapter_apply(X, W, ad, plan, Y)
    lc.loca_adapter_backward(X, dY, W, ad, plan, dX=dX)
    both = torch.zeros((N, d + o), dtype=torch.bfloat16, device="cuda")  # X and Y side by side
    both[:, :d] = X
    lc.loca_adapter_apply(both[:, :d], W, ad, plan, both[:, d:])
    assert torch.equal(both[:, d:], Y) and torch.equal(both[:, :d], X)
    again = X.clone()  # dX alone reads no X
    lc.loca_adapter_backward(again, dY, W, ad, plan, dX=again)
    assert torch.equal(again, dX)
    head, y = (rn(V, d) / 11).to(torch.bfloat16), torch.randint(-300, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    loss, lse, dH = torch.empty((N,), device="cuda"), torch.empty((N,), device="cuda"), torch.empty_like(X)
    lc.loca_head_loss(X, head, y, loss, lse=lse)
    dW, dW2 = torch.empty_like(head), torch.empty_like(head)
    lc.loca_head_loss_backward(X, head, y, lse, dH=dH, dW=dW)
    again = X.clone()  # dH in the place of H
    lc.loca_head_loss_backward(again, head, y, lse, dH=again, dW=dW2)
    torch.cuda.synchronize()
    assert torch.equal(again, dH) and torch.equal(dW, dW2) and lc.loca_device_status() == 0
