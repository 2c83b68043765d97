"""Distillation, gated feed-forward and 4-bit projection where elements lie more than 2^31 behind the first: the first and the
last rows against the definition in 64 bits, with the tolerances of each operator's own tests."""

import pytest
import torch

import test_distill_gpu as distill
import test_gated_gpu as gated
import test_q4_gpu as q4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lc():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_03020_gb300 import _build

    _build.build()
    from paper_2608_03020_gb300 import loca

    loca.lib()
    return loca


def _ends(n, k=3):
    return torch.cat([torch.arange(k), torch.arange(n - k, n)]).cuda()


def test_gated(lc):
    N, d, f = 33000, 64, 65536
    X, Wg, Wu, _ = gated._inputs(1, d, f)
    X = torch.randn((N, d), device="cuda").to(torch.bfloat16)
    dH = torch.empty((N, f), dtype=torch.bfloat16, device="cuda").normal_()
    out = gated._run(lc, X, Wg, Wu, dH, "silu", want=("H", "dX"))
    at = _ends(N)
    val, tol = gated._reference(X[at], Wg, Wu, dH[at], "silu")
    gated._check({k: v[at] for k, v in out.items()}, val, tol)


def test_distill(lc):
    N, d, V, K = 1_100_000, 2048, 300, 4
    _, W, _, _, _, _ = distill._inputs(1, d, V, K)
    H = torch.empty((N, d), dtype=torch.bfloat16, device="cuda").normal_()
    idx = torch.randint(0, V, (N, K), device="cuda", dtype=torch.int32)
    t, w, gl = torch.randn((N, K), device="cuda"), torch.rand((N,), device="cuda") + 0.5, torch.randn((N,), device="cuda")
    out = distill._run(lc, H, W, idx, t, w, gl, 2.0, 0.5, dw=False)
    at = _ends(N)
    ref = distill._reference(H[at], W, idx[at], t[at], w[at], gl[at], 2.0, 0.5)
    distill._check({k: v[at] for k, v in out.items()}, ref, w[at], 2.0, V, K)


def test_q4_weight(lc):
    o, d, group = 140_000, 32768, 128
    codes = torch.empty((o, d // 2), dtype=torch.uint8, device="cuda").random_(0, 256)
    scales = (torch.rand((o, d // group), device="cuda") + 0.1) * d ** -0.5
    zeros = torch.randint(0, 16, scales.shape, device="cuda", dtype=torch.uint8)
    weight, at = lc.Q4Weight(codes, scales, zeros=zeros), _ends(o, 40)
    c = codes[at]
    q = torch.stack([c & 15, c >> 4], 2).reshape(80, d // group, group).double()
    W = (scales[at].double()[:, :, None] * (q - zeros[at].double()[:, :, None])).reshape(80, d)
    del codes
    for N in (2, 40):
        X, Y = q4._tokens(N, d), torch.full((N, o), float("nan"), dtype=torch.bfloat16, device="cuda")
        lc.loca_q4_apply(X, weight, Y)
        torch.cuda.synchronize()
        assert lc.loca_device_status() == 0
        y, tol = q4._reference(X, W)
        assert bool(((Y[:, at].double() - y).abs() <= tol).all()) and bool(Y.isfinite().all()), N


@pytest.mark.parametrize("N,pitch", [(16, 1 << 28), (70, 1 << 26)])
def test_q4_rows(lc, N, pitch):
    codes, scales, z, W = q4._weight(136, 256, 64, torch.bfloat16, True)
    weight, X = lc.Q4Weight(codes, scales, zeros=z), q4._tokens(N, 256)
    want = q4._check(lc, X, weight, W)
    flat = torch.empty(((N - 1) * pitch + 512,), dtype=torch.bfloat16, device="cuda")
    xs, ys = flat.as_strided((N, 256), (pitch, 1)), flat.as_strided((N, 136), (pitch, 1), 256)
    xs.copy_(X)
    lc.loca_q4_apply(xs, weight, ys)
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0 and torch.equal(ys, want) and torch.equal(xs, X)
