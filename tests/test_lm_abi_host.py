"""Host-side checks of the head loss, adapter and clipping entry points (no GPU needed): sizes, and
argument validation that rejects bad calls with the documented codes before any CUDA call."""

import ctypes

import pytest

P = ctypes.c_void_p
F = P(256)  # never dereferenced: validation fails first
f = ctypes.c_float
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    from paper_2608_03020_gb300 import _build
    from paper_2608_03020_gb300 import loca

    _build.build()
    return loca.lib()


def _size(fn, *args):
    out = ctypes.c_size_t(0)
    rc = fn(*args, ctypes.byref(out))
    return rc, out.value


def test_head_loss_sizes(L):
    rc, n = _size(L.loca_head_loss_workspace_size, 4096, 151936, 5120, 4)
    # the hidden states once, and two pairs of floats per row and 256 columns (a 64th of the logits in fp32)
    assert rc == 0 and 4096 * 5120 * 2 < n < 4096 * 5120 * 2 + 16 * 4096 * 594 + (1 << 20)
    rc, small = _size(L.loca_head_loss_workspace_size, 1, 1, 8, 0)
    assert rc == 0 and small > 0
    rc, n = _size(L.loca_head_loss_backward_workspace_size, 1 << 17, 151936, 5120, 1, 0)
    assert rc == 0 and n < (1 << 30) + (1 << 17) * 5120 * 2 + 32 * 8192 * 5120 * 4 + (1 << 22)
    for bad in ((-1, 10, 64), (4, 0, 64), (4, 10, 60), (4, 10, 0), (4, 10, 65544), (1 << 25, 10, 64)):
        assert _size(L.loca_head_loss_workspace_size, *bad, 0)[0] == 2, bad
        assert _size(L.loca_head_loss_backward_workspace_size, *bad, 1, 1)[0] == 2, bad
    assert _size(L.loca_head_loss_workspace_size, 4, 10, 64, 1025)[0] == 2
    assert L.loca_head_loss_workspace_size(4, 10, 64, 0, None) == 1


def test_head_loss_codes(L):
    def fwd(H=F, ldh=64, N=4, d=64, W=F, V=10, y=F, w=None, cols=None, C=0, loss=F, lse=F, E=None, ws=F, n=BIG):
        return L.loca_head_loss(H, ldh, N, d, W, V, y, w, cols, C, loss, lse, E, ws, n, None)

    assert fwd(N=0, H=None, W=None, y=None, loss=None, ws=None, n=0) == 0  # nothing to do
    assert fwd(N=-1) == 2 and fwd(V=0) == 2 and fwd(d=12, ldh=12) == 2
    assert fwd(H=None) == 1 and fwd(W=None) == 1 and fwd(y=None) == 1 and fwd(loss=None) == 1
    assert fwd(E=F, cols=F, C=0) == 2 and fwd(E=F, cols=None, C=3) == 1 and fwd(E=F, cols=F, C=2000) == 2
    assert fwd(ldh=56) == 2 and fwd(ldh=68) == 3 and fwd(H=P(264)) == 3 and fwd(W=P(8)) == 3 and fwd(y=P(2)) == 3
    assert fwd(ws=None) == 7 and fwd(n=16) == 7 and fwd(ws=P(16)) == 3
    assert b"256-byte" in L.loca_last_error_string()

    def bwd(H=F, ldh=64, N=4, d=64, W=F, V=10, y=F, w=None, lse=F, g=None, s=1.0, dH=F, lddh=64, dW=F, ws=F, n=BIG):
        return L.loca_head_loss_backward(H, ldh, N, d, W, V, y, w, lse, g, f(s), dH, lddh, dW, ws, n, None)

    assert bwd(dH=None, dW=None) == 1 and bwd(lse=None) == 1 and bwd(W=None) == 1
    assert bwd(N=0, dW=None) == 0
    assert bwd(lddh=56) == 2 and bwd(lddh=68) == 3 and bwd(dW=P(8)) == 3 and bwd(g=P(2)) == 3
    assert bwd(s=float("inf")) == 1 and bwd(s=float("nan")) == 1
    assert bwd(n=16) == 7


def test_adapter_sizes(L):
    rc, one = _size(L.loca_adapter_packed_size, 1, 896, 1024, 5)
    rc2, many = _size(L.loca_adapter_packed_size, 10, 896, 1024, 5)
    assert rc == 0 and rc2 == 0 and one >= 4 * 2 * 16 * (896 + 1024) and many > 9 * (one - 4096)
    assert _size(L.loca_adapter_plan_size, 0, 1)[0] == 0
    rc, n = _size(L.loca_adapter_plan_size, 1 << 22, 1)
    assert rc == 0 and n >= 2 * 4 * (1 << 22)
    rc, fwd = _size(L.loca_adapter_workspace_size, 8192, 2048, 2048, 32, 8, 0)
    rc2, bwd = _size(L.loca_adapter_workspace_size, 8192, 2048, 2048, 32, 8, 1)
    assert rc == 0 and rc2 == 0 and 0 < fwd < bwd
    for bad in ((0, 64, 64, 4), (70000, 64, 64, 4), (1, 60, 64, 4), (1, 64, 4, 4), (1, 64, 64, 0), (1, 64, 64, 65)):
        assert _size(L.loca_adapter_packed_size, *bad)[0] == 2, bad
    assert _size(L.loca_adapter_plan_size, (1 << 22) + 1, 1)[0] == 2
    assert L.loca_adapter_packed_size(1, 64, 64, 4, None) == 1


def test_adapter_codes(L):
    def pack(A=F, B=F, t=0, n=2, i=64, o=72, k=4, s=None, to=F):
        return L.loca_adapter_pack(A, B, t, n, i, o, k, s, to, None)

    assert pack(t=5) == 4 and pack(k=65) == 2 and pack(A=None) == 1 and pack(to=None) == 1
    assert pack(A=P(2)) == 3 and pack(s=P(2)) == 3 and pack(to=P(64)) == 3
    assert L.loca_adapter_plan(None, 0, 2, None, None) == 0
    assert L.loca_adapter_plan(None, 4, 2, F, None) == 1 and L.loca_adapter_plan(F, 4, 0, F, None) == 2
    assert L.loca_adapter_plan(P(2), 4, 2, F, None) == 3 and L.loca_adapter_plan(F, 4, 2, P(64), None) == 3

    def apply(X=F, ldx=64, N=4, i=64, W=F, o=72, packed=F, n=2, k=4, plan=F, Y=F, ldy=72, ws=F, nb=BIG):
        return L.loca_adapter_apply(X, ldx, N, i, W, o, packed, n, k, plan, Y, ldy, ws, nb, None)

    assert apply(N=0, X=None, W=None, packed=None, plan=None, Y=None, ws=None, nb=0) == 0
    assert apply(X=None) == 1 and apply(W=None) == 1 and apply(plan=None) == 1 and apply(Y=None) == 1
    assert apply(ldx=56) == 2 and apply(ldy=64) == 2 and apply(ldx=68) == 3 and apply(ldy=76) == 3
    assert apply(X=P(8)) == 3 and apply(Y=P(8)) == 3 and apply(W=P(8)) == 3 and apply(plan=P(64)) == 3
    assert apply(ws=None) == 7 and apply(nb=16) == 7

    def back(X=F, ldx=64, dY=F, lddy=72, N=4, i=64, W=F, o=72, packed=F, n=2, k=4, plan=F, dX=F, lddx=64, dA=F, dB=F,
             t=0, ws=F, nb=BIG):
        return L.loca_adapter_backward(X, ldx, dY, lddy, N, i, W, o, packed, n, k, plan, dX, lddx, dA, dB, t, ws, nb,
                                       None)

    assert back(dX=None, dA=None, dB=None) == 1 and back(t=9) == 4 and back(dY=None) == 1
    assert back(lddx=56) == 2 and back(lddx=68) == 3 and back(dA=P(2)) == 3 and back(dB=P(1), t=1) == 3
    assert back(nb=16) == 7


def test_grad_clip_codes(L):
    def call(ptr=(256, 512), out=None, numel=(10, 20), dtype=(0, 1), n=2, m=1.0, norm=F, ws=F, nb=BIG):
        a = (P * 2)(*ptr)
        o = None if out is None else (P * 2)(*out)
        return L.loca_grad_clip(a, o, (ctypes.c_int64 * 2)(*numel), (ctypes.c_int32 * 2)(*dtype), n, f(m), norm, ws, nb,
                                None)

    assert _size(L.loca_grad_clip_workspace_size, 0)[0] == 0
    assert _size(L.loca_grad_clip_workspace_size, 100000)[1] > _size(L.loca_grad_clip_workspace_size, 10)[1] > 0
    assert _size(L.loca_grad_clip_workspace_size, -1)[0] == 2 and _size(L.loca_grad_clip_workspace_size, 100001)[0] == 2
    assert call(n=-1) == 2 and call(numel=(-1, 3)) == 2 and call(numel=(10, 1 << 50)) == 2
    assert call(m=0.0) == 1 and call(m=float("nan")) == 1 and call(norm=None) == 1 and call(ptr=(256, None)) == 1
    assert call(out=(256, None)) == 1 and call(dtype=(0, 2)) == 4
    assert call(ptr=(258, 512)) == 3 and call(out=(256, 513)) == 3 and call(norm=P(2)) == 3
    assert call(nb=8) == 7
