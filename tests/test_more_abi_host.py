"""Host-side checks of the gated feed-forward, distillation and 4-bit entry points (no GPU needed): sizes, and
argument validation that rejects bad calls with the documented codes before any CUDA call."""

import ctypes

import pytest

P = ctypes.c_void_p
BIG = 1 << 40


def at(i):
    """An address that is never dereferenced: validation fails first.  Buffers lie 16 MB apart."""
    return P((i + 1) << 24)


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


def test_gated_sizes(L):
    assert _size(L.loca_gated_workspace_size, 4096, 2048, 8192) == (0, 256)
    rc, n = _size(L.loca_gated_backward_workspace_size, 4096, 2048, 8192, 1, 1)
    # dG and dU in bf16, and the k ranges of dX in fp32
    assert rc == 0 and 4 * 4096 * 8192 <= n <= 4 * 4096 * 8192 + 32 * 4 * 4096 * 2048 + 4096
    rc, rows = _size(L.loca_gated_backward_workspace_size, 1 << 20, 2048, 8192, 1, 0)
    assert rc == 0 and rows < (1 << 30) + 32 * 4 * 32768 * 2048 + 4096
    rc, cols = _size(L.loca_gated_backward_workspace_size, 1 << 20, 2048, 8192, 0, 1)
    assert rc == 0 and cols <= (4 << 30) + 4096
    for bad in ((-1, 64, 64), (4, 60, 64), (4, 64, 60), (4, 0, 64), (4, 64, 65544), ((1 << 24) + 1, 64, 64)):
        assert _size(L.loca_gated_workspace_size, *bad)[0] == 2, bad
        assert _size(L.loca_gated_backward_workspace_size, *bad, 1, 1)[0] == 2, bad
    assert L.loca_gated_workspace_size(4, 64, 64, None) == 1


def test_gated_codes(L):
    def fwd(X=at(0), ldx=64, N=4, d=64, Wg=at(1), Wu=at(2), f=72, act=0, H=at(3), ldh=72, ws=at(4), n=BIG):
        return L.loca_gated(X, ldx, N, d, Wg, Wu, f, act, H, ldh, ws, n, None)

    assert fwd(N=0, X=None, Wg=None, Wu=None, H=None, ws=None, n=0) == 0  # nothing to do
    assert fwd(N=-1) == 2 and fwd(d=12) == 2 and fwd(f=12) == 2 and fwd(act=2) == 1 and fwd(act=-1) == 1
    assert fwd(X=None) == 1 and fwd(Wg=None) == 1 and fwd(Wu=None) == 1 and fwd(H=None) == 1
    assert fwd(ldx=56) == 2 and fwd(ldh=64) == 2 and fwd(ldx=68) == 3 and fwd(ldh=76) == 3
    assert fwd(X=P(8)) == 3 and fwd(Wg=P(8)) == 3 and fwd(Wu=P(8)) == 3 and fwd(H=P(8)) == 3
    assert fwd(ws=None) == 7 and fwd(n=16) == 7 and fwd(ws=P(16)) == 3
    assert fwd(H=at(0)) == 1 and fwd(H=at(1)) == 1 and fwd(H=at(2)) == 1
    # rows side by side share no byte, rows that reach into each other do
    assert fwd(H=P(at(0).value + 128), ldx=136, ldh=136, ws=None) == 7
    assert fwd(H=P(at(0).value + 112), ldx=136, ldh=136) == 1

    def back(X=at(0), ldx=64, N=4, d=64, Wg=at(1), Wu=at(2), f=72, act=0, dH=at(3), lddh=72, dX=at(4), lddx=64, dWg=at(5),
             dWu=at(6), ws=at(7), n=BIG):
        return L.loca_gated_backward(X, ldx, N, d, Wg, Wu, f, act, dH, lddh, dX, lddx, dWg, dWu, ws, n, None)

    assert back(N=0, X=None, Wg=None, Wu=None, dH=None, dWg=None, dWu=None, ws=None, n=0) == 0
    assert back(dX=None, dWg=None, dWu=None) == 1 and back(act=7) == 1
    assert back(X=None) == 1 and back(dH=None) == 1 and back(Wg=None) == 1 and back(Wu=None) == 1
    assert back(lddh=64) == 2 and back(lddx=56) == 2 and back(lddx=68) == 3 and back(dWg=P(8)) == 3 and back(dWu=P(8)) == 3
    assert back(n=256) == 7 and back(ws=None) == 7
    for out in ("dX", "dWg", "dWu"):
        for inp in (0, 1, 2, 3):
            assert back(**{out: at(inp)}) == 1, (out, inp)
    assert back(dWu=at(5)) == 1 and back(dX=at(5)) == 1 and back(dX=at(6)) == 1


def test_distill_sizes(L):
    rc, n = _size(L.loca_head_distill_workspace_size, 4096, 151936, 5120, 64)
    # the hidden states once, two pairs of floats per row and 256 columns, three words' worth per entry, and the
    # table's two bytes per row and 128 columns (1188 of them, kept to a multiple of 8)
    table = 2 * 1192
    assert rc == 0 and 4096 * 5120 * 2 < n < 4096 * (5120 * 2 + 16 * 594 + 12 * 64 + table) + (1 << 20)
    rc, b = _size(L.loca_head_distill_backward_workspace_size, 1 << 17, 151936, 5120, 64, 1, 0)
    assert rc == 0 and b < (1 << 30) + (1 << 17) * (5120 * 2 + 64 * 8 + table) + 32 * 8192 * 5120 * 4 + (1 << 22)
    for bad in ((-1, 10, 64, 4), (4, 0, 64, 4), (4, 10, 60, 4), (4, 10, 64, 0), (4, 10, 64, 257), (1 << 25, 10, 64, 4)):
        assert _size(L.loca_head_distill_workspace_size, *bad)[0] == 2, bad
        assert _size(L.loca_head_distill_backward_workspace_size, *bad, 1, 1)[0] == 2, bad
    assert L.loca_head_distill_workspace_size(4, 10, 64, 2, None) == 1


def test_distill_codes(L):
    f = ctypes.c_float

    def fwd(H=at(0), ldh=64, N=4, d=64, W=at(1), V=10, idx=at(2), t=at(3), K=3, tau=1.0, w=None, loss=at(4), lse=at(5),
            ws=at(6), n=BIG):
        return L.loca_head_distill(H, ldh, N, d, W, V, idx, t, K, f(tau), w, loss, lse, ws, n, None)

    assert fwd(N=0, H=None, W=None, idx=None, t=None, loss=None, ws=None, n=0) == 0  # nothing to do
    assert fwd(N=-1) == 2 and fwd(V=0) == 2 and fwd(d=12) == 2 and fwd(K=0) == 2 and fwd(K=257) == 2
    assert fwd(tau=0.0) == 1 and fwd(tau=float("nan")) == 1 and fwd(tau=float("inf")) == 1 and fwd(tau=-1.0) == 1
    assert fwd(H=None) == 1 and fwd(W=None) == 1 and fwd(idx=None) == 1 and fwd(t=None) == 1 and fwd(loss=None) == 1
    assert fwd(ldh=56) == 2 and fwd(ldh=68) == 3 and fwd(H=P(8)) == 3 and fwd(W=P(8)) == 3
    assert fwd(idx=P(2)) == 3 and fwd(t=P(2)) == 3 and fwd(loss=P(2)) == 3 and fwd(lse=P(2)) == 3 and fwd(w=P(2)) == 3
    assert fwd(ws=None) == 7 and fwd(n=16) == 7 and fwd(ws=P(16)) == 3

    def back(H=at(0), ldh=64, N=4, d=64, W=at(1), V=10, idx=at(2), t=at(3), K=3, tau=1.0, w=None, lse=at(4), g=None, s=1.0,
             dH=at(5), lddh=64, dW=at(6), ws=at(7), n=BIG):
        return L.loca_head_distill_backward(H, ldh, N, d, W, V, idx, t, K, f(tau), w, lse, g, f(s), dH, lddh, dW, ws, n, None)

    assert back(dH=None, dW=None) == 1 and back(lse=None) == 1 and back(H=None) == 1 and back(idx=None) == 1
    assert back(N=0, H=None, W=None, idx=None, t=None, lse=None, dW=None, ws=None, n=0) == 0
    assert back(s=float("nan")) == 1 and back(tau=0.0) == 1
    assert back(lddh=56) == 2 and back(lddh=68) == 3 and back(dW=P(8)) == 3 and back(g=P(2)) == 3 and back(lse=P(2)) == 3
    assert back(n=256) == 7
    assert back(dH=at(0), ws=None) == 7  # over H itself: allowed
    assert back(dH=P(at(0).value + 16)) == 1 and back(dW=at(0)) == 1 and back(dW=at(1)) == 1 and back(dH=at(1)) == 1
    assert back(dH=at(6)) == 1


@pytest.mark.parametrize("tau", [1e-39, 1e-45, 2e19, 3e38])
def test_temperatures_whose_square_or_reciprocal_is_not_finite(L, tau):
    one, f = at(0), ctypes.c_float
    assert L.loca_head_distill(one, 64, 4, 64, at(1), 10, at(2), at(3), 3, f(tau), None, at(4), at(5), at(6), BIG, None) == 1
    assert L.loca_head_distill_backward(one, 64, 4, 64, at(1), 10, at(2), at(3), 3, f(tau), None, at(4), None, f(1.0), at(5), 64,
                                        at(6), at(7), BIG, None) == 1


def test_q4_sizes(L):
    rc, n = _size(L.loca_q4_packed_size, 20480, 5120, 64, 1, 1)
    # four bits a code, a scale and half a byte of zero for each group
    want = 20480 * 5120 // 2 + 20480 * 80 * 2 + 20480 * 80 // 2
    assert rc == 0 and want <= n <= want + 1024
    assert _size(L.loca_q4_packed_size, 20480, 5120, 64, 0, 0)[1] > n
    for bad in ((0, 64, 32), (64, 0, 32), (64, 48, 32), (64, 64, 16), (64, 64, 128), (64, 65568, 32), ((1 << 24) + 1, 64, 32)):
        assert _size(L.loca_q4_packed_size, *bad, 0, 0)[0] == 2, bad
    assert _size(L.loca_q4_packed_size, 64, 64, 32, 3, 0)[0] == 4
    assert _size(L.loca_q4_workspace_size, 64, 5120, 20480, 0, 0) == (0, 256)
    rc, n = _size(L.loca_q4_workspace_size, 64, 5120, 20480, 16, 4)
    assert rc == 0 and n >= 64 * 16 * 4
    assert _size(L.loca_q4_workspace_size, 64, 5120, 20481, 16, 4)[0] == 2  # adapters want multiples of 8
    assert _size(L.loca_q4_workspace_size, 65536, 5120, 20480, 0, 0)[0] == 2
    assert _size(L.loca_q4_workspace_size, 64, 5120, 20480, 65, 4)[0] == 2
    assert L.loca_q4_packed_size(64, 64, 32, 0, 0, None) == 1 and L.loca_q4_workspace_size(4, 64, 64, 0, 0, None) == 1


def test_q4_codes(L):
    def pack(codes=at(0), scales=at(1), t=0, zeros=None, o=72, d=64, group=32, to=at(2)):
        return L.loca_q4_pack(codes, scales, t, zeros, o, d, group, to, None)

    assert pack(codes=None) == 1 and pack(scales=None) == 1 and pack(to=None) == 1
    assert pack(t=2) == 4 and pack(group=48) == 2 and pack(d=96, group=64) == 2 and pack(o=0) == 2
    assert pack(scales=P(2)) == 3 and pack(scales=P(1), t=1) == 3 and pack(to=P(16)) == 3

    def run(X=at(0), ldx=64, N=4, d=64, w=at(1), o=72, group=32, t=0, z=0, ad=at(2), n=2, k=4, plan=at(3), Y=at(4), ldy=72,
            ws=at(5), nb=BIG):
        return L.loca_q4_apply(X, ldx, N, d, w, o, group, t, z, ad, n, k, plan, Y, ldy, ws, nb, None)

    assert run(N=0, X=None, w=None, Y=None, ws=None, nb=0) == 0  # nothing to do
    assert run(N=-1) == 2 and run(N=65536) == 2 and run(group=16) == 2 and run(t=5) == 4 and run(d=80, ldx=80) == 2
    assert run(ad=None) == 1 and run(plan=None) == 1 and run(ad=None, plan=None) == 1 and run(ad=None, plan=None, n=0) == 1
    assert run(o=73, ldy=80) == 2 and run(k=65) == 2 and run(n=0) == 2  # adapters' own limits
    assert run(X=None) == 1 and run(w=None) == 1 and run(Y=None) == 1
    assert run(ldx=56) == 2 and run(ldx=68) == 3 and run(ldy=71) == 2 and run(X=P(8)) == 3 and run(Y=P(1)) == 3
    assert run(w=P(16)) == 3 and run(ad=P(16)) == 3 and run(plan=P(16)) == 3
    assert run(ws=None) == 7 and run(nb=16) == 7
    assert run(Y=at(0)) == 1
