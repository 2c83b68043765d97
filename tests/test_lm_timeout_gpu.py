"""The failure path of the bounded waits in the head loss and the adapted projection, without a GPU
fault: a wait limit of 1 us (loca_set_wait_limit) makes a wait that has not succeeded after 8 polls
give up.  The kernel must record LOCA_ERR_TIMEOUT, let its copies and MMAs land, free its tensor memory
and return; with the default limit restored the same call gives the bits it gave before.  A call whose
waits all succeed within 8 polls finishes normally and must match; the call is repeated until one
gives up.
"""

import pytest
import torch

pytestmark = pytest.mark.gpu

LOCA_ERR_TIMEOUT = 6


@pytest.fixture(scope="module")
def lc():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_03020_gb300 import _build

    _build.build()
    from paper_2608_03020_gb300 import loca

    loca.lib()
    yield loca
    loca.loca_set_wait_limit(0)


def _head(lc, N, d, V, backward):
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    H = torch.randn((N, d), generator=g, device="cuda").to(torch.bfloat16)
    W = (torch.randn((V, d), generator=g, device="cuda") / d ** 0.5).to(torch.bfloat16)
    y = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    lse = torch.logsumexp(H.float() @ W.float().T, 1)
    nf = lc.head_loss_workspace_size(N, V, d)
    nb = lc.head_loss_backward_workspace_size(N, V, d)
    ws = torch.zeros(max(nf, nb), dtype=torch.uint8, device="cuda")

    def call():
        if backward:
            out = [torch.empty((N, d), dtype=torch.bfloat16, device="cuda"), torch.empty_like(W)]
            lc.loca_head_loss_backward(H, W, y, lse, dH=out[0], dW=out[1], workspace=ws)
        else:
            out = [torch.empty((N,), device="cuda"), torch.empty((N,), device="cuda")]
            lc.loca_head_loss(H, W, y, out[0], lse=out[1], workspace=ws)
        torch.cuda.synchronize()
        return out

    return call


def _adapter(lc, N, d, o, k, n, backward):
    g = torch.Generator(device="cuda")
    g.manual_seed(N + n)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    X, W, dY = rn(N, d).to(torch.bfloat16), (rn(o, d) / d ** 0.5).to(torch.bfloat16), rn(N, o).to(torch.bfloat16)
    A, B = rn(n, d, k) / d ** 0.5, rn(n, o, k)
    ids = torch.randint(-1, n, (N,), generator=g, device="cuda", dtype=torch.int32)
    ad = lc.AdapterSet(n, d, o, k).pack(A, B)
    plan = lc.AdapterPlan(ids, n)
    ws = torch.zeros(lc.adapter_workspace_size(N, d, o, k, n, backward=backward), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()

    def call():
        if backward:
            out = [torch.empty_like(X), torch.empty_like(A), torch.empty_like(B)]
            lc.loca_adapter_backward(X, dY, W, ad, plan, dX=out[0], dA=out[1], dB=out[2], workspace=ws)
        else:
            out = [torch.empty_like(dY)]
            lc.loca_adapter_apply(X, W, ad, plan, out[0], workspace=ws)
        torch.cuda.synchronize()
        return out

    return call


# name: (call, whether it has waits so long that one must give up: a tile of many k-blocks)
CASES = {
    "head": (lambda lc: _head(lc, 2000, 1024, 20000, False), False),
    "head backward": (lambda lc: _head(lc, 1000, 16384, 8000, True), True),
    "head, few tokens": (lambda lc: _head(lc, 64, 2048, 30000, False), False),
    "head backward, few tokens": (lambda lc: _head(lc, 64, 2048, 30000, True), False),
    "adapters": (lambda lc: _adapter(lc, 3000, 16384, 2048, 16, 3, False), True),
    "adapters backward": (lambda lc: _adapter(lc, 3000, 2048, 16384, 16, 3, True), True),
    "adapters, one tile by slots": (lambda lc: _adapter(lc, 100, 65536, 2048, 16, 3, False), True),
    "adapters, token by token": (lambda lc: _adapter(lc, 64, 65536, 2048, 16, 64, False), True),
    "adapters backward, one tile": (lambda lc: _adapter(lc, 100, 4096, 2048, 16, 3, True), False),
}


@pytest.mark.parametrize("case", sorted(CASES))
def test_wait_timeout_is_reported_and_the_next_call_is_right(lc, case):
    lc.loca_set_wait_limit(0)
    assert lc.loca_device_status() == 0
    make, must = CASES[case]
    call = make(lc)
    ref = call()
    assert lc.loca_device_status() == 0
    timed_out = False
    for attempt in range(20):
        lc.loca_set_wait_limit(1000)
        out = call()
        status = lc.loca_device_status()
        lc.loca_set_wait_limit(0)
        if status == LOCA_ERR_TIMEOUT:
            timed_out = True
            again = call()
            assert lc.loca_device_status() == 0
            for a, b in zip(ref, again):
                assert torch.equal(a, b), case
        else:
            assert status == 0, (case, attempt, status)
            for a, b in zip(ref, out):
                assert torch.equal(a, b), (case, attempt)
    assert timed_out or not must, case
