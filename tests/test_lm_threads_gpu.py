"""Calls from several host threads at once, each on its own stream with its own workspace: what one
thread's launch asks for (shared memory, cluster size) must not reach another's."""

import threading

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


# name: N, d, o, k, n: token by token, one tile of slots, few tokens by slots, many tokens; their kernels
# take different amounts of shared memory
CALLS = {
    "tokens": (64, 1024, 512, 16, 64),
    "one tile": (100, 1024, 512, 16, 2),
    "several tiles": (400, 512, 512, 64, 2),
    "many": (3000, 256, 1024, 40, 3),
}


def _program(lc, N, d, o, k, n, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    X, W, dY = rn(N, d).to(torch.bfloat16), (rn(o, d) / d ** 0.5).to(torch.bfloat16), rn(N, o).to(torch.bfloat16)
    A, B = rn(n, d, k) / d ** 0.5, rn(n, o, k)
    ids = torch.randint(0, n, (N,), generator=g, device="cuda", dtype=torch.int32)
    ad, plan = lc.AdapterSet(n, d, o, k).pack(A, B), lc.AdapterPlan(ids, n)
    ws = torch.empty(lc.adapter_workspace_size(N, d, o, k, n, backward=True), dtype=torch.uint8, device="cuda")
    Y, dX, dA = torch.empty_like(dY), torch.empty_like(X), torch.empty_like(A)

    def call():
        lc.loca_adapter_apply(X, W, ad, plan, Y, workspace=ws)
        lc.loca_adapter_backward(X, dY, W, ad, plan, dX=dX, dA=dA, workspace=ws)
        return Y, dX, dA

    return call


def test_threads_with_calls_of_different_sizes(lc):
    programs = [_program(lc, *sizes, seed=i) for i, sizes in enumerate(CALLS.values())]
    want = [[t.clone() for t in p()] for p in programs]
    torch.cuda.synchronize()
    failed, start = [], threading.Barrier(len(programs))

    def work(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                start.wait(timeout=60)
                for _ in range(1500):
                    got = programs[i]()
                s.synchronize()
                for a, b in zip(want[i], got):
                    assert torch.equal(a, b), list(CALLS)[i]
        except Exception as e:  # noqa: BLE001 (reported below)
            failed.append((list(CALLS)[i], repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(programs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    assert lc.loca_device_status() == 0
