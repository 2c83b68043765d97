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


def _arguments(lc, N, d, o, k, n, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    m = dict(X=rn(N, d).to(torch.bfloat16), W=(rn(o, d) / d ** 0.5).to(torch.bfloat16))
    ids = torch.randint(0, n, (N,), generator=g, device="cuda", dtype=torch.int32)
    m["set"] = lc.AdapterSet(n, d, o, k).pack(rn(n, d, k) / d ** 0.5, rn(n, o, k))
    m["plan"] = lc.AdapterPlan(ids, n)
    m["ws"] = torch.empty(lc.adapter_workspace_size(N, d, o, k, n), dtype=torch.uint8, device="cuda")
    m["Y"] = torch.empty((N, o), dtype=torch.bfloat16, device="cuda")
    p = lc._ptr
    m["args"] = (p(m["X"]), d, N, d, p(m["W"]), o, p(m["set"].packed), n, k, p(m["plan"].buf), p(m["Y"]), o, p(m["ws"]),
                 m["ws"].numel())
    torch.cuda.synchronize()
    return m


def test_threads_with_calls_of_different_sizes(lc):
    """The C calls in a tight loop (the interpreter's lock is free while they run): the same kernel with
    206 KB of shared memory from one thread and with 110 KB from another."""
    names = ["tokens", "one tile", "tokens", "one tile"]
    made = [_arguments(lc, *CALLS[name], seed=i) for i, name in enumerate(names)]
    fn = lc.lib().loca_adapter_apply
    for m in made:
        assert fn(*m["args"], lc._stream(None)) == 0
    torch.cuda.synchronize()
    want = [m["Y"].clone() for m in made]
    codes, start = [{} for _ in names], threading.Barrier(len(names))

    def work(i):
        s = torch.cuda.Stream()
        args = (*made[i]["args"], lc._stream(s))
        start.wait(timeout=60)
        for _ in range(100):
            for _ in range(100):
                rc = fn(*args)
                codes[i][rc] = codes[i].get(rc, 0) + 1
            s.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(names))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert codes == [{0: 10000}] * len(names), codes
    assert all(torch.equal(w, m["Y"]) for w, m in zip(want, made))
    assert lc.loca_device_status() == 0


@pytest.mark.parametrize("name", sorted(CALLS))
def test_first_cuda_call_of_a_thread(lc, name):
    """A host thread that has made no CUDA call has no current context yet."""
    m = _arguments(lc, *CALLS[name], seed=1)
    args = (*m["args"], lc._stream(None))
    assert lc.lib().loca_adapter_apply(*args) == 0
    torch.cuda.synchronize()
    want, codes = m["Y"].clone(), []
    m["Y"].zero_()
    torch.cuda.synchronize()
    t = threading.Thread(target=lambda: codes.append(lc.lib().loca_adapter_apply(*args)))
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert codes == [0]
    assert torch.equal(want, m["Y"]) and lc.loca_device_status() == 0
