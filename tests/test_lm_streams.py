"""Calls on a stream given by ``stream=`` while other work goes on on the current one: scratch memory
that a call allocates belongs to the stream it runs on, and one handle used on two streams keeps two."""

import contextlib

import pytest
import torch


def test_scratch_memory_is_allocated_under_the_calls_stream(monkeypatch):
    from paper_2608_03020_gb300 import loca

    class Stream:
        cuda_stream = 0x1234

    seen, inside = [], []

    @contextlib.contextmanager
    def under(s):
        inside.append(s)
        yield
        inside.pop()

    def empty(n, **kw):
        seen.append((n, inside[-1].handle if inside else None))
        return "memory"

    class External:
        def __init__(self, handle):
            self.handle = handle

    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(torch.cuda, "ExternalStream", External)
    monkeypatch.setattr(torch, "empty", empty)
    assert loca._workspace(512, "cuda", None, Stream()) == "memory"
    assert loca._workspace(256, "cuda") == "memory"
    assert loca._workspace(0, "cuda", None, Stream()) is None
    assert seen == [(512, 0x1234), (256, None)]


@pytest.fixture(scope="module")
def lc():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_03020_gb300 import _build

    _build.build()
    from paper_2608_03020_gb300 import loca

    loca.lib()
    return loca


def _busy(stream):
    """Some milliseconds of work in front of what comes next on `stream`."""
    with torch.cuda.stream(stream):
        a = torch.zeros((8192, 8192), device="cuda")
        for _ in range(4):
            a = a @ a
    return a


def _fill():
    """Takes memory of many sizes on the current stream and overwrites it."""
    return [torch.full((1 << e,), -1, dtype=torch.uint8, device="cuda") for e in range(9, 28) for _ in range(3)]


@pytest.mark.gpu
@pytest.mark.parametrize("N", [40, 700])
def test_calls_beside_the_current_stream(lc, N):
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    d, V, o, k, n = 256, 3000, 320, 8, 3
    H, head = rn(N, d).to(torch.bfloat16), (rn(V, d) / 16).to(torch.bfloat16)
    y = torch.randint(-1, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    W, dY = (rn(o, d) / 16).to(torch.bfloat16), rn(N, o).to(torch.bfloat16)
    A, B = rn(n, d, k) / 16, rn(n, o, k)
    ids = torch.randint(-1, n, (N,), generator=g, device="cuda", dtype=torch.int32)

    def calls(stream):
        out = [torch.empty((N,), device="cuda"), torch.empty((N,), device="cuda"), torch.empty_like(H),
               torch.empty_like(head), torch.empty_like(dY), torch.empty_like(H), torch.empty_like(A), torch.empty_like(B)]
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
            keep.append(_busy(stream))
        lc.loca_head_loss(H, head, y, out[0], lse=out[1], stream=stream)
        lc.loca_head_loss_backward(H, head, y, out[1], dH=out[2], dW=out[3], stream=stream)
        ad = lc.AdapterSet(n, d, o, k).pack(A, B, stream=stream)
        plan = lc.AdapterPlan(ids, n, stream=stream)
        lc.loca_adapter_apply(H, W, ad, plan, out[4], stream=stream)
        lc.loca_adapter_backward(H, dY, W, ad, plan, dX=out[5], dA=out[6], dB=out[7], stream=stream)
        return out

    keep = []
    want = calls(None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = calls(s)  # the set and the plan go out of scope while their calls wait
    keep.append(_fill())
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0
    for i, (a, b) in enumerate(zip(want, got)):
        assert torch.equal(a, b), i


@pytest.mark.gpu
def test_one_clip_handle_on_two_streams(lc):
    grads = [torch.randn((100000 + 7 * i,), device="cuda") for i in range(20)]
    clip = lc.GradClip(grads)  # in place: without a limit nothing is written but the norm
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    norms = [torch.zeros((1,), device="cuda") for _ in range(3)]
    clip.run(float("inf"), norms[2])
    torch.cuda.synchronize()
    for _ in range(50):
        for s, norm in zip(streams, norms):
            clip.run(float("inf"), norm, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(norms[0], norms[2]) and torch.equal(norms[1], norms[2])
    assert len({t.data_ptr() for t in clip._ws.values()}) == 3
