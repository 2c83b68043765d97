"""Memory that outlives its names: what a 4-bit weight is packed from, and the layouts of weights, adapters and plans,
dropped while calls on another stream still wait for their turn.  The allocator may not hand it out before they are done."""

import ctypes

import pytest
import torch


class _Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.fixture
def marks(monkeypatch):
    """The binding over host tensors and a library that does nothing: (tensor, stream handle) of every record."""
    from paper_2608_03020_gb300 import loca

    class Lib:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith("_size"):
                    args[-1]._obj.value = 512
                return 0

            return call

    seen = []
    current = _Stream(7)
    monkeypatch.setattr(loca, "lib", lambda: Lib())
    monkeypatch.setattr(loca, "_dev", lambda *a: None)
    monkeypatch.setattr(loca, "_same_device", lambda *a: None)
    monkeypatch.setattr(loca, "_rows2d", lambda t, *a: t.stride(0))
    monkeypatch.setattr(loca, "_size", lambda *a: 512)
    monkeypatch.setattr(loca, "_empty", lambda n, device, stream=None: torch.empty(n, dtype=torch.uint8))
    monkeypatch.setattr(loca, "_stream", lambda s: ctypes.c_void_p((current if s is None else s).cuda_stream))
    monkeypatch.setattr(loca, "_torch_stream", lambda s: s)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: current)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: seen.append((t.data_ptr(), s.cuda_stream)), raising=False)
    return loca, seen


def _weight(loca, stream=None, zeros=True):
    codes = torch.zeros((64, 64), dtype=torch.uint8)
    scales = torch.zeros((64, 4))
    z = torch.zeros((64, 4), dtype=torch.uint8) if zeros else None
    return loca.Q4Weight(codes, scales, z, stream=stream), [t.data_ptr() for t in (codes, scales, z) if t is not None]


@pytest.mark.parametrize("zeros", [True, False])
def test_what_a_weight_is_packed_from(marks, zeros):
    loca, seen = marks
    _, args = _weight(loca, _Stream(9), zeros)
    assert set(seen) >= {(p, 9) for p in args}
    seen.clear()
    _, args = _weight(loca, None, zeros)
    assert set(seen) >= {(p, 7) for p in args}


def test_layouts_used_on_other_streams(marks):
    loca, seen = marks
    X, Y = torch.zeros((3, 128), dtype=torch.bfloat16), torch.zeros((3, 64), dtype=torch.bfloat16)
    W, ids = torch.zeros((64, 128), dtype=torch.bfloat16), torch.zeros((3,), dtype=torch.int32)
    weight, _ = _weight(loca, _Stream(9))
    plan = loca.AdapterPlan(ids, 2, stream=_Stream(9))
    adapters = object.__new__(loca.AdapterSet)
    adapters.n, adapters.d_in, adapters.d_out, adapters.k = 2, 128, 64, 4
    adapters.packed = torch.zeros(512, dtype=torch.uint8)
    adapters._memory = loca._Owned(adapters.packed)  # on the current stream
    w, p, a = weight.packed.data_ptr(), plan.buf.data_ptr(), adapters.packed.data_ptr()
    seen.clear()
    loca.loca_q4_apply(X, weight, Y, adapters, plan)  # on the current stream
    assert sorted(seen) == sorted([(w, 7), (p, 7)])
    loca.loca_q4_apply(X, weight, Y, adapters, plan)  # known by now
    loca.loca_adapter_apply(X, W, adapters, plan, Y)
    assert len(seen) == 2
    loca.loca_q4_apply(X, weight, Y, adapters, plan, stream=_Stream(9))
    assert seen[2:] == [(a, 9)]
    loca.loca_adapter_apply(X, W, adapters, plan, Y, stream=_Stream(11))
    assert sorted(seen[3:]) == sorted([(a, 11), (p, 11)])
    seen.clear()
    plan.update(ids, stream=_Stream(13))
    adapters.pack(torch.zeros((2, 128, 4)), torch.zeros((2, 64, 4)), stream=_Stream(13))
    assert sorted(seen) == sorted([(p, 13), (a, 13)])
    seen.clear()
    loca.loca_adapter_backward(X, Y, W, adapters, plan, dX=torch.zeros_like(X), stream=_Stream(15))
    assert sorted(seen) == sorted([(p, 15), (a, 15)])


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


def _fill(stream):
    """Takes memory of many sizes of a stream's and overwrites it there."""
    with torch.cuda.stream(stream):
        return [torch.full((1 << e,), -1, dtype=torch.uint8, device="cuda") for e in range(9, 26) for _ in range(3)]


@pytest.mark.gpu
@pytest.mark.parametrize("N", [3, 40])
def test_dropped_while_calls_wait(lc, N):
    o, d, group, k, n = 264, 512, 64, 8, 3
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    codes = torch.randint(0, 256, (o, d // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales, zeros = rn(o, d // group), torch.randint(0, 16, (o, d // group), generator=g, device="cuda", dtype=torch.uint8)
    X, A, B = rn(N, d).to(torch.bfloat16), rn(n, d, k) / 16, rn(n, o, k)
    ids = torch.randint(-1, n, (N,), generator=g, device="cuda", dtype=torch.int32)
    adapters = lc.AdapterSet(n, d, o, k).pack(A, B)
    want, got, later = (torch.zeros((N, o), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    lc.loca_q4_apply(X, lc.Q4Weight(codes, scales, zeros), want, adapters, lc.AdapterPlan(ids, n))
    torch.cuda.synchronize()
    here, side = torch.cuda.current_stream(), torch.cuda.Stream()
    keep = [_busy(side)]
    # packed on the other stream from tensors of this one that nobody holds any more
    parts = [t.clone() for t in (codes, scales, zeros)]
    side.wait_stream(here)
    weight = lc.Q4Weight(*parts, stream=side)
    del parts
    keep.append(_fill(here))
    plan = lc.AdapterPlan(ids, n, stream=side)
    torch.cuda.synchronize()
    # used on this stream, memory of the other one
    keep.append(_busy(here))
    lc.loca_q4_apply(X, weight, got, adapters, plan)
    del weight, plan
    keep.append(_fill(side))
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    # and a weight whose whole life waits on the other stream
    keep.append(_busy(side))
    parts = [t.clone() for t in (codes, scales, zeros)]
    side.wait_stream(here)
    lc.loca_q4_apply(X, lc.Q4Weight(*parts, stream=side), later, adapters, lc.AdapterPlan(ids, n, stream=side), stream=side)
    del parts
    keep += [_fill(here), _fill(side)]
    torch.cuda.synchronize()
    assert torch.equal(later, want) and lc.loca_device_status() == 0
