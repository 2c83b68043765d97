"""The head loss, the adapted projection and gradient clipping through the LOCA_DEBUG build: every
output, workspace, packed set and plan lies between two poisoned guard bands that must stay intact,
no index check may fail, and the results must equal the release build's.
"""

import pytest
import torch

pytestmark = pytest.mark.gpu

GUARD = 16384
POISON = 0xA5


@pytest.fixture(scope="module")
def lc():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_03020_gb300 import _build

    _build.build()
    _build.build(debug=True)
    from paper_2608_03020_gb300 import loca

    loca.use_debug_library(False)
    yield loca
    loca.use_debug_library(False)


class Guarded:
    def __init__(self, lc):
        self.lc, self.bufs = lc, []

    def empty(self, shape, dtype):
        n = torch.Size(shape).numel() * torch.empty((), dtype=dtype).element_size()
        raw = torch.full((n + 2 * GUARD,), POISON, dtype=torch.uint8, device="cuda")
        self.bufs.append((raw, n))
        return raw[GUARD:GUARD + n].view(dtype).view(shape)

    def check(self, where):
        torch.cuda.synchronize()
        for i, (raw, n) in enumerate(self.bufs):
            assert bool((raw[:GUARD] == POISON).all()), f"{where}: memory before buffer {i} written"
            assert bool((raw[GUARD + n:] == POISON).all()), f"{where}: memory behind buffer {i} written"
        status = self.lc.loca_device_status()
        assert status == 0, f"{where}: device status {status}: {self.lc.loca_last_error()}"


def _head(lc, mk, N, d, V, C):
    g = torch.Generator(device="cuda")
    g.manual_seed(N + d)
    H = torch.randn((N, d), generator=g, device="cuda").to(torch.bfloat16)
    W = (torch.randn((V, d), generator=g, device="cuda") / d ** 0.5).to(torch.bfloat16)
    y = torch.randint(-1, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    cols = torch.arange(C, device="cuda", dtype=torch.int32) * (V // C)
    o = {"loss": mk.empty((N,), torch.float32), "lse": mk.empty((N,), torch.float32), "E": mk.empty((N, C), torch.float32),
         "dH": mk.empty((N, d), torch.bfloat16), "dW": mk.empty((V, d), torch.bfloat16)}
    ws = mk.empty((lc.head_loss_workspace_size(N, V, d, C),), torch.uint8)
    lc.loca_head_loss(H, W, y, o["loss"], lse=o["lse"], label_cols=cols, E=o["E"], workspace=ws)
    mk.check("loca_head_loss")
    ws = mk.empty((lc.head_loss_backward_workspace_size(N, V, d),), torch.uint8)
    lc.loca_head_loss_backward(H, W, y, o["lse"], dH=o["dH"], dW=o["dW"], workspace=ws)
    mk.check("loca_head_loss_backward")
    return o


def _adapters(lc, mk, N, d, out, k, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(N + k)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    X, W, dY = rn(N, d).to(torch.bfloat16), rn(out, d).to(torch.bfloat16), rn(N, out).to(torch.bfloat16)
    A, B = rn(n, d, k), rn(n, out, k)
    ids = torch.randint(-1, n + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
    ad = lc.AdapterSet(n, d, out, k)
    ad.packed = mk.empty(ad.packed.shape, torch.uint8)
    ad.pack(A, B)
    plan = lc.AdapterPlan(ids, n)
    plan.buf = mk.empty(plan.buf.shape, torch.uint8)
    plan.update(ids)
    mk.check("loca_adapter_pack, loca_adapter_plan")
    o = {"Y": mk.empty((N, out), torch.bfloat16), "dX": mk.empty((N, d), torch.bfloat16),
         "dA": mk.empty((n, d, k), torch.float32), "dB": mk.empty((n, out, k), torch.float32)}
    ws = mk.empty((lc.adapter_workspace_size(N, d, out, k, n),), torch.uint8)
    lc.loca_adapter_apply(X, W, ad, plan, o["Y"], workspace=ws)
    mk.check("loca_adapter_apply")
    ws = mk.empty((lc.adapter_workspace_size(N, d, out, k, n, backward=True),), torch.uint8)
    lc.loca_adapter_backward(X, dY, W, ad, plan, dX=o["dX"], dA=o["dA"], dB=o["dB"], workspace=ws)
    mk.check("loca_adapter_backward")
    return o


def _clip(lc, mk, sizes):
    g = torch.Generator(device="cuda")
    g.manual_seed(len(sizes))
    grads = [torch.randn((n,), generator=g, device="cuda").to(torch.bfloat16 if i % 3 == 0 else torch.float32)
             for i, n in enumerate(sizes)]
    out = [mk.empty(t.shape, t.dtype) for t in grads]
    norm = mk.empty((1,), torch.float32)
    lc.GradClip(grads, out=out).run(0.5, norm)
    mk.check("loca_grad_clip")
    return dict({f"out{i}": t for i, t in enumerate(out)}, norm=norm)


@pytest.mark.parametrize("name,call", [
    ("head, one token", lambda lc, mk: _head(lc, mk, 1, 72, 301, 3)),
    ("head, few tokens", lambda lc, mk: _head(lc, mk, 77, 328, 5003, 5)),
    ("head", lambda lc, mk: _head(lc, mk, 1301, 200, 1999, 4)),
    ("adapters, one token", lambda lc, mk: _adapters(lc, mk, 1, 72, 136, 5, 2)),
    ("adapters, token by token", lambda lc, mk: _adapters(lc, mk, 61, 520, 392, 12, 40)),
    ("adapters, one tile", lambda lc, mk: _adapters(lc, mk, 99, 520, 392, 33, 2)),
    ("adapters", lambda lc, mk: _adapters(lc, mk, 1501, 328, 1416, 24, 5)),
    ("clip", lambda lc, mk: _clip(lc, mk, [1, 7, 8193, 20000, 33])),
])
def test_debug_build_matches_and_stays_inside(lc, name, call):
    lc.use_debug_library(False)
    ref = call(lc, Guarded(lc))
    lc.use_debug_library(True)
    assert lc.loca_debug_build()
    got = call(lc, Guarded(lc))
    lc.use_debug_library(False)
    for k in ref:
        assert torch.equal(ref[k], got[k]), (name, k)
