"""The head loss, the adapted projection and clipping captured in a CUDA graph: replays on new values in
the same buffers give the bits that the calls give, and a captured call that gives up on a wait
(loca_set_wait_limit) never leaves a wrong result behind a status word that says nothing."""

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


def _head(lc, N, d, V):
    s = dict(H=torch.empty((N, d), dtype=torch.bfloat16, device="cuda"),
             W=torch.empty((V, d), dtype=torch.bfloat16, device="cuda"),
             y=torch.empty((N,), dtype=torch.int32, device="cuda"))
    out = [torch.empty((N,), device="cuda"), torch.empty((N,), device="cuda"), torch.empty_like(s["H"]), torch.empty_like(s["W"])]
    ws = torch.empty(max(lc.head_loss_workspace_size(N, V, d), lc.head_loss_backward_workspace_size(N, V, d)),
                     dtype=torch.uint8, device="cuda")

    def fill(seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        s["H"].copy_(torch.randn((N, d), generator=g, device="cuda"))
        s["W"].copy_(torch.randn((V, d), generator=g, device="cuda") / d ** 0.5)
        s["y"].copy_(torch.randint(-V // 2, V, (N,), generator=g, device="cuda"))

    def call():
        lc.loca_head_loss(s["H"], s["W"], s["y"], out[0], lse=out[1], workspace=ws)
        lc.loca_head_loss_backward(s["H"], s["W"], s["y"], out[1], dH=out[2], dW=out[3], workspace=ws)

    return fill, call, out


def _adapters(lc, N, d, o, k, n, train):
    f32 = dict(device="cuda")
    b16 = dict(dtype=torch.bfloat16, device="cuda")
    X, W, dY = torch.empty((N, d), **b16), torch.empty((o, d), **b16), torch.empty((N, o), **b16)
    A, B = torch.empty((n, d, k), **f32), torch.empty((n, o, k), **f32)
    ids = torch.zeros((N,), dtype=torch.int32, device="cuda")
    ad, plan = lc.AdapterSet(n, d, o, k), lc.AdapterPlan(ids, n)
    ws = torch.empty(lc.adapter_workspace_size(N, d, o, k, n, backward=train), dtype=torch.uint8, device="cuda")
    grads = [torch.empty_like(X), torch.empty_like(A), torch.empty_like(B)] if train else []
    out = [torch.empty_like(dY)] + grads
    norm = torch.empty((1,), device="cuda")
    clip = lc.GradClip(grads[1:]) if train else None
    if train:
        out.append(norm)

    def fill(seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        for t, scale in ((X, 1.0), (W, d ** -0.5), (dY, 1.0), (A, d ** -0.5), (B, 1.0)):
            t.copy_(scale * torch.randn(t.shape, generator=g, device="cuda"))
        ids.copy_(torch.randint(-1, n, (N,), generator=g, device="cuda"))

    def call():
        ad.pack(A, B)
        plan.update(ids)
        lc.loca_adapter_apply(X, W, ad, plan, out[0], workspace=ws)
        if train:
            lc.loca_adapter_backward(X, dY, W, ad, plan, dX=grads[0], dA=grads[1], dB=grads[2], workspace=ws)
            clip.run(1.0, norm)

    return fill, call, out


PROGRAMS = {
    "head, many tokens": lambda lc: _head(lc, 900, 328, 3001),
    "head, few tokens": lambda lc: _head(lc, 40, 328, 3001),
    "one token": lambda lc: _adapters(lc, 1, 512, 264, 16, 4, False),
    "decode": lambda lc: _adapters(lc, 64, 512, 264, 16, 64, False),
    "train, few tokens": lambda lc: _adapters(lc, 100, 512, 264, 16, 3, True),
    "train, many tokens": lambda lc: _adapters(lc, 3000, 512, 264, 16, 3, True),
    "long": lambda lc: _adapters(lc, 100, 65536, 2048, 16, 3, False),
    "long, token by token": lambda lc: _adapters(lc, 64, 65536, 2048, 16, 64, False),
}


def _capture(call):
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    return graph


@pytest.mark.parametrize("name", sorted(PROGRAMS))
def test_replays_give_the_calls_bits(lc, name):
    lc.loca_set_wait_limit(0)
    fill, call, out = PROGRAMS[name](lc)
    fill(1)
    graph = _capture(call)
    for seed in (2, 3):
        fill(seed)
        call()
        want = [t.clone() for t in out]
        for t in out:
            t.fill_(7)
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        assert lc.loca_device_status() == 0
        for i, (a, b) in enumerate(zip(want, out)):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("name", sorted(PROGRAMS))
def test_a_replay_after_one_that_gave_up(lc, name):
    lc.loca_set_wait_limit(0)
    fill, call, out = PROGRAMS[name](lc)
    fill(1)
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    assert lc.loca_device_status() == 0
    lc.loca_set_wait_limit(1000)  # the captured launches keep it
    fill(1)
    graph = _capture(call)
    lc.loca_set_wait_limit(0)
    lc.loca_device_status()
    for replay in range(30):
        fill(1)
        graph.replay()
        torch.cuda.synchronize()
        status = lc.loca_device_status()
        assert status in (0, LOCA_ERR_TIMEOUT), status
        if status == 0:
            for i, (a, b) in enumerate(zip(want, out)):
                assert torch.equal(a, b), (replay, i)
    fill(1)
    call()
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(want, out))
