"""The distillation loss, the gated feed-forward and the 4-bit projection in the ways a program runs them: captured in
CUDA graphs, on a stream beside the current one, from several host threads, with bounded waits that run out,
through the debug build, and together as one training step and its serving.
"""

import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

LOCA_ERR_TIMEOUT = 6
GUARD, POISON = 16384, 0xA5


@pytest.fixture(scope="module")
def lc():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_03020_gb300 import _build

    _build.build()
    from paper_2608_03020_gb300 import loca

    loca.use_debug_library(False)
    yield loca
    loca.use_debug_library(False)
    loca.loca_set_wait_limit(0)


def _plain(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _distill(lc, mk, N, d, V, K):
    """(fill, call, outputs): fill(seed) makes new inputs in the same buffers."""
    b16, f32 = torch.bfloat16, torch.float32
    H, W = _plain((N, d), b16), _plain((V, d), b16)
    idx, t = _plain((N, K), torch.int32), _plain((N, K), f32)
    out = [mk((N,), f32), mk((N,), f32), mk((N, d), b16), mk((V, d), b16)]
    ws = mk((lc.head_distill_workspace_size(N, V, d, K),), torch.uint8)
    wb = mk((lc.head_distill_backward_workspace_size(N, V, d, K),), torch.uint8)

    def fill(seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        H.copy_(torch.randn(H.shape, generator=g, device="cuda"))
        W.copy_(torch.randn(W.shape, generator=g, device="cuda") / d ** 0.5)
        idx.copy_(torch.randint(-V // 2, V, idx.shape, generator=g, device="cuda"))
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))

    def call(stream=None):
        lc.loca_head_distill(H, W, idx, t, out[0], lse=out[1], tau=1.5, workspace=ws, stream=stream)
        lc.loca_head_distill_backward(H, W, idx, t, out[1], dH=out[2], dW=out[3], tau=1.5, workspace=wb, stream=stream)

    return fill, call, out


def _gated(lc, mk, N, d, f, dw=True):
    b16 = torch.bfloat16
    X, Wg, Wu, dH = _plain((N, d), b16), _plain((f, d), b16), _plain((f, d), b16), _plain((N, f), b16)
    out = [mk((N, f), b16), mk((N, d), b16)] + ([mk((f, d), b16), mk((f, d), b16)] if dw else [])
    ws = mk((max(lc.gated_workspace_size(N, d, f), lc.gated_backward_workspace_size(N, d, f, True, dw)),), torch.uint8)

    def fill(seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        for x, scale in ((X, 1.0), (Wg, d ** -0.5), (Wu, d ** -0.5), (dH, 1.0)):
            x.copy_(scale * torch.randn(x.shape, generator=g, device="cuda"))

    def call(stream=None):
        lc.loca_gated(X, Wg, Wu, out[0], workspace=ws, stream=stream)
        grads = dict(dWg=out[2], dWu=out[3]) if dw else {}
        lc.loca_gated_backward(X, Wg, Wu, dH, dX=out[1], act="gelu", workspace=ws, stream=stream, **grads)

    return fill, call, out


def _q4(lc, mk, N, d, o, group, k, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(N + d)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    codes = torch.randint(0, 256, (o, d // 2), generator=g, device="cuda", dtype=torch.uint8)
    zeros = torch.randint(0, 16, (o, d // group), generator=g, device="cuda", dtype=torch.uint8)
    weight = lc.Q4Weight(codes, (rn(o, d // group).abs() / d ** 0.5).contiguous(), zeros=zeros)
    packed = mk(weight.packed.shape, torch.uint8)
    packed.copy_(weight.packed)
    weight.packed = packed
    X = _plain((N, d), torch.bfloat16)
    A, B, ids = rn(n, d, k) / d ** 0.5, rn(n, o, k), torch.zeros((N,), dtype=torch.int32, device="cuda")
    ad, plan = lc.AdapterSet(n, d, o, k).pack(A, B), lc.AdapterPlan(ids, n)
    out = [mk((N, o), torch.bfloat16), mk((N, o), torch.bfloat16)]
    ws = mk((lc.q4_workspace_size(N, d, o, k, n),), torch.uint8)
    torch.cuda.synchronize()

    def fill(seed):
        h = torch.Generator(device="cuda")
        h.manual_seed(seed)
        X.copy_(torch.randn(X.shape, generator=h, device="cuda"))
        ids.copy_(torch.randint(-1, n, ids.shape, generator=h, device="cuda"))

    def call(stream=None):
        plan.update(ids, stream=stream)
        lc.loca_q4_apply(X, weight, out[0], adapters=ad, plan=plan, workspace=ws, stream=stream)
        lc.loca_q4_apply(X, weight, out[1], stream=stream)

    return fill, call, out


PROGRAMS = {
    "distill, many positions": lambda lc, mk: _distill(lc, mk, 900, 328, 3001, 12),
    "distill, few positions": lambda lc, mk: _distill(lc, mk, 100, 328, 3001, 12),
    "distill, one position": lambda lc, mk: _distill(lc, mk, 1, 328, 3001, 200),
    "gated, many tokens": lambda lc, mk: _gated(lc, mk, 1500, 328, 1416),
    "gated, few tokens": lambda lc, mk: _gated(lc, mk, 100, 328, 1416),
    "gated, one token": lambda lc, mk: _gated(lc, mk, 1, 136, 264, dw=False),
    "q4, one token": lambda lc, mk: _q4(lc, mk, 1, 640, 264, 128, 16, 3),
    "q4, decode": lambda lc, mk: _q4(lc, mk, 40, 1056, 1000, 32, 24, 40),
    "q4, two blocks of tokens": lambda lc, mk: _q4(lc, mk, 100, 512, 136, 64, 8, 3),
    "q4, sixteen tokens": lambda lc, mk: _q4(lc, mk, 16, 1056, 264, 32, 8, 5),
    "q4, tiles of 128 tokens": lambda lc, mk: _q4(lc, mk, 150, 1152, 264, 128, 16, 3),
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
def test_replays_on_new_inputs(lc, name):
    fill, call, out = PROGRAMS[name](lc, _plain)
    fill(1)
    graph = _capture(call)
    for seed in (2, 3):
        fill(seed)
        call()
        want = [t.clone() for t in out]
        for t in out:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert lc.loca_device_status() == 0
        for i, (a, b) in enumerate(zip(want, out)):
            assert torch.equal(a, b), i


def test_two_graphs_share_a_workspace(lc):
    """Replayed one after the other, each gives its own results."""
    big = torch.empty((1 << 28,), dtype=torch.uint8, device="cuda")
    taken = []

    def shared(shape, dtype):  # workspaces come last and take the same memory
        if dtype == torch.uint8:
            return big[:shape[0]]
        taken.append(_plain(shape, dtype))
        return taken[-1]

    made = [_distill(lc, shared, 300, 328, 3001, 12), _gated(lc, shared, 700, 328, 1416)]
    want = []
    for fill, call, out in made:
        fill(5)
        call()
        want.append([t.clone() for t in out])
    graphs = [_capture(call) for _, call, _ in made]
    for _ in range(3):
        for _, _, out in made:
            for t in out:
                t.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert lc.loca_device_status() == 0
        for w, (_, _, out) in zip(want, made):
            assert all(torch.equal(a, b) for a, b in zip(w, out))


@pytest.mark.parametrize("name", sorted(PROGRAMS))
def test_beside_the_current_stream(lc, name):
    """Behind other work on a stream of its own, while the current stream takes and overwrites memory."""
    fill, call, out = PROGRAMS[name](lc, _plain)
    fill(3)
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    for t in out:
        t.fill_(7)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = torch.zeros((8192, 8192), device="cuda")
        for _ in range(4):
            a = a @ a
    call(stream=s)
    junk = [torch.full((1 << e,), -1, dtype=torch.uint8, device="cuda") for e in range(9, 27) for _ in range(3)]
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0 and len(junk) == 54
    for i, (x, y) in enumerate(zip(want, out)):
        assert torch.equal(x, y), i


def test_without_a_workspace(lc):
    """Scratch memory that a call takes itself belongs to the stream of the call."""
    N, d, f = 200, 136, 264
    X, Wg, Wu = (torch.randn(s, device="cuda").to(torch.bfloat16) for s in ((N, d), (f, d), (f, d)))
    dH = torch.randn((N, f), device="cuda").to(torch.bfloat16)
    want, got = torch.empty_like(X), torch.empty_like(X)
    lc.loca_gated_backward(X, Wg, Wu, dH, dX=want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    lc.loca_gated_backward(X, Wg, Wu, dH, dX=got, stream=s)
    junk = [torch.full((1 << e,), -1, dtype=torch.uint8, device="cuda") for e in range(9, 24) for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(want, got) and junk


def test_threads(lc):
    """Four host threads, each with a program and a stream of its own."""
    names = ["distill, few positions", "gated, many tokens", "q4, decode", "gated, few tokens"]
    made = [PROGRAMS[n](lc, _plain) for n in names]
    want, errors, start = [], [], threading.Barrier(len(made))
    for i, (fill, call, out) in enumerate(made):
        fill(i)
        call()
        torch.cuda.synchronize()
        want.append([t.clone() for t in out])

    def work(i):
        try:
            s = torch.cuda.Stream()
            start.wait(timeout=60)
            for _ in range(200):
                made[i][1](stream=s)
            s.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append((names[i], repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(made))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    assert lc.loca_device_status() == 0
    for name, w, (_, _, out) in zip(names, want, made):
        assert all(torch.equal(a, b) for a, b in zip(w, out)), name


# name: whether it has waits so long that one must give up
LONG = {
    "distill": (lambda lc: _distill(lc, _plain, 1000, 8192, 8000, 8), True),
    "distill, few positions": (lambda lc: _distill(lc, _plain, 64, 2048, 30000, 8), False),
    "gated": (lambda lc: _gated(lc, _plain, 1000, 16384, 2048), True),
    "gated, narrow tiles": (lambda lc: _gated(lc, _plain, 700, 20000, 1024), True),
    "gated, few tokens": (lambda lc: _gated(lc, _plain, 64, 8192, 4096), False),
    "q4, many tokens": (lambda lc: _q4(lc, _plain, 200, 65536, 1024, 64, 8, 2), True),
}


@pytest.mark.parametrize("name", sorted(LONG))
def test_a_wait_that_runs_out_is_reported(lc, name):
    lc.loca_set_wait_limit(0)
    assert lc.loca_device_status() == 0
    make, must = LONG[name]
    fill, call, out = make(lc)
    fill(1)
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    timed_out = False
    for attempt in range(10):
        lc.loca_set_wait_limit(1000)
        call()
        torch.cuda.synchronize()
        status = lc.loca_device_status()
        lc.loca_set_wait_limit(0)
        if status == LOCA_ERR_TIMEOUT:
            timed_out = True
            call()
            torch.cuda.synchronize()
            assert lc.loca_device_status() == 0
        else:
            assert status == 0, (attempt, status)
        assert all(torch.equal(a, b) for a, b in zip(want, out)), attempt
    assert timed_out or not must


@pytest.mark.parametrize("name", sorted(PROGRAMS))
def test_debug_build_matches_and_stays_inside(lc, name):
    from paper_2608_03020_gb300 import _build

    _build.build(debug=True)
    results = []
    for debug in (False, True):
        bufs = []

        def guarded(shape, dtype):
            n = torch.Size(shape).numel() * torch.empty((), dtype=dtype).element_size()
            raw = torch.full((n + 2 * GUARD,), POISON, dtype=torch.uint8, device="cuda")
            bufs.append((raw, n))
            return raw[GUARD:GUARD + n].view(dtype).view(shape)

        lc.use_debug_library(debug)
        try:
            assert lc.loca_debug_build() == debug
            fill, call, out = PROGRAMS[name](lc, guarded)
            fill(4)
            call()
            torch.cuda.synchronize()
            status = lc.loca_device_status()
            assert status == 0, (status, lc.loca_last_error())
        finally:
            lc.use_debug_library(False)
        for i, (raw, n) in enumerate(bufs):
            assert bool((raw[:GUARD] == POISON).all()) and bool((raw[GUARD + n:] == POISON).all()), i
        results.append([t.clone() for t in out])
    for i, (a, b) in enumerate(zip(*results)):
        assert torch.equal(a, b), i


def test_together(lc):
    """A student block under a teacher: H = gated(X), Y = H W^T (4-bit, adapters beside), the distillation loss of Y
    and its gradient back through the projection's 4-bit values (frozen) into the block.  Each stage against 64
    bits from the stage's own inputs, and the whole chain's gradients against autograd in 64 bits."""
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    N, d, f, V, K, k, n, group = 48, 256, 512, 1003, 8, 8, 3, 64
    X = rn(N, d).to(torch.bfloat16)
    Wg, Wu = (rn(f, d) / d ** 0.5).to(torch.bfloat16), (rn(f, d) / d ** 0.5).to(torch.bfloat16)
    head = (2 * rn(V, d) / d ** 0.5).to(torch.bfloat16)
    codes = torch.randint(0, 256, (d, f // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = ((0.5 + torch.rand((d, f // group), generator=g, device="cuda")) * 0.3 / f ** 0.5).to(torch.bfloat16)
    A, B, ids = rn(n, f, k) / f ** 0.5, 0.3 * rn(n, d, k), torch.randint(-1, n, (N,), generator=g, device="cuda", dtype=torch.int32)
    idx = torch.randint(0, V, (N, K), generator=g, device="cuda", dtype=torch.int32)
    idx[::5] = -1
    t, tau = 2 * rn(N, K), 2.0
    b16 = dict(dtype=torch.bfloat16, device="cuda")
    H, Y, dY, dX = torch.empty((N, f), **b16), torch.empty((N, d), **b16), torch.empty((N, d), **b16), torch.empty((N, d), **b16)
    dWg, dWu, dH = torch.empty_like(Wg), torch.empty_like(Wu), torch.empty((N, f), **b16)
    loss, lse = torch.empty((N,), device="cuda"), torch.empty((N,), device="cuda")
    weight = lc.Q4Weight(codes, scales)
    ad, plan = lc.AdapterSet(n, f, d, k).pack(A, B), lc.AdapterPlan(ids, n)
    # the frozen projection's values in bf16, for its transposed product
    q = torch.stack([codes & 15, codes >> 4], 2).reshape(d, f // group, group).float() - 8
    W = (scales.float()[:, :, None] * q).reshape(d, f).to(torch.bfloat16)
    lc.loca_gated(X, Wg, Wu, H)
    lc.loca_q4_apply(H, weight, Y, adapters=ad, plan=plan)
    lc.loca_head_distill(Y, head, idx, t, loss, lse=lse, tau=tau)
    lc.loca_head_distill_backward(Y, head, idx, t, lse, dH=dY, tau=tau, grad_scale=1.0 / N)
    lc.loca_adapter_backward(H, dY, W, ad, plan, dX=dH)
    lc.loca_gated_backward(X, Wg, Wu, dH, dX=dX, dWg=dWg, dWu=dWu)
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0
    leaves = [x.double().requires_grad_() for x in (X, Wg, Wu)]
    h = torch.nn.functional.silu(leaves[0] @ leaves[1].T) * (leaves[0] @ leaves[2].T)
    y = h @ (scales.double()[:, :, None] * q.double()).reshape(d, f).T
    for a in range(n):
        m = (ids == a).double()[:, None]
        y = y + m * ((h @ A[a].double()) @ B[a].double().T)
    logp = torch.log_softmax(y @ head.double().T / tau, 1)
    has = idx >= 0
    logq = torch.log_softmax(torch.where(has, t.double() / tau, -float("inf")).where(has.any(1, keepdim=True), torch.zeros(())), 1)
    each = torch.where(has, logq.exp() * (logq - logp.gather(1, idx.clamp(min=0).long())), 0.0)
    want = tau ** 2 * each.sum(1)
    (want.sum() / N).backward()
    want = want.detach()
    # eight values are rounded to bf16 on the way to the gradients (W, H, Y, dZ, dY, dH, dG and dU, the gradient
    # itself), each within 2^-8 of its size; the loss sees three of them
    assert float((loss.double() - want).abs().max()) <= 3 * 2.0 ** -8 * float(want.abs().max())
    for got, leaf in zip((dX, dWg, dWu), leaves):
        norm = float(torch.linalg.norm(leaf.grad))
        assert float(torch.linalg.norm(got.double() - leaf.grad)) <= 8 * 2.0 ** -8 * norm
