"""Fit an adapter from hidden states, serve it to requests, and polish it by gradient steps.

One frozen square projection ``W`` (d x d) under a frozen vocabulary head.  The library's calls, in the
order a program makes them:

1. ``loca_head_loss`` on the projection's output: loss, normaliser and label-column error ``E`` without
   the logits; ``loca_head_loss_backward``: the gradient ``dH``, the probe target of the feedback map
2. the adaptation pass: ``loca_calib_fit`` on (E, dH), ``loca_targets``, ``loca_accumulate``,
   ``loca_ridge_solve``: the adapter's ``B`` in closed form
3. ``AdapterSet.pack`` and ``AdapterPlan``: the fitted adapter beside others, each request with its own
   (or none); ``loca_adapter_apply``
4. gradient steps on all adapters: ``loca_head_loss_backward``, ``loca_adapter_backward``,
   ``GradClip``, a plain update, ``pack`` again

    python examples/adapt_and_serve.py
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_03020_gb300 import loca as lc  # noqa: E402


def inputs(N, d, V, C, requests, seed):
    """Hidden states whose labels a low-rank change of the projection would predict better."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    X = rn(N, d).to(torch.bfloat16)
    W = (rn(d, d) / d ** 0.5).to(torch.bfloat16)
    head = (rn(V, d) / d ** 0.5).to(torch.bfloat16)
    cols = torch.randperm(V, generator=g, device="cuda")[:C].to(torch.int32)
    better = X.float() @ (rn(d, C) * 2.0 / d ** 0.5)
    y = cols[better.argmax(1)].clone()
    y[torch.rand((N,), generator=g, device="cuda") < 0.3] = -1  # prompt positions
    cut = torch.sort(torch.randint(1, N, (requests - 1,), generator=g, device="cuda")).values
    request = torch.bucketize(torch.arange(N, device="cuda"), cut, right=True)
    return X, W, head, cols, y, request.to(torch.int32), g


def mean_loss(loss, y):
    return float(loss.double().sum() / (y >= 0).sum())


def run(N=4096, d=512, V=8192, C=4, k=8, requests=5, steps=8, seed=0, eta=1.0, lr=2.0, verbose=True):
    X, W, head, cols, y, request, g = inputs(N, d, V, C, requests, seed)
    f32 = dict(dtype=torch.float32, device="cuda")
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    loss, lse, E = torch.empty((N,), **f32), torch.empty((N,), **f32), torch.empty((N, C), **f32)
    H, dH = torch.empty((N, d), **bf16), torch.empty((N, d), **bf16)
    live = float((y >= 0).sum())
    told = []

    def note(what):
        told.append((what, mean_loss(loss, y)))
        if verbose:
            print(f"{what:34s} loss {told[-1][1]:.4f}")

    # the fitted adapter will be number 0; requests 0 .. 2 use it, the fourth none, the others number 1
    ids = torch.where(request <= 2, 0, torch.where(request == 3, -1, 1)).to(torch.int32)
    n = 2
    A = torch.linalg.qr(torch.randn((n, d, k), generator=g, device="cuda")).Q.contiguous()
    B = torch.zeros((n, d, k), **f32)
    adapters = lc.AdapterSet(n, d, d, k).pack(A, B)
    plan = lc.AdapterPlan(ids, n)
    ws = torch.empty(lc.adapter_workspace_size(N, d, d, k, n, backward=True), dtype=torch.uint8, device="cuda")
    lw = torch.empty(max(lc.head_loss_workspace_size(N, V, d, C),
                         lc.head_loss_backward_workspace_size(N, V, d, want_dW=False)), dtype=torch.uint8, device="cuda")

    def forward():
        lc.loca_adapter_apply(X, W, adapters, plan, H, workspace=ws)
        lc.loca_head_loss(H, head, y, loss, lse=lse, label_cols=cols, E=E, workspace=lw)

    # 1. the frozen model: error and probe gradient
    forward()
    note("frozen")
    lc.loca_head_loss_backward(H, head, y, lse, dH=dH, workspace=lw)

    # 2. the adaptation pass (one block): feedback map, targets, statistics, closed-form solve
    r = min(C, 4)
    P, Q = torch.empty((1, C, r), **f32), torch.empty((1, r, d), **f32)
    beta = 1e-3 * float(E.double().square().sum()) / C
    lc.loca_calib_fit(E, dH.float().unsqueeze(0), beta, r, P, Q)
    T, tsq = torch.empty((1, N, d), **bf16), torch.empty((1,), dtype=torch.float64, device="cuda")
    lc.loca_targets(E, P, Q, T, tsq=tsq)
    gram, cross = torch.empty((1, d, d), **f32), torch.empty((1, d, d), **f32)
    xsq = torch.empty((1,), dtype=torch.float64, device="cuda")
    lc.loca_accumulate(X.unsqueeze(0), T, tsq, eta, gram, cross, xsq, zero_first=True)
    solved, info = torch.empty((1, 1, d, k), **f32), torch.empty((1, 1), dtype=torch.int32, device="cuda")
    lc.loca_ridge_solve(gram, cross, A[:1].contiguous(), [1e-3], solved, info, xsq_total=xsq)

    # 3. served beside the other adapter
    B[0] = solved[0, 0]
    adapters.pack(A, B)
    forward()
    note("adapter 0 fitted in closed form")

    # 4. gradient steps on both adapters
    dA, dB = torch.empty_like(A), torch.empty_like(B)
    clip, norm = lc.GradClip([dA, dB]), torch.empty((1,), **f32)
    for step in range(steps):
        lc.loca_head_loss_backward(H, head, y, lse, dH=dH, grad_scale=1.0 / live, workspace=lw)
        lc.loca_adapter_backward(X, dH, W, adapters, plan, dA=dA, dB=dB, workspace=ws)
        clip.run(1.0, norm)
        A -= lr * dA
        B -= lr * dB
        adapters.pack(A, B)
        forward()
    note(f"{steps} gradient steps")
    torch.cuda.synchronize()
    status = lc.loca_device_status()
    assert status == 0 and int(info) == 0, (status, int(info))
    return dict(told=told, X=X, W=W, head=head, y=y, ids=ids, A=A, B=B, loss=loss, norm=float(norm))


if __name__ == "__main__":
    from paper_2608_03020_gb300 import _build

    _build.build()
    run()
