"""Distillation at the head and its gradients against the definition in 64 bits.

Tolerances, derived before the first run.  A logit is within 2e-5 (1 + max |z|) of its exact value (64 steps of at
most 2^-22 of the running sum before a sum restarts, and two ulp of the exponentials).  ``lse`` moves with the
scaled logits, by at most their error over tau.  ``loss = w tau^2 (sum q log q - sum q (z / tau - lse))`` moves by at
most twice that times w tau^2, and each of its terms, at most log K and (max - min of z) / tau + log V in size,
carries roundings of fp32: 2^-20 of them.  Gradients come out in bf16: one rounding of dZ and one of the sum, each
uniform within 2^-8 of a binade's size, so less than 2^-8 together in norm.
"""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lc():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_03020_gb300 import _build

    _build.build()
    from paper_2608_03020_gb300 import loca

    loca.lib()
    return loca


def _inputs(N, d, V, K, seed=0, mask="none", scale=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 7 * N + 11 * d + 13 * V + 17 * K)
    H = torch.randn((N, d), generator=g, device="cuda").to(torch.bfloat16)
    W = (scale / d ** 0.5 * torch.randn((V, d), generator=g, device="cuda")).to(torch.bfloat16)
    idx = torch.randint(0, V, (N, K), generator=g, device="cuda", dtype=torch.int32)  # words may come twice
    t = 3.0 * torch.randn((N, K), generator=g, device="cuda")
    drop = torch.rand((N, K), generator=g, device="cuda")
    if mask == "some":  # entries and whole positions without a word
        idx[drop < 0.3] = -1
        idx[::3] = -1
    elif mask == "all":
        idx[:] = V
    elif mask == "one":
        idx[torch.arange(N, device="cuda") != N // 2] = -5
    elif mask == "edges":  # the first and last words of the vocabulary and of its tiles
        edge = torch.tensor([0, V - 1, 127, 128, 255, 256, V // 2], device="cuda", dtype=torch.int32).clamp(max=V - 1)
        idx = edge[torch.randint(0, 7, (N, K), generator=g, device="cuda")]
    w = torch.rand((N,), generator=g, device="cuda") + 0.5
    gl = torch.randn((N,), generator=g, device="cuda")
    return H, W, idx.contiguous(), t, w, gl


def _reference(H, W, idx, t, w, dloss, tau, scale):
    V = W.shape[0]
    at = idx.long()
    has = (at >= 0) & (at < V)
    td = torch.where(has, t.double(), -INF) / tau
    live = (td > -INF).any(1) | td.isnan().any(1)
    td = torch.where(live[:, None], td, 0.0)
    logq = torch.log_softmax(td, 1)
    q = torch.where(live[:, None], logq.exp(), 0.0)
    Hd = torch.where(live[:, None], H.double(), 0.0)
    z = Hd @ W.double().T
    lse = torch.logsumexp(z / tau, 1)
    at = torch.where(has, at, 0)
    each = q * (logq - (z.gather(1, at) / tau - lse[:, None]))
    wd = torch.where(live, w.double(), 0.0)
    out = {"loss": wd * tau ** 2 * torch.where(q == 0, 0.0, each).sum(1), "lse": torch.where(live, lse, 0.0)}
    dz = torch.exp(z / tau - lse[:, None]).scatter_add_(1, at, -q)
    dz *= (wd * dloss.double() * tau)[:, None]
    out["dH"] = scale * (dz @ W.double())
    out["dW"] = scale * (dz.T @ Hd)
    out["zmax"] = float(z.abs().max()) if z.numel() else 0.0
    return out


def _run(lc, H, W, idx, t, w, dloss, tau, scale, dh=True, dw=True):
    N, d = H.shape
    V = W.shape[0]
    out = {"loss": torch.full((N,), NAN, device="cuda"), "lse": torch.full((N,), NAN, device="cuda")}
    lc.loca_head_distill(H, W, idx, t, out["loss"], lse=out["lse"], w=w, tau=tau)
    if dh:
        out["dH"] = torch.full((N, d), NAN, dtype=torch.bfloat16, device="cuda")
    if dw:
        out["dW"] = torch.full((V, d), NAN, dtype=torch.bfloat16, device="cuda")
    if dh or dw:
        lc.loca_head_distill_backward(H, W, idx, t, out["lse"], dH=out.get("dH"), dW=out.get("dW"), w=w, dloss=dloss,
                                      tau=tau, grad_scale=scale)
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0
    return out


def _check(out, ref, w, tau, V, K):
    ez = 2e-5 * (1.0 + ref["zmax"]) / tau
    top = max(1.0, float(w.max()) if w.numel() else 1.0)
    size = math.log(K) + 2 * ref["zmax"] / tau + math.log(V)
    tol = {"lse": ez + 2.0 ** -20 * size, "loss": top * tau ** 2 * (2 * ez + 2.0 ** -20 * size)}
    for k in ("lse", "loss"):
        worst = float((out[k].double() - ref[k]).abs().max()) if out[k].numel() else 0.0
        assert worst <= tol[k], (k, worst, tol[k])
    for k in ("dH", "dW"):
        if k in out:
            off = float(torch.linalg.norm(out[k].double() - ref[k]))
            norm = float(torch.linalg.norm(ref[k]))
            assert off <= 2.0 ** -8 * norm + 1e-30, (k, off / max(norm, 1e-300))


@pytest.mark.parametrize("N,d,V,K,mask,tau", [
    (1, 8, 1, 1, "none", 1.0), (1, 64, 5, 3, "none", 2.0), (3, 72, 255, 7, "none", 0.5), (37, 896, 256, 32, "some", 1.0),
    (128, 136, 4099, 33, "edges", 1.0), (129, 64, 1000, 5, "some", 4.0), (255, 200, 257, 256, "none", 1.0),
    (256, 64, 1000, 64, "edges", 1.5), (257, 2048, 513, 16, "one", 1.0), (300, 136, 4099, 100, "some", 0.7),
    (64, 64, 300, 4, "all", 1.0), (500, 64, 300, 4, "all", 1.0), (700, 328, 20011, 255, "some", 2.0),
    (2000, 512, 3001, 1, "none", 1.0),
])
def test_matches_definition(lc, N, d, V, K, mask, tau):
    H, W, idx, t, w, gl = _inputs(N, d, V, K, mask=mask)
    ref = _reference(H, W, idx, t, w, gl, tau, 0.25)
    _check(_run(lc, H, W, idx, t, w, gl, tau, 0.25), ref, w, tau, V, K)


def test_weights_and_gradients_of_one(lc):
    """w, dloss and lse left out: ones, ones, none."""
    H, W, idx, t, w, gl = _inputs(200, 136, 1003, 9, mask="some")
    one = torch.ones_like(w)
    ref = _reference(H, W, idx, t, one, one, 1.0, 1.0)
    out = _run(lc, H, W, idx, t, None, None, 1.0, 1.0)
    _check(out, ref, one, 1.0, 1003, 9)
    loss = torch.empty_like(w)
    lc.loca_head_distill(H, W, idx, t, loss)
    assert torch.equal(loss, out["loss"])


@pytest.mark.parametrize("dh,dw", [(True, False), (False, True)])
def test_one_gradient_alone(lc, dh, dw):
    H, W, idx, t, w, gl = _inputs(300, 136, 2003, 12, mask="some")
    ref = _reference(H, W, idx, t, w, gl, 1.0, 1.0)
    _check(_run(lc, H, W, idx, t, w, gl, 1.0, 1.0, dh, dw), ref, w, 1.0, 2003, 12)


@pytest.mark.parametrize("N", [50, 400])
def test_one_word_is_the_cross_entropy(lc, N):
    """K = 1: q = 1, the loss, lse and gradients of loca_head_loss at that label."""
    H, W, idx, t, w, gl = _inputs(N, 264, 1999, 1, mask="some")
    out = _run(lc, H, W, idx, t, w, gl, 1.0, 1.0)
    loss, lse = torch.empty_like(w), torch.empty_like(w)
    y = idx[:, 0].contiguous()
    lc.loca_head_loss(H, W, y, loss, lse=lse, w=w)
    dH = torch.empty_like(H)
    lc.loca_head_loss_backward(H, W, y, lse, dH=dH, w=w, dloss=gl)
    assert torch.allclose(out["lse"], lse, rtol=0, atol=4e-6) and torch.allclose(out["loss"], loss, rtol=0, atol=1e-5)
    norm = float(torch.linalg.norm(dH.double()))
    assert float(torch.linalg.norm(out["dH"].double() - dH.double())) <= 2.0 ** -7 * norm


@pytest.mark.parametrize("N", [6, 300])
def test_a_word_that_comes_twice(lc, N):
    """The shares of one word add up; the order of the entries changes nothing but roundings."""
    H, W, idx, t, w, gl = _inputs(N, 136, 777, 8)
    idx[:, 1], idx[:, 5], idx[0] = idx[:, 0], idx[:, 0], 776
    ref = _reference(H, W, idx, t, w, gl, 1.0, 1.0)
    out = _run(lc, H, W, idx, t, w, gl, 1.0, 1.0)
    _check(out, ref, w, 1.0, 777, 8)
    flip = _run(lc, H, W, idx.flip(1).contiguous(), t.flip(1).contiguous(), w, gl, 1.0, 1.0)
    _check(flip, ref, w, 1.0, 777, 8)


@pytest.mark.parametrize("N", [8, 300])
def test_logits_without_a_share_and_not_finite(lc, N):
    H, W, idx, t, w, gl = _inputs(N, 136, 777, 6)
    clean = _run(lc, H, W, idx, t, w, gl, 1.0, 1.0)
    t2, idx2, H2 = t.clone(), idx.clone(), H.clone()
    t2[0, :3] = -INF                    # words without a share
    t2[1] = -INF                        # no share at all: masked
    H2[1], H2[4] = NAN, INF             # in masked positions nothing counts
    t2[2, 1], t2[3, 2] = NAN, INF       # spoil their own position
    idx2[4] = -1
    idx2[5, 0], t2[5, 0] = 777, NAN     # a NaN in an entry that is none
    t2[6] = -1e30                       # far below, equal: a sixth each
    good = _run(lc, H2, W, idx2, t2, w, gl, 1.0, 1.0)
    for k in ("loss", "lse", "dH"):
        assert bool((good[k][[1, 4]] == 0).all()), k
        assert torch.equal(good[k][7:], clean[k][7:]), k
    assert bool(good["loss"][[2, 3]].isnan().all()) and bool(good["dH"][[2, 3]].isnan().all())
    assert bool(good["dW"].isnan().any())
    rows = [0, 5, 6]
    ref = _reference(H2[rows], W, idx2[rows], t2[rows], w[rows], gl[rows], 1.0, 1.0)
    _check({k: good[k][rows] for k in ("loss", "lse", "dH")}, ref, w[rows], 1.0, 777, 6)


def test_a_student_that_agrees(lc):
    """The teacher's logits are the student's own over the whole vocabulary: the loss and p - q vanish as far as
    fp32 logits of both sides allow."""
    N, d, V = 200, 136, 200
    H, W, _, _, w, gl = _inputs(N, d, V, 1)
    t = (H.double() @ W.double().T).float()
    idx = torch.arange(V, device="cuda", dtype=torch.int32).repeat(N, 1)
    out = _run(lc, H, W, idx, t, w, gl, 1.0, 1.0)
    zmax = float(t.abs().max())
    ez = 2e-5 * (1 + zmax)
    size = 2 * math.log(V) + 2 * zmax
    assert float(out["loss"].abs().max()) <= float(w.max()) * (2 * ez + 2.0 ** -20 * size)
    # |p - q| <= p (e^{2 ez} - 1 + 2^-20 size)
    bound = (w * gl.abs()).double()[:, None] * (torch.softmax(t.double(), 1) @ W.double().abs()) * (2.1 * ez + 2.0 ** -20 * size)
    assert bool((out["dH"].double().abs() <= 1.01 * bound + 1e-30).all())


def test_gradients_against_differences(lc):
    H, W, idx, t, w, gl = _inputs(60, 72, 301, 7, mask="some")
    tau, e = 1.7, 1e-5
    out = _run(lc, H, W, idx, t, w, gl, tau, 1.0)

    def total(h, m):
        return float((gl.double() * _reference(h, m, idx, t, w, gl, tau, 1.0)["loss"]).sum())

    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for k, base in (("dH", H.double()), ("dW", W.double())):
        v = torch.randn(base.shape, generator=g, device="cuda", dtype=torch.float64)
        hi, lo = ((total(base + s * v, W.double()) if k == "dH" else total(H.double(), base + s * v)) for s in (e, -e))
        num, got = (hi - lo) / (2 * e), float((out[k].double() * v).sum())
        # off by at most 2^-8 of the gradient in norm, so by that times |v|; differences to 1e-6 of F's scale
        room = 2.0 ** -8 * float(torch.linalg.norm(out[k].double())) * float(torch.linalg.norm(v))
        assert abs(num - got) <= room + 1e-4, (k, num, got)


def test_pieces_of_rows_and_vocabulary(lc):
    """Past 16384 rows forward, past 8192 backward (dH alone), and N V past 2^31 with dW: the vocabulary in pieces."""
    N, d, V, K = 17000, 64, 1003, 6
    H, W, idx, t, w, gl = _inputs(N, d, V, K, mask="some")
    ref = _reference(H, W, idx, t, w, gl, 1.0, 1.0)
    _check(_run(lc, H, W, idx, t, w, gl, 1.0, 1.0, dw=False), ref, w, 1.0, V, K)
    N, V = 70000, 32003
    H, W, idx, t, w, gl = _inputs(N, d, V, K, mask="some")
    out = _run(lc, H, W, idx, t, w, gl, 1.0, 1.0)
    dW = torch.zeros((V, d), dtype=torch.float64, device="cuda")
    for rows in torch.arange(N, device="cuda").split(10000):
        ref = _reference(H[rows], W, idx[rows], t[rows], w[rows], gl[rows], 1.0, 1.0)
        dW += ref["dW"]
        _check({k: out[k][rows] for k in ("loss", "lse", "dH")}, ref, w, 1.0, V, K)
    assert float(torch.linalg.norm(out["dW"].double() - dW)) <= 2.0 ** -8 * float(torch.linalg.norm(dW))


@pytest.mark.parametrize("N", [20, 500])
def test_spaced_rows_and_in_place(lc, N):
    H, W, idx, t, w, gl = _inputs(N, 136, 999, 5, mask="some")
    want = _run(lc, H, W, idx, t, w, gl, 1.0, 1.0)
    big = torch.full((N, 160), 7.0, dtype=torch.bfloat16, device="cuda")
    view = big[:, 8:144]
    view.copy_(H)
    loss, lse = torch.empty_like(w), torch.empty_like(w)
    lc.loca_head_distill(view, W, idx, t, loss, lse=lse, w=w)
    assert torch.equal(loss, want["loss"]) and torch.equal(lse, want["lse"])
    lc.loca_head_distill_backward(view, W, idx, t, lse, dH=view, w=w, dloss=gl)  # over H itself
    assert torch.equal(view, want["dH"])
    assert bool((big[:, :8] == 7).all()) and bool((big[:, 144:] == 7).all())


def test_the_same_bits_again(lc):
    H, W, idx, t, w, gl = _inputs(900, 328, 5003, 40, mask="some")
    a, b = (_run(lc, H, W, idx, t, w, gl, 2.0, 1.0) for _ in range(2))
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_no_positions(lc):
    H, W, idx, t, w, gl = _inputs(0, 64, 72, 3)
    out = _run(lc, H, W, idx, t, w, gl, 1.0, 1.0)
    assert bool((out["dW"] == 0).all())


def test_python_refusals(lc):
    H, W, idx, t, w, gl = _inputs(10, 64, 72, 3)
    loss, lse, dH = torch.empty_like(w), torch.zeros_like(w), torch.empty_like(H)
    for tau in (0.0, -1.0, NAN, INF):
        with pytest.raises(lc.LocaError, match="tau"):
            lc.loca_head_distill(H, W, idx, t, loss, tau=tau)
    with pytest.raises(TypeError):
        lc.loca_head_distill(H, W, idx.long(), t, loss)
    with pytest.raises(TypeError):
        lc.loca_head_distill(H, W, idx, t.half(), loss)
    with pytest.raises(ValueError):
        lc.loca_head_distill(H, W, idx, t[:, :2].contiguous(), loss)
    with pytest.raises(lc.LocaError, match="256 words"):
        lc.loca_head_distill(H, W, torch.zeros((10, 257), dtype=torch.int32, device="cuda"), torch.zeros((10, 257), device="cuda"), loss)
    with pytest.raises(lc.LocaError, match="required"):
        lc.loca_head_distill_backward(H, W, idx, t, lse)
    for bad in (dict(dH=dH, dW=W), dict(dW=W), dict(dH=W[:10])):
        with pytest.raises(lc.LocaError, match="overlap"):
            lc.loca_head_distill_backward(H, W, idx, t, lse, **bad)


@pytest.mark.parametrize("N,K", [(1, 1), (1, 3), (5, 1), (63, 2), (64, 1)])
def test_few_positions_round_their_gradients_once(lc, N, K):
    """Up to 64 positions dZ has two parts (2^-17): what is left is the gradients' own rounding, half a step (2^-8)
    of each value, plus the products' 2^-15 (two parts and sums) of the sums of magnitudes, and where the student's
    logits are off (2 ez of p) as in _check."""
    H, W, idx, t, w, gl = _inputs(N, 264, 1999, K, mask="none")
    out = _run(lc, H, W, idx, t, w, gl, 1.0, 1.0)
    ref = _reference(H, W, idx, t, w, gl, 1.0, 1.0)
    z = H.double() @ W.double().T
    p = torch.softmax(z, 1)
    dz = p.clone()
    dz.scatter_add_(1, idx.long(), -torch.softmax(t.double(), 1))
    dz = dz.abs() * (w * gl.abs()).double()[:, None]
    ez = 2e-5 * (1 + ref["zmax"])
    off = 2.0 ** -15 * dz + 3 * ez * p * (w * gl.abs()).double()[:, None]
    for k, e in (("dH", off @ W.double().abs()), ("dW", off.T @ H.double().abs())):
        tol = 2.0 ** -8 * ref[k].abs() + 1.01 * e + 1e-37
        assert bool(((out[k].double() - ref[k]).abs() <= tol).all()), k
