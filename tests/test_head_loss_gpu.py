"""Head loss and its gradients against the definition in 64 bits.

Tolerances, fixed before the first run.  The products of bf16 values are exact; the tensor cores lose
up to 2^-22 of the running sum per step, toward zero, and a sum restarts after 64 steps, so a logit is
within 64 * 2^-22 = 1.5e-5 of the largest partial sum, taken as 2e-5 (1 + max |z|) with the fp32
exponentials (2 ulp each).  ``loss``, ``lse`` and ``E`` (whose derivative with respect to a logit is at
most w) are held to that times the weight.  Gradients come out in bf16: one rounding of dZ and one of
the sum, each uniform within 2^-8 of a binade's size, so less than 2^-8 together in norm.
"""

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


def _inputs(N, d, V, seed=0, mask="none", scale=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 7 * N + 11 * d + 13 * V)
    H = torch.randn((N, d), generator=g, device="cuda").to(torch.bfloat16)
    W = (scale / d ** 0.5 * torch.randn((V, d), generator=g, device="cuda")).to(torch.bfloat16)
    y = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    if N > 2:
        y[1], y[2] = V - 1, 0
    if mask == "half":
        y[torch.rand((N,), generator=g, device="cuda") < 0.5] = -1
    elif mask == "all":
        y[:] = -1
    elif mask == "one":
        keep = y[N // 2].clone()
        y[:] = -100
        y[N // 2] = keep
    elif mask == "tail":
        y[N // 3:] = V  # past the vocabulary: masked too
    w = torch.rand((N,), generator=g, device="cuda") + 0.5
    gl = torch.randn((N,), generator=g, device="cuda")
    return H, W, y, w, gl


def _reference(H, W, y, w, dloss, cols, scale):
    V = W.shape[0]
    live = (y >= 0) & (y < V)
    Hd = torch.where(live[:, None], H.double(), 0.0)
    z = Hd @ W.double().T
    lse = torch.logsumexp(z, 1)
    at = torch.where(live, y.long(), 0)
    wd = torch.where(live, w.double(), 0.0)
    out = {"loss": wd * (lse - z.gather(1, at[:, None])[:, 0]), "lse": torch.where(live, lse, 0.0)}
    err = torch.exp(z - lse[:, None])
    err.scatter_add_(1, at[:, None], -torch.ones_like(at, dtype=torch.float64)[:, None])
    err *= wd[:, None]
    if cols is not None:
        out["E"] = err[:, cols.long()]
    dz = err * dloss.double()[:, None]
    out["dH"] = scale * (dz @ W.double())
    out["dW"] = scale * (dz.T @ Hd)
    out["zmax"] = float(z.abs().max()) if z.numel() else 0.0
    return out


def _run(lc, H, W, y, w, dloss, cols, scale, dh=True, dw=True):
    N, d = H.shape
    V = W.shape[0]
    nan = float("nan")
    out = {"loss": torch.full((N,), nan, device="cuda"), "lse": torch.full((N,), nan, device="cuda")}
    E = None if cols is None else torch.full((N, cols.numel()), nan, device="cuda")
    lc.loca_head_loss(H, W, y, out["loss"], lse=out["lse"], w=w, label_cols=cols, E=E)
    if E is not None:
        out["E"] = E
    if dh:
        out["dH"] = torch.full((N, d), nan, dtype=torch.bfloat16, device="cuda")
    if dw:
        out["dW"] = torch.full((V, d), nan, dtype=torch.bfloat16, device="cuda")
    if dh or dw:
        lc.loca_head_loss_backward(H, W, y, out["lse"], dH=out.get("dH"), dW=out.get("dW"), w=w, dloss=dloss,
                                   grad_scale=scale)
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0
    return out


def _check(out, ref, w):
    tol = 2e-5 * (1.0 + ref["zmax"])
    top = float(w.max()) if w.numel() else 1.0
    for k in ("loss", "lse", "E"):
        if k in out:
            worst = float((out[k].double() - ref[k]).abs().max()) if out[k].numel() else 0.0
            assert worst <= tol * max(1.0, top), (k, worst, tol)
    for k in ("dH", "dW"):
        if k in out:
            off = float(torch.linalg.norm(out[k].double() - ref[k]))
            norm = float(torch.linalg.norm(ref[k]))
            assert off <= 2.0 ** -8 * norm, (k, off / max(norm, 1e-300))


@pytest.mark.parametrize("N,d,V,mask", [
    (1, 8, 1, "none"), (1, 64, 5, "none"), (3, 72, 255, "none"), (37, 896, 256, "half"), (255, 200, 257, "half"),
    (256, 64, 1000, "none"), (257, 2048, 513, "one"), (300, 136, 4099, "tail"), (64, 64, 300, "all"),
    (777, 896, 3001, "half"), (130, 5120, 777, "none"), (2000, 328, 129, "half"),
])
def test_loss_and_gradients(lc, N, d, V, mask):
    H, W, y, w, gl = _inputs(N, d, V, mask=mask)
    cols = torch.unique(torch.tensor([V - 1, 0, V // 2, V // 3], device="cuda")).to(torch.int32)
    ref = _reference(H, W, y, w, gl, cols, 0.25)
    _check(_run(lc, H, W, y, w, gl, cols, 0.25), ref, w)


@pytest.mark.parametrize("C", [1, 33, 200, 1024])
def test_many_label_columns_in_any_order(lc, C):
    N, d, V = 70, 64, 1500
    H, W, y, w, gl = _inputs(N, d, V, seed=C)
    g = torch.Generator(device="cuda")
    g.manual_seed(C)
    cols = torch.randperm(V, generator=g, device="cuda")[:C].to(torch.int32)
    y[:40] = cols[torch.arange(40, device="cuda") % C]
    ref = _reference(H, W, y, w, gl, cols, 1.0)
    _check(_run(lc, H, W, y, w, gl, cols, 1.0, dh=False, dw=False), ref, w)


def test_optional_arguments_default_to_ones(lc):
    N, d, V = 90, 128, 700
    H, W, y, _, _ = _inputs(N, d, V, mask="half")
    one = torch.ones((N,), device="cuda")
    ref = _reference(H, W, y, one, one, None, 1.0)
    loss = torch.empty((N,), device="cuda")
    lc.loca_head_loss(H, W, y, loss)
    _check({"loss": loss}, ref, one)
    lse = ref["lse"].float()
    dH = torch.empty((N, d), dtype=torch.bfloat16, device="cuda")
    lc.loca_head_loss_backward(H, W, y, lse, dH=dH)
    dW = torch.empty((V, d), dtype=torch.bfloat16, device="cuda")
    lc.loca_head_loss_backward(H, W, y, lse, dW=dW)
    _check({"dH": dH, "dW": dW}, ref, one)


def test_masked_rows_may_hold_anything(lc):
    N, d, V = 513, 72, 800
    H, W, y, w, gl = _inputs(N, d, V, mask="half")
    cols = torch.tensor([5, 3], dtype=torch.int32, device="cuda")
    ref = _reference(H, W, y, w, gl, cols, 1.0)
    dead = (y < 0)[:, None]
    odd = torch.arange(N, device="cuda")[:, None] % 3
    H = torch.where(dead & (odd == 0), float("nan"), torch.where(dead & (odd == 1), float("inf"), H.float()))
    H = torch.where(dead & (odd == 2), torch.finfo(torch.bfloat16).min, H).to(torch.bfloat16)
    w = torch.where(dead[:, 0], float("nan"), w)
    out = _run(lc, H, W, y, w, gl, cols, 1.0)
    _check(out, ref, torch.nan_to_num(w))
    for k in ("loss", "lse", "E", "dH"):
        assert torch.all(out[k][dead[:, 0]] == 0), k


def test_a_live_row_that_is_not_finite_stays_in_its_row(lc):
    N, d, V = 300, 64, 600
    H, W, y, w, gl = _inputs(N, d, V)
    clean = _run(lc, H, W, y, w, gl, None, 1.0, dw=False)
    H[17, 3] = float("inf")
    H[200, 1] = float("nan")
    got = _run(lc, H, W, y, w, gl, None, 1.0, dw=False)
    rest = torch.ones((N,), dtype=torch.bool, device="cuda")
    rest[[17, 200]] = False
    for k in ("loss", "lse", "dH"):
        assert torch.equal(clean[k][rest], got[k][rest]), k
        assert not torch.isfinite(got[k][200].float()).any(), k
    assert not torch.isfinite(got["loss"][17])


def test_large_logits(lc):
    N, d, V = 200, 256, 900
    H, W, y, w, gl = _inputs(N, d, V, scale=60.0)
    ref = _reference(H, W, y, w, gl, None, 1.0)
    assert ref["zmax"] > 150
    out = _run(lc, H, W, y, w, gl, None, 1.0)
    tol = 2e-5 * (1.0 + ref["zmax"])
    assert float((out["loss"].double() - ref["loss"]).abs().max()) <= tol * 1.5
    # p moves by at most the logits' error relative to itself
    for k in ("dH", "dW"):
        off = float(torch.linalg.norm(out[k].double() - ref[k]) / torch.linalg.norm(ref[k]))
        assert off <= 2.0 ** -8 + 2 * tol, (k, off)


def test_row_pitch_and_another_stream(lc):
    N, d, V = 333, 200, 450
    H, W, y, w, gl = _inputs(N, d, V, mask="half")
    wide = torch.full((N, d + 56), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + d] = H
    into = torch.full((N, d + 24), 3.0, dtype=torch.bfloat16, device="cuda")
    ref = _reference(H, W, y, w, gl, None, 1.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        loss = torch.empty((N,), device="cuda")
        lse = torch.empty((N,), device="cuda")
        lc.loca_head_loss(wide[:, 8:8 + d], W, y, loss, lse=lse, w=w)
        lc.loca_head_loss_backward(wide[:, 8:8 + d], W, y, lse, dH=into[:, 16:16 + d], w=w, dloss=gl)
    s.synchronize()
    _check({"loss": loss, "lse": lse, "dH": into[:, 16:16 + d]}, ref, w)
    assert torch.all(into[:, :16] == 3.0) and torch.all(into[:, 16 + d:] == 3.0)


@pytest.mark.parametrize("N,d,V,dw", [(17000, 64, 300, False), (9000, 72, 70001, False), (3000, 64, 200000, True)])
def test_pieces_of_rows_and_of_the_vocabulary(lc, N, d, V, dw):
    """More rows than a forward piece; more rows and a larger vocabulary than a backward piece."""
    H, W, y, w, gl = _inputs(N, d, V, mask="half")
    out = _run(lc, H, W, y, w, gl, None, 1.0, dw=dw)
    live = torch.nonzero(y >= 0)[:, 0]
    dW = torch.zeros((V, d), dtype=torch.float64, device="cuda")
    for rows in live.split(1000):
        ref = _reference(H[rows], W, y[rows], w[rows], gl[rows], None, 1.0)
        dW += ref.pop("dW")
        _check({k: out[k][rows] for k in ("loss", "lse", "dH")}, ref, w[rows])
    if dw:
        assert float(torch.linalg.norm(out["dW"].double() - dW)) <= 2.0 ** -8 * float(torch.linalg.norm(dW))


def test_gradients_against_differences(lc):
    """Central differences of the summed loss along random directions of H and of W.  H and the
    perturbation are multiples of 1/16 below 8 and W of 1/512 below 1/4 in size, so H +- e and W +- e
    are exact in bf16; logits move by about 0.1, so the difference quotient's third-order term is below
    0.2%, the gradients' rounding 0.4%, and the fp32 losses' 1e-5: held to 1%."""
    N, d, V = 64, 64, 400
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    H = (torch.randint(-64, 65, (N, d), generator=g, device="cuda") / 16.0).to(torch.bfloat16)
    W = (torch.randint(-60, 61, (V, d), generator=g, device="cuda") / 512.0).to(torch.bfloat16)
    y = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    y[5] = -1
    one = torch.ones((N,), device="cuda")
    out = _run(lc, H, W, y, one, one, None, 1.0)

    def total(Hx, Wx):
        loss = torch.empty((N,), device="cuda")
        lc.loca_head_loss(Hx, Wx, y, loss)
        return float(loss.double().sum())

    # along the gradient's signs, so that the directional derivative is large
    D = torch.sign(out["dH"].float())
    got = (total((H.float() + D / 16).to(torch.bfloat16), W) - total((H.float() - D / 16).to(torch.bfloat16), W)) * 8
    want = float((out["dH"].double() * D.double()).sum())
    assert abs(got - want) <= 0.01 * abs(want)
    D = torch.sign(out["dW"].float())
    got = (total(H, (W.float() + D / 512).to(torch.bfloat16)) - total(H, (W.float() - D / 512).to(torch.bfloat16))) * 256
    want = float((out["dW"].double() * D.double()).sum())
    assert abs(got - want) <= 0.01 * abs(want)


def test_same_bits_every_time(lc):
    H, W, y, w, gl = _inputs(1000, 328, 5000, mask="half")
    a = _run(lc, H, W, y, w, gl, None, 1.0)
    b = _run(lc, H, W, y, w, gl, None, 1.0)
    for k in a:
        assert torch.equal(a[k], b[k]), k


def test_no_tokens(lc):
    W = torch.randn((40, 64), device="cuda").to(torch.bfloat16)
    H = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    y = torch.empty((0,), dtype=torch.int32, device="cuda")
    e = torch.empty((0,), device="cuda")
    lc.loca_head_loss(H, W, y, e, lse=e)
    dW = torch.full((40, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    lc.loca_head_loss_backward(H, W, y, e, dH=torch.empty_like(H), dW=dW)
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0 and torch.all(dW == 0)


def test_agrees_with_the_error_from_logits(lc):
    """E equals loca_error's on the same logits (fp32), so the adaptation pass can start from either."""
    N, d, V, C = 200, 128, 2000, 4
    H, W, y, w, _ = _inputs(N, d, V)
    cols = torch.tensor([1999, 7, 256, 255], dtype=torch.int32, device="cuda")
    word = torch.randint(0, C, (N,), device="cuda", dtype=torch.int32)
    word[3] = -1
    y = torch.where(word < 0, -1, cols[word.clamp(min=0).long()])
    E = torch.empty((N, C), device="cuda")
    loss = torch.empty((N,), device="cuda")
    lc.loca_head_loss(H, W, y, loss, w=w, label_cols=cols, E=E)
    z = (H.double() @ W.double().T).float()
    E2, ce = torch.empty_like(E), torch.empty_like(loss)
    lc.loca_error(z, cols, word, E2, w=w, ce=ce)
    torch.cuda.synchronize()
    tol = 2e-5 * (1.0 + float(z.abs().max())) * float(w.max())
    assert float((E - E2).abs().max()) <= tol and float((loss - ce).abs().max()) <= tol


def test_refusals(lc):
    N, d, V = 16, 64, 32
    H, W, y, w, _ = _inputs(N, d, V)
    loss = torch.empty((N,), device="cuda")
    ok = dict(lse=loss)
    with pytest.raises(TypeError):
        lc.loca_head_loss(H.float(), W, y, loss)
    with pytest.raises(TypeError):
        lc.loca_head_loss(H.cpu(), W, y, loss)
    with pytest.raises(TypeError):
        lc.loca_head_loss(H, W, y.long(), loss)
    with pytest.raises(ValueError):
        lc.loca_head_loss(H, W[:, :32].contiguous(), y, loss)
    with pytest.raises(ValueError):
        lc.loca_head_loss(H, W, y[:8].contiguous(), loss)
    with pytest.raises(ValueError):
        lc.loca_head_loss(H.T.contiguous().T, W, y, loss)
    with pytest.raises(ValueError):  # E without label words
        lc.loca_head_loss(H, W, y, loss, E=torch.empty((N, 3), device="cuda"))
    with pytest.raises(lc.LocaError) as e:  # d = 60 is no multiple of 8
        lc.loca_head_loss(H[:, :60].contiguous(), W[:, :60].contiguous(), y, loss)
    assert e.value.status == 2
    with pytest.raises(lc.LocaError) as e:  # rows 2 bytes off a 16-byte boundary
        wide = torch.zeros((N, d + 8), dtype=torch.bfloat16, device="cuda")
        lc.loca_head_loss(wide[:, 1:1 + d], W, y, loss)
    assert e.value.status == 3
    with pytest.raises(lc.LocaError) as e:
        lc.loca_head_loss_backward(H, W, y, **ok)
    assert e.value.status == 1
    with pytest.raises(lc.LocaError) as e:
        lc.loca_head_loss_backward(H, W, y, loss, dH=torch.empty_like(H), grad_scale=float("nan"))
    assert e.value.status == 1
    with pytest.raises(ValueError):
        lc.loca_head_loss(H, W, y, loss, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
