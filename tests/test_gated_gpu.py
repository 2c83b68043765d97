"""Gated feed-forward and its gradients against the definition in 64 bits, element by element.

Tolerances, derived before the first run.  Products of bf16 values are exact in fp32; the tensor cores lose up
to 2^-22 of the running sum at each step of 16 k, toward zero, and a running sum is at most the sum S of the
terms' magnitudes.  A sum restarts after 4096 k, or runs over up to 16384 k in the wide tiles, so a sum over K terms is
within  c(K) S,  c(K) = ceil(min(K, 16384) / 16) 2^-22 + 2^-20  of its exact value (2^-20: the joins of
segments and ranges, round to nearest).  The activation and its derivative add 2^-20 of themselves (two
approximate functions of 2^-22 each and four roundings), and move by at most |act'| <= 1.13 and
|act''| <= 1 times the error of their argument (SiLU: 1.10 and 0.5, GELU: 1.13 and 0.8).  Each rounding to bf16
is half a step, 2^-8 of the value: one of dG and dU, one of each output.
"""

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -8  # a rounding to bf16


@pytest.fixture(scope="module")
def lc():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_03020_gb300 import _build

    _build.build()
    from paper_2608_03020_gb300 import loca

    loca.lib()
    return loca


def _act(name, g):
    s = torch.sigmoid(g) if name == "silu" else torch.sigmoid(2 * (2 / torch.pi) ** 0.5 * (g + 0.044715 * g ** 3))
    slope = 1.0 if name == "silu" else 2 * (2 / torch.pi) ** 0.5 * (1 + 3 * 0.044715 * g ** 2)
    return g * s, s + g * s * (1 - s) * slope


def _inputs(N, d, f, seed=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 7 * N + 11 * d + 13 * f)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    X = rn(N, d).to(torch.bfloat16)
    Wg, Wu = (scale * rn(f, d) / d ** 0.5).to(torch.bfloat16), (rn(f, d) / d ** 0.5).to(torch.bfloat16)
    return X, Wg, Wu, rn(N, f).to(torch.bfloat16)


def _c(K):
    return -(-min(K, 16384) // 16) * 2.0 ** -22 + 2.0 ** -20


def _reference(X, Wg, Wu, dH, act):
    """Values and how far each may be off."""
    x, wg, wu, dh = X.double(), Wg.double(), Wu.double(), dH.double()
    N, d = x.shape
    f = wg.shape[0]
    g, u = x @ wg.T, x @ wu.T
    a, da = _act(act, g)
    eg, eu = _c(d) * (x.abs() @ wg.abs().T), _c(d) * (x.abs() @ wu.abs().T)
    ea = 1.13 * eg + 2.0 ** -20 * a.abs()
    eda = eg + 2.0 ** -20 * (1.13 + da.abs())
    val, tol = {}, {}
    val["H"] = a * u
    tol["H"] = (ea * (u.abs() + eu) + a.abs() * eu) * (1 + U) + U * val["H"].abs()
    dg, du = dh * u * da, dh * a
    edg = dh.abs() * (eu * (da.abs() + eda) + u.abs() * eda) * (1 + U) + U * dg.abs()
    edu = dh.abs() * ea * (1 + U) + U * du.abs()
    val["dX"] = dg @ wg + du @ wu
    sums = (dg.abs() + edg) @ wg.abs() + (du.abs() + edu) @ wu.abs()
    tol["dX"] = (edg @ wg.abs() + edu @ wu.abs() + _c(2 * f) * sums) * (1 + U) + U * val["dX"].abs()
    for name, v, e in (("dWg", dg, edg), ("dWu", du, edu)):
        val[name] = v.T @ x
        tol[name] = (e.T @ x.abs() + _c(N) * ((v.abs() + e).T @ x.abs())) * (1 + U) + U * val[name].abs()
    return val, tol


def _run(lc, X, Wg, Wu, dH, act, want=("H", "dX", "dWg", "dWu")):
    N, d = X.shape
    f = Wg.shape[0]
    shapes = {"H": (N, f), "dX": (N, d), "dWg": (f, d), "dWu": (f, d)}
    out = {k: torch.full(shapes[k], float("nan"), dtype=torch.bfloat16, device="cuda") for k in want}
    if "H" in out:
        lc.loca_gated(X, Wg, Wu, out["H"], act=act)
    grads = {k: v for k, v in out.items() if k != "H"}
    if grads:
        lc.loca_gated_backward(X, Wg, Wu, dH, act=act, **grads)
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0
    return out


def _check(out, val, tol):
    for k in out:
        off = (out[k].double() - val[k]).abs()
        bad = ~(off <= tol[k] + 1e-37)
        assert not bool(bad.any()), (k, int(bad.sum()), float((off / (tol[k] + 1e-37)).nan_to_num(1e30).max()))


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("N,d,f", [
    (1, 8, 8), (1, 64, 64), (2, 72, 136), (37, 896, 200), (63, 200, 1032), (128, 512, 264), (129, 64, 72),
    (255, 136, 1000), (256, 1024, 256), (257, 328, 520), (300, 72, 2056), (1000, 904, 648), (513, 2048, 128),
])
def test_matches_definition(lc, N, d, f, act):
    X, Wg, Wu, dH = _inputs(N, d, f)
    _check(_run(lc, X, Wg, Wu, dH, act), *_reference(X, Wg, Wu, dH, act))


@pytest.mark.parametrize("N,d,f", [(3000, 1024, 2048), (4096, 512, 1536), (1, 3584, 14336), (100, 2048, 9000)])
def test_many_tiles_and_long_sums(lc, N, d, f):
    """More tiles than the GPU takes at once (both pair shapes), k ranges of dX, wide weights against one token."""
    X, Wg, Wu, dH = _inputs(N, d, f)
    _check(_run(lc, X, Wg, Wu, dH, "silu"), *_reference(X, Wg, Wu, dH, "silu"))


@pytest.mark.parametrize("N,d,f", [(64, 20000, 96), (700, 18000, 136)])
def test_k_beyond_the_wide_tiles(lc, N, d, f):
    X, Wg, Wu, dH = _inputs(N, d, f)
    val, tol = _reference(X, Wg, Wu, dH, "gelu")
    _check(_run(lc, X, Wg, Wu, dH, "gelu"), val, tol)


@pytest.mark.parametrize("want", [("dX",), ("dWg",), ("dWu",), ("dX", "dWu"), ("dWg", "dWu")])
def test_any_of_the_gradients_alone(lc, want):
    X, Wg, Wu, dH = _inputs(300, 136, 264)
    _check(_run(lc, X, Wg, Wu, dH, "silu", want), *_reference(X, Wg, Wu, dH, "silu"))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_far_arguments(lc, act):
    """Gates from -300 to 300: the sigmoid is 0 or 1, powers of g must not overflow, tails keep their size."""
    X, Wg, Wu, dH = _inputs(200, 64, 72, scale=60.0)
    out = _run(lc, X, Wg, Wu, dH, act)
    val, tol = _reference(X, Wg, Wu, dH, act)
    # what underflows in fp32 (a sigmoid below 2^-126) may come out as 0
    tol = {k: t + 2.0 ** -100 for k, t in tol.items()}
    _check(out, val, tol)
    assert all(bool(torch.isfinite(t).all()) for t in out.values())


def test_gradients_against_differences(lc):
    """<dX, v> and <dW, v> against (F(. + e v) - F(. - e v)) / 2e of F = sum dH * H in 64 bits."""
    X, Wg, Wu, dH = _inputs(150, 200, 328)
    out = _run(lc, X, Wg, Wu, dH, "gelu")
    _, tol = _reference(X, Wg, Wu, dH, "gelu")
    base = {"dX": X.double(), "dWg": Wg.double(), "dWu": Wu.double()}

    def total(x):
        return float((dH.double() * _act("gelu", x["dX"] @ x["dWg"].T)[0] * (x["dX"] @ x["dWu"].T)).sum())

    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for k in base:
        v = torch.randn(base[k].shape, generator=g, device="cuda", dtype=torch.float64)
        e = 1e-5
        num = (total({**base, k: base[k] + e * v}) - total({**base, k: base[k] - e * v})) / (2 * e)
        # differences: e^2 / 6 of a third derivative that is about as large as F itself, and rounding / e
        slack = 1e-6 * float((dH.double().abs()).sum())
        assert abs(num - float((out[k].double() * v).sum())) <= float((tol[k] * v.abs()).sum()) + slack, k


@pytest.mark.parametrize("N", [5, 300])
def test_rows_apart_stay_apart(lc, N):
    """A row of NaN or infinities spoils its own outputs and, in the row-wise outputs, no other's."""
    X, Wg, Wu, dH = _inputs(N, 136, 264)
    clean = _run(lc, X, Wg, Wu, dH, "silu")
    X2, dH2 = X.clone(), dH.clone()
    X2[1], X2[3, 5], dH2[2] = float("nan"), float("inf"), float("nan")
    out = _run(lc, X2, Wg, Wu, dH2, "silu")
    keep = [i for i in range(N) if i not in (1, 2, 3)]
    for k in ("H", "dX"):
        assert torch.equal(out[k][keep], clean[k][keep])
    assert bool(out["H"][1].isnan().all()) and bool(out["dX"][1].isnan().all()) and bool(out["dX"][2].isnan().all())
    assert torch.equal(out["H"][2], clean["H"][2]) and not bool(out["H"][3].isfinite().all())
    assert bool(out["dWg"].isnan().any()) and bool(out["dWu"].isnan().any())


@pytest.mark.parametrize("N", [3, 500])
def test_spaced_rows(lc, N):
    """Rows inside wider buffers: the same bits, and what lies between them stays."""
    d, f = 136, 328
    X, Wg, Wu, dH = _inputs(N, d, f)
    want = _run(lc, X, Wg, Wu, dH, "silu")
    big = {k: torch.full((N, c + 24), 7.0, dtype=torch.bfloat16, device="cuda") for k, c in
           (("X", d), ("dH", f), ("H", f), ("dX", d))}
    view = {k: t[:, 8:8 + t.shape[1] - 24] for k, t in big.items()}
    view["X"].copy_(X)
    view["dH"].copy_(dH)
    lc.loca_gated(view["X"], Wg, Wu, view["H"])
    lc.loca_gated_backward(view["X"], Wg, Wu, view["dH"], dX=view["dX"])
    torch.cuda.synchronize()
    for k in ("H", "dX"):
        assert torch.equal(view[k], want[k])
    for t in big.values():
        assert bool((t[:, :8] == 7).all()) and bool((t[:, -16:] == 7).all())
    # X and H side by side in one buffer
    both = torch.zeros((N, d + f), dtype=torch.bfloat16, device="cuda")
    both[:, :d] = X
    lc.loca_gated(both[:, :d], Wg, Wu, both[:, d:])
    assert torch.equal(both[:, d:], want["H"])


def test_pieces_of_the_rows(lc):
    """dG and dU of all rows past 1 GiB: the rows come in pieces, and give the bits that each gives alone."""
    N, d, f = 70001, 64, 4096
    X, Wg, Wu, dH = _inputs(N, d, f)
    assert lc.gated_backward_workspace_size(N, d, f, True, False) < (1 << 30) + (1 << 28)
    out = _run(lc, X, Wg, Wu, dH, "silu", ("dX",))
    for a, b in ((0, 300), (35000, 35300), (N - 259, N)):
        val, tol = _reference(X[a:b], Wg, Wu, dH[a:b], "silu")
        _check({"dX": out["dX"][a:b]}, {"dX": val["dX"]}, {"dX": tol["dX"]})


def test_pieces_of_the_columns(lc):
    """With dWg and dWu past 4 GiB the columns come in pieces and dX adds them up in fp32."""
    N, d, f = 300000, 64, 4096
    X, Wg, Wu, dH = _inputs(N, d, f)
    out = _run(lc, X, Wg, Wu, dH, "silu", ("dX", "dWg", "dWu"))
    for a, b in ((0, 300), (N - 259, N)):
        val, tol = _reference(X[a:b], Wg, Wu, dH[a:b], "silu")
        _check({"dX": out["dX"][a:b]}, {"dX": val["dX"]}, {"dX": tol["dX"]})
    for c in (slice(0, 40), slice(4050, 4096)):  # some rows of the weights' gradients
        val, tol = _reference(X, Wg[c], Wu[c], dH[:, c], "silu")
        _check({k: out[k][c] for k in ("dWg", "dWu")}, val, tol)


def test_no_rows(lc):
    X, Wg, Wu, dH = _inputs(0, 64, 72)
    out = _run(lc, X, Wg, Wu, dH, "silu")
    assert bool((out["dWg"] == 0).all()) and bool((out["dWu"] == 0).all())


def test_the_same_bits_again(lc):
    X, Wg, Wu, dH = _inputs(777, 904, 1336)
    a, b = _run(lc, X, Wg, Wu, dH, "gelu"), _run(lc, X, Wg, Wu, dH, "gelu")
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_python_refusals(lc):
    X, Wg, Wu, dH = _inputs(10, 64, 72)
    H, dX = torch.empty_like(dH), torch.empty_like(X)
    with pytest.raises(ValueError, match="act"):
        lc.loca_gated(X, Wg, Wu, H, act="relu")
    with pytest.raises(ValueError):
        lc.loca_gated(X, Wg, Wu[:64], H)
    with pytest.raises(ValueError):
        lc.loca_gated(X, Wg, Wu, H[:, :64])
    with pytest.raises(TypeError):
        lc.loca_gated(X.float(), Wg, Wu, H)
    with pytest.raises(ValueError):
        lc.loca_gated_backward(X, Wg, Wu, dH, dX=dX, dWg=Wg[:8].clone())
    for bad in (dict(dX=X), dict(dWg=Wg), dict(dWu=Wg), dict(dWg=Wu)):
        with pytest.raises(lc.LocaError, match="overlap"):
            lc.loca_gated_backward(X, Wg, Wu, dH, **bad)
    with pytest.raises(lc.LocaError, match="required"):
        lc.loca_gated_backward(X, Wg, Wu, dH)
    sq = torch.empty((64, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(lc.LocaError, match="overlap"):
        lc.loca_gated(sq, sq.clone(), sq.clone(), sq)
