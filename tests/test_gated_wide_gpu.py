"""Gated feed-forward and its gradients in the wide shape of the pair product (256 x 512 by two CTAs, two accumulators that
share A), which prompts, probes and training steps of real widths take in every product: sizes whose last tile has no
second accumulator, ragged rows and columns, and sums over 2 f of up to 32768 terms that run on without a restart.

Tolerances as in the operator's other tests, from the definition in 64 bits, element by element, but with what a running
sum may lose counted for each product: a step of 16 k loses up to 2^-22 of the running sum, toward zero, and a running
sum is at most the sum S of the terms' magnitudes.  H, dG, dU, dWg and dWu restart after 16384 k at the latest, dX
after 32768, so a sum over K terms is within  c(K, most) S,  c = ceil(min(K, most) / 16) 2^-22 + 2^-20.
"""

import re

import pytest
import test_gated_gpu as gated
import torch

pytestmark = pytest.mark.gpu
lc = gated.lc  # the fixture
U = gated.U


def _c(K, most=16384):
    return -(-min(K, most) // 16) * 2.0 ** -22 + 2.0 ** -20


def _reference(X, Wg, Wu, dH, act):
    """Values and how far each may be off (the derivation is that of the operator's other tests)."""
    x, wg, wu, dh = X.double(), Wg.double(), Wu.double(), dH.double()
    d, f, N = x.shape[1], wg.shape[0], x.shape[0]
    g, u = x @ wg.T, x @ wu.T
    a, da = gated._act(act, g)
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
    tol["dX"] = (edg @ wg.abs() + edu @ wu.abs() + _c(2 * f, 32768) * sums) * (1 + U) + U * val["dX"].abs()
    for name, v, e in (("dWg", dg, edg), ("dWu", du, edu)):
        val[name] = v.T @ x
        tol[name] = (e.T @ x.abs() + _c(N) * ((v.abs() + e).T @ x.abs())) * (1 + U) + U * val[name].abs()
    return val, tol


def _shapes(run):
    """What `run` launches of the pair product: {use: template number of its shape}, 1 the wide one."""
    events, tries = [], 0
    while not events and tries < 4:  # (a process's first recording may come out empty)
        tries += 1
        with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
            run()
            torch.cuda.synchronize()
        events = prof.key_averages()
    found = {}
    for e in events:
        m = re.search(r"k_gemm_pair<(?:\(int\))?(\d), (\w+), (\w+), (.*)", e.key)
        if m:
            rest = m[4]
            use = ("dX" if "SecondPair" in rest else "back" if "EpiGateBack" in rest else "H" if "EpiGate" in rest else
                   "dW" if m[2] in ("true", "1") else rest)
            found.setdefault(use, set()).add(int(m[1]))
    return found


WIDE = [
    (1900, 3080, 1288, "silu"),   # 8 columns in the last tiles: their second accumulators hold nothing
    (1291, 3080, 2312, "gelu"),
    (2301, 2056, 3336, "gelu"),
    (3801, 1544, 3464, "silu"),   # 136 columns: 8 of the second accumulator
    (4096, 2048, 8192, "silu"),   # whole tiles
    (1291, 4104, 8328, "silu"),   # 2 f past 16384
    (1531, 5120, 13656, "gelu"),  # 27312, 88 columns in the last tiles
]


@pytest.mark.parametrize("N,d,f,act", WIDE)
def test_wide_tiles_match_definition(lc, N, d, f, act):
    X, Wg, Wu, dH = gated._inputs(N, d, f)
    val, tol = _reference(X, Wg, Wu, dH, act)
    gated._check(gated._run(lc, X, Wg, Wu, dH, act), val, tol)
    alone = gated._run(lc, X, Wg, Wu, dH, act, ("dX",))
    gated._check(alone, {"dX": val["dX"]}, {"dX": tol["dX"]})


@pytest.mark.parametrize("N,d,f,act", WIDE)
def test_these_sizes_take_wide_tiles(lc, N, d, f, act):
    """The choice is by cost and may change: then the sizes above have to change with it."""
    X, Wg, Wu, dH = gated._inputs(N, d, f)
    gated._run(lc, X, Wg, Wu, dH, act)
    found = _shapes(lambda: gated._run(lc, X, Wg, Wu, dH, act))
    assert found == {"H": {1}, "back": {1}, "dX": {1}, "dW": {1}}, found


@pytest.mark.parametrize("N,d,f", [(1291, 4104, 8328), (1531, 5120, 13656)])
def test_long_sums_that_cancel(lc, N, d, f):
    """The second half of the columns has the first half's weights and its dH negated, so that dG and dU of both are equal
    and opposite bit for bit (the same sums, rounded the same way) and dX is zero; all of the first half's terms are
    positive, so the running sum goes up to the sum of the first half of dG's, back to zero, and the same for dU: what is
    left is what the steps lost, at most c(2 f, 32768) times the larger of both."""
    X, Wg, Wu, dH = (t.abs() for t in gated._inputs(N, d, f))
    Wg, Wu = Wg / 64, Wu / 64  # (exact: powers of two; G and U are then about one)
    h = f // 2
    Wg[h:], Wu[h:], dH[:, h:] = Wg[:h], Wu[:h], -dH[:, :h]
    dX = gated._run(lc, X, Wg, Wu, dH, "silu", ("dX",))["dX"]
    x, wg, wu, dh = X.double(), Wg[:h].double(), Wu[:h].double(), dH[:, :h].double()
    a, da = gated._act("silu", x @ wg.T)
    # with a rounding of dG and dU (2^-8), one of dX and what G and U may be off (below 2^-9)
    most = torch.maximum((dh * (x @ wu.T) * da) @ wg, (dh * a) @ wu) * (1 + 2.0 ** -6)
    assert bool((dX.double().abs() <= _c(2 * f, 32768) * most).all()), float((dX.double().abs() / most).max())
