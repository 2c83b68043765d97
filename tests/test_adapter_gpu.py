"""Adapters beside a shared projection, forward and backward, against the definition in 64 bits.

Tolerances, fixed before the first run.  Outputs in bf16 carry one rounding of the sum (uniform within
2^-8 of a binade's size, so below 2^-9 in norm) and, for the low-rank term, of U and of s B (the same,
relative to that term): 2^-8 of the sum plus 2^-8 of the term, in norm.  Gradients of the adapters in float32: U and T from three-part
adapters, in three parts (2^-26 each), summed on the tensor cores in segments of 32 steps, each step
losing up to 2^-22 of the running sum: 32 * 2^-22 = 8e-6 in each of two sums, so 2e-5 of the products'
absolute sums; taken as 2e-5 in norm.  In bf16 one rounding more: 2^-9 + 2e-5.
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


def _inputs(N, d, o, k, n, ids="mixed", dtype=torch.float32, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + N + 3 * d + 5 * o + 7 * k + 11 * n)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    v = dict(X=rn(N, d).to(torch.bfloat16), W=(rn(o, d) / d ** 0.5).to(torch.bfloat16),
             A=(rn(n, d, k) / d ** 0.5).to(dtype), B=(rn(n, o, k) / k ** 0.5).to(dtype),
             scale=torch.rand((n,), generator=g, device="cuda") + 0.5, dY=rn(N, o).to(torch.bfloat16))
    if ids == "mixed":  # any order, some without an adapter, some ids past the last adapter
        i = torch.randint(-1, n + 1, (N,), generator=g, device="cuda")
    elif ids == "runs":
        i = torch.arange(N, device="cuda") * (n + 1) // max(N, 1) - 1
    elif ids == "none":
        i = torch.full((N,), -1, device="cuda")
    else:
        i = torch.full((N,), n - 1, device="cuda")
    v["ids"] = i.to(torch.int32)
    return v


def _reference(v):
    X, W, dY = v["X"].double(), v["W"].double(), v["dY"].double()
    A, B, s = v["A"].double(), v["B"].double(), v["scale"].double()
    n = A.shape[0]
    out = {"Y": X @ W.T, "dX": dY @ W, "dA": torch.zeros_like(A), "dB": torch.zeros_like(B)}
    low = {"Y": torch.zeros_like(out["Y"]), "dX": torch.zeros_like(out["dX"])}
    for a in torch.unique(v["ids"]).tolist():
        if a < 0 or a >= n:
            continue
        r = torch.nonzero(v["ids"] == a)[:, 0]
        U, T = X[r] @ A[a], s[a] * (dY[r] @ B[a])
        low["Y"][r] = s[a] * (U @ B[a].T)
        low["dX"][r] = T @ A[a].T
        out["dA"][a] = X[r].T @ T
        out["dB"][a] = s[a] * (dY[r].T @ U)
    out["Y"] += low["Y"]
    out["dX"] += low["dX"]
    return out, low


def _run(lc, v, grads=("dX", "dA", "dB"), out=None):
    n, d, k = v["A"].shape
    o = v["B"].shape[1]
    N = v["X"].shape[0]
    nan = float("nan")
    ad = lc.AdapterSet(n, d, o, k).pack(v["A"], v["B"], v["scale"])
    plan = lc.AdapterPlan(v["ids"], n)
    got = {"Y": torch.full((N, o), nan, dtype=torch.bfloat16, device="cuda")}
    lc.loca_adapter_apply(v["X"], v["W"], ad, plan, got["Y"])
    new = {"dX": lambda: torch.full((N, d), nan, dtype=torch.bfloat16, device="cuda"),
           "dA": lambda: torch.full_like(v["A"], nan), "dB": lambda: torch.full_like(v["B"], nan)}
    want = {g: new[g]() for g in grads}
    if want:
        lc.loca_adapter_backward(v["X"], v["dY"], v["W"], ad, plan, **want)
    got.update(want)
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0
    return got


def _check(got, ref, low):
    for key, x in got.items():
        off = float(torch.linalg.norm(x.double() - ref[key]))
        norm = float(torch.linalg.norm(ref[key]))
        if key in low:
            tol = 2.0 ** -8 * norm + 2.0 ** -8 * float(torch.linalg.norm(low[key]))
        else:
            tol = (2e-5 + (2.0 ** -9 if x.dtype == torch.bfloat16 else 0.0)) * norm
        assert off <= tol, (key, off / max(norm, 1e-300), tol / max(norm, 1e-300))


@pytest.mark.parametrize("N,d,o,k,n,ids", [
    (1, 8, 8, 1, 1, "last"), (1, 896, 64, 16, 3, "mixed"), (2, 72, 200, 5, 2, "mixed"), (17, 200, 136, 8, 40, "mixed"),
    (64, 2048, 896, 16, 96, "mixed"), (64, 1536, 520, 24, 2, "runs"), (128, 328, 256, 64, 1, "last"),
    (100, 256, 128, 33, 300, "mixed"), (129, 64, 136, 8, 1, "last"), (300, 136, 72, 12, 4, "runs"),
    (513, 520, 1032, 32, 5, "runs"), (700, 200, 328, 16, 200, "mixed"), (2049, 896, 896, 8, 1, "last"),
    (3000, 1536, 1024, 16, 3, "mixed"), (2500, 2048, 2056, 40, 7, "runs"), (1000, 896, 896, 16, 2, "none"),
    (4097, 512, 2048, 20, 1000, "mixed"),
])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_projection_and_gradients(lc, N, d, o, k, n, ids, dtype):
    v = _inputs(N, d, o, k, n, ids, dtype)
    ref, low = _reference(v)
    _check(_run(lc, v), ref, low)


@pytest.mark.parametrize("grads", [("dX",), ("dA",), ("dB",), ("dA", "dB"), ("dX", "dB")])
def test_each_gradient_alone(lc, grads):
    v = _inputs(700, 264, 392, 12, 5, "mixed")
    ref, low = _reference(v)
    _check(_run(lc, v, grads), ref, low)


@pytest.mark.parametrize("N", [40, 1500])
def test_tokens_outside_an_adapter_do_not_reach_it(lc, N):
    """Infinities, NaN and the lowest value in rows of tokens without an adapter, and of one request."""
    v = _inputs(N, 136, 264, 16, 3, "mixed")
    v["ids"][v["ids"] == 2] = -1
    v["ids"][N // 2] = 2
    ref, low = _reference(v)
    bad = v["ids"] < 0
    bad[N // 2] = True
    rows = torch.nonzero(bad)[:, 0]
    for name in ("X", "dY"):
        for j, value in enumerate((float("nan"), float("inf"), torch.finfo(torch.bfloat16).min)):
            v[name][rows[j::3], j] = value
    v["X"][N // 2], v["dY"][N // 2] = float("nan"), float("nan")
    got = _run(lc, v)
    good = ~bad
    for key in ("Y", "dX"):
        _check({key: got[key][good]}, {key: ref[key][good]}, {key: low[key][good]})
    for key in ("dA", "dB"):
        _check({key: got[key][:2].contiguous()}, {key: ref[key][:2]}, {})


def test_an_adapter_that_is_not_finite_stays_with_its_tokens(lc):
    v = _inputs(300, 72, 136, 8, 3, "mixed")
    ref, low = _reference(v)
    v["A"][1, 3, 2] = float("nan")
    v["B"][1, 5, 1] = float("inf")
    got = _run(lc, v)
    rest = v["ids"] != 1
    for key in ("Y", "dX"):
        _check({key: got[key][rest]}, {key: ref[key][rest]}, {key: low[key][rest]})
    for key in ("dA", "dB"):
        _check({key: got[key][[0, 2]]}, {key: ref[key][[0, 2]]}, {})


@pytest.mark.parametrize("N", [5, 600])
def test_row_pitch_and_another_stream(lc, N):
    v = _inputs(N, 136, 264, 12, 4, "mixed")
    ref, low = _reference(v)
    pad = lambda t, extra: torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=t.dtype, device="cuda")  # noqa: E731
    Xw, dYw = pad(v["X"], 24), pad(v["dY"], 40)
    Xw[:, 16:16 + 136] = v["X"]
    dYw[:, 8:8 + 264] = v["dY"]
    Yw = torch.full((N, 264 + 16), 3.0, dtype=torch.bfloat16, device="cuda")
    dXw = torch.full((N, 136 + 32), 3.0, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ad = lc.AdapterSet(4, 136, 264, 12).pack(v["A"], v["B"], v["scale"])
        plan = lc.AdapterPlan(v["ids"], 4)
        X, dY = Xw[:, 16:16 + 136], dYw[:, 8:8 + 264]
        dA, dB = torch.empty_like(v["A"]), torch.empty_like(v["B"])
        lc.loca_adapter_apply(X, v["W"], ad, plan, Yw[:, 8:8 + 264])
        lc.loca_adapter_backward(X, dY, v["W"], ad, plan, dX=dXw[:, 16:16 + 136], dA=dA, dB=dB)
    s.synchronize()
    assert lc.loca_device_status() == 0
    _check({"Y": Yw[:, 8:8 + 264], "dX": dXw[:, 16:16 + 136], "dA": dA, "dB": dB}, ref, low)
    for t, a, b in ((Yw, 8, 8 + 264), (dXw, 16, 16 + 136)):
        assert torch.all(t[:, :a] == 3.0) and torch.all(t[:, b:] == 3.0)


def test_next_step_and_repacked_adapters(lc):
    """One set and one plan used again: new ids, then new adapter values."""
    v = _inputs(200, 128, 128, 8, 6, "mixed")
    ad = lc.AdapterSet(6, 128, 128, 8).pack(v["A"], v["B"], v["scale"])
    plan = lc.AdapterPlan(v["ids"], 6)
    ws = torch.empty(lc.adapter_workspace_size(200, 128, 128, 8, 6), dtype=torch.uint8, device="cuda")
    for step in range(3):
        Y = torch.empty((200, 128), dtype=torch.bfloat16, device="cuda")
        lc.loca_adapter_apply(v["X"], v["W"], ad, plan, Y, workspace=ws)
        ref, low = _reference(v)
        _check({"Y": Y}, {"Y": ref["Y"]}, {"Y": low["Y"]})
        v["ids"] = torch.roll(v["ids"], 7)
        plan.update(v["ids"])
        v["A"], v["scale"] = v["A"] * 1.5, v["scale"] + 0.25
        ad.pack(v["A"], v["B"], v["scale"])


def test_scale_defaults_to_one(lc):
    v = _inputs(70, 64, 72, 4, 3, "mixed")
    v["scale"] = torch.ones((3,), device="cuda")
    ref, low = _reference(v)
    v["scale"] = None
    got = _run(lc, v)
    _check(got, ref, low)


def test_gradients_against_differences(lc):
    """Central differences of <dY, Y> along the gradients' signs.  Y is linear in X and bilinear in
    (A, B), so the quotient has no higher-order term; Y's rounding to bf16 averages over 300 x 264
    elements to below 1% of the difference, to which the quotient is held."""
    v = _inputs(300, 136, 264, 8, 2, "mixed")
    got = _run(lc, v)

    def total(**changed):
        w = dict(v, **changed)
        return float((_run(lc, w, ())["Y"].double() * v["dY"].double()).sum())

    X = torch.round(v["X"].float() * 8) / 8
    v["X"] = X.to(torch.bfloat16)
    got = _run(lc, v)
    D = torch.sign(got["dX"].float())
    quotient = (total(X=(X + D / 8).to(torch.bfloat16)) - total(X=(X - D / 8).to(torch.bfloat16))) * 4
    want = float((got["dX"].double() * D.double()).sum())
    assert abs(quotient - want) <= 0.01 * abs(want)
    for name, key in (("A", "dA"), ("B", "dB")):
        D = torch.sign(got[key]) * 0.05
        quotient = (total(**{name: v[name] + D}) - total(**{name: v[name] - D})) / 2
        want = float((got[key].double() * D.double()).sum())
        assert abs(quotient - want) <= 0.01 * abs(want), name


def test_same_bits_every_time(lc):
    for N in (33, 1111):
        v = _inputs(N, 392, 520, 16, 5, "mixed")
        a, b = _run(lc, v), _run(lc, v)
        for k in a:
            assert torch.equal(a[k], b[k]), k


def test_no_tokens(lc):
    v = _inputs(0, 64, 72, 4, 2, "none")
    got = _run(lc, v)
    assert torch.all(got["dA"] == 0) and torch.all(got["dB"] == 0)


def test_refusals(lc):
    v = _inputs(20, 64, 72, 4, 2, "mixed")
    ad = lc.AdapterSet(2, 64, 72, 4).pack(v["A"], v["B"], v["scale"])
    plan = lc.AdapterPlan(v["ids"], 2)
    Y = torch.empty((20, 72), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(lc.LocaError) as e:
        lc.AdapterSet(2, 64, 72, 65)
    assert e.value.status == 2
    with pytest.raises(lc.LocaError) as e:
        lc.AdapterSet(2, 60, 72, 4)
    assert e.value.status == 2
    with pytest.raises(ValueError):
        ad.pack(v["A"], v["A"])
    with pytest.raises(TypeError):
        ad.pack(v["A"], v["B"].to(torch.bfloat16))
    with pytest.raises(TypeError):
        lc.AdapterPlan(v["ids"].long(), 2)
    with pytest.raises(ValueError):
        plan.update(v["ids"][:10].contiguous())
    with pytest.raises(ValueError):  # a plan for other adapters
        lc.loca_adapter_apply(v["X"], v["W"], ad, lc.AdapterPlan(v["ids"], 3), Y)
    with pytest.raises(ValueError):
        lc.loca_adapter_apply(v["X"], v["W"].T.contiguous(), ad, plan, Y)
    with pytest.raises(TypeError):
        lc.loca_adapter_apply(v["X"].float(), v["W"], ad, plan, Y)
    with pytest.raises(lc.LocaError) as e:  # rows 2 bytes off a 16-byte boundary
        wide = torch.zeros((20, 72), dtype=torch.bfloat16, device="cuda")
        lc.loca_adapter_apply(wide[:, 1:65], v["W"], ad, plan, Y)
    assert e.value.status == 3
    with pytest.raises(lc.LocaError) as e:
        lc.loca_adapter_backward(v["X"], v["dY"], v["W"], ad, plan)
    assert e.value.status == 1
    with pytest.raises(ValueError):
        lc.loca_adapter_apply(v["X"], v["W"], ad, plan, Y, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
