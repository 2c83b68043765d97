"""Global gradient norm and clipping against the definition in 64 bits.

Tolerances, fixed before the first run: a thread sums at most 64 squares in fp32 (64 * 2^-24 relative at
worst), the rest is fp64 and the norm is the square root, rounded to fp32: 2e-6 + 6e-8.  A clipped fp32
value has the factor's and one product's rounding on top (2^-23 in all), a bf16 one a rounding of 2^-9.
"""

import math

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


def _tensors(sizes, dtypes, seed=0, scale=0.1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + len(sizes))
    return [(scale * torch.randn((n,), generator=g, device="cuda")).to(dtypes[i % len(dtypes)])
            for i, n in enumerate(sizes)]


def _check(lc, grads, max_norm, out=None):
    want = math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in grads))
    f = max_norm / want if want > max_norm else 1.0
    ref = [t.double() * f for t in grads]
    norm = torch.full((1,), float("nan"), device="cuda")
    lc.GradClip(grads, out=out).run(max_norm, norm)
    torch.cuda.synchronize()
    assert abs(float(norm) - want) <= 2.1e-6 * want
    for got, r in zip(grads if out is None else out, ref):
        if got.dtype == torch.float32:
            assert torch.all((got.double() - r).abs() <= 2.2e-6 * r.abs() + 1e-45)
        else:
            low = (r.abs() * (1 - 2.2e-6)).to(torch.bfloat16)
            high = (r.abs() * (1 + 2.2e-6)).to(torch.bfloat16)
            assert torch.all((got.abs() >= low) & (got.abs() <= high))
            assert torch.all((got == 0) | (got.sign() == r.sign().to(got.dtype)))


F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("sizes", [
    [1], [7], [8192], [8193, 1, 0, 3], [5, 100000, 31], [896 * 8] * 48, [17] * 300, [3] * 2500, [2_000_003, 12],
])
@pytest.mark.parametrize("dtypes", [[F32], [BF16], [F32, BF16]])
@pytest.mark.parametrize("max_norm", [0.01, 1e6])
def test_norm_and_clipping(lc, sizes, dtypes, max_norm):
    _check(lc, _tensors(sizes, dtypes), max_norm)
    grads = _tensors(sizes, dtypes, seed=1)
    _check(lc, grads, max_norm, out=[torch.full_like(t, float("nan")) for t in grads])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_views_at_every_alignment(lc, dtype):
    base = _tensors([40000], [dtype])[0]
    into = torch.full((40000,), 5.0, dtype=dtype, device="cuda")
    grads = [base[1000 * i + i:1000 * i + i + 900 + i] for i in range(20)]
    out = [into[1000 * i + 3 * i:1000 * i + 3 * i + 900 + i] for i in range(20)]
    _check(lc, grads, 0.5, out=out)
    touched = torch.zeros((40000,), dtype=torch.bool, device="cuda")
    for i in range(20):
        touched[1000 * i + 3 * i:1000 * i + 3 * i + 900 + i] = True
    assert torch.all(into[~touched] == 5.0)
    _check(lc, grads, 0.5)


@pytest.mark.parametrize("scale", [1e-25, 1e-22, 1e25, 1e30])
def test_squares_outside_fp32(lc, scale):
    _check(lc, _tensors([70000, 50], [F32], scale=scale), scale)


def test_zeros_and_a_norm_at_the_limit(lc):
    grads = [torch.zeros((5000,), device="cuda")]
    norm = torch.ones((1,), device="cuda")
    lc.GradClip(grads).run(1.0, norm)
    assert float(norm) == 0.0 and torch.all(grads[0] == 0)
    grads = [torch.full((4,), 0.5, device="cuda")]  # norm exactly 1: not clipped
    lc.GradClip(grads).run(1.0, norm)
    assert float(norm) == 1.0 and torch.all(grads[0] == 0.5)


def test_norms_that_are_not_finite(lc):
    norm = torch.zeros((1,), device="cuda")
    grads = _tensors([9000, 10], [F32])
    grads[1][3] = float("nan")
    before = [t.clone() for t in grads]
    lc.GradClip(grads).run(1.0, norm)
    assert math.isnan(float(norm)) and torch.equal(grads[0], before[0])
    grads[1][3] = float("-inf")
    lc.GradClip(grads).run(1.0, norm)
    assert math.isinf(float(norm)) and torch.all(grads[0] == 0)


def test_norm_alone_and_no_tensors(lc):
    grads = _tensors([10001], [BF16])
    before = grads[0].clone()
    _check(lc, grads, math.inf)
    assert torch.equal(grads[0], before)
    norm = torch.ones((1,), device="cuda")
    lc.GradClip([]).run(1.0, norm)
    assert float(norm) == 0.0


def test_same_bits_on_another_stream(lc):
    grads = _tensors([300000, 77, 5000], [F32, BF16])
    out = [[torch.empty_like(t) for t in grads] for _ in range(2)]
    norms = torch.zeros((2, 1), device="cuda")
    lc.GradClip(grads, out=out[0]).run(0.5, norms[0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        lc.GradClip(grads, out=out[1]).run(0.5, norms[1])
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(norms[0], norms[1])
    for a, b in zip(*out):
        assert torch.equal(a, b)


def test_refusals(lc):
    g = torch.ones((8,), device="cuda")
    norm = torch.zeros((1,), device="cuda")
    with pytest.raises(TypeError):
        lc.GradClip([g.double()])
    with pytest.raises(TypeError):
        lc.GradClip([g.cpu()])
    with pytest.raises(TypeError):
        lc.GradClip([g], out=[g.to(torch.bfloat16)])
    with pytest.raises(ValueError):
        lc.GradClip([g], out=[])
    with pytest.raises(ValueError):
        lc.GradClip([torch.ones((4, 4), device="cuda").T[:, :2]])
    for bad in (0.0, -1.0, float("nan")):
        with pytest.raises(lc.LocaError) as e:
            lc.GradClip([g]).run(bad, norm)
        assert e.value.status == 1
    with pytest.raises(ValueError):
        lc.GradClip([g]).run(1.0, torch.zeros((2,), device="cuda"))
