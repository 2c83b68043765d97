"""The 4-bit projection with adapters beside it against the definition in 64 bits, element by element.

Tolerances, derived before the first run.  q - z and X are exact in bf16; the tensor cores lose at most 2^-22 of the
sum of the terms' magnitudes at each of the four steps of 64 k, and the scaled sums are added in fp32, one
rounding of 2^-24 of the running sum for each of at most d / 32 parts and the warps' sums:
c(d) = 2^-20 + (d / 32 + 16) 2^-24 of S = sum |x w|.  The low-rank term takes A and s B rounded to bf16 (2^-8 of each
value, and 2^-9 more of s B where s is not a power of two, taken as 2^-7 together) and sums in fp32.  Y is rounded once:
half a step, 2^-8.
"""

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -8


@pytest.fixture(scope="module")
def lc():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_03020_gb300 import _build

    _build.build()
    from paper_2608_03020_gb300 import loca

    loca.lib()
    return loca


def _weight(o, d, group, dtype, zeros, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 7 * o + 11 * d + group)
    codes = torch.randint(0, 256, (o, d // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = ((torch.rand((o, d // group), generator=g, device="cuda") + 0.1) * d ** -0.5).to(dtype)
    scales[::3] *= -1.0
    z = torch.randint(0, 16, scales.shape, generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    q = torch.stack([codes & 15, codes >> 4], 2).reshape(o, d // group, group).double()
    zd = 8.0 if z is None else z.double()[:, :, None]
    return codes, scales, z, (scales.double()[:, :, None] * (q - zd)).reshape(o, d)


def _tokens(N, d, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 3 * N + d)
    return torch.randn((N, d), generator=g, device="cuda").to(torch.bfloat16)


def _adapters(lc, N, d, o, k, n, dtype, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + N + 5 * k + n)
    A = (torch.randn((n, d, k), generator=g, device="cuda") * d ** -0.5).to(dtype)
    B = torch.randn((n, o, k), generator=g, device="cuda").to(dtype)
    scale = torch.rand((n,), generator=g, device="cuda") + 0.5
    ids = torch.randint(-1, n + 1, (N,), generator=g, device="cuda", dtype=torch.int32)  # -1 and n: none
    return A, B, scale, ids


def _reference(X, W, ad=None):
    x = X.double()
    d = x.shape[1]
    y = x @ W.T
    tol = (2.0 ** -20 + (d / 32 + 16) * 2.0 ** -24) * (x.abs() @ W.abs().T)
    if ad is not None:
        A, B, scale, ids = ad
        for a in range(A.shape[0]):
            rows = torch.nonzero(ids == a)[:, 0]
            if len(rows):
                sB = scale[a].double() * B[a].double()
                y[rows] += (x[rows] @ A[a].double()) @ sB.T
                tol[rows] += (2.0 ** -7 + 2.0 ** -8 + 2.0 ** -12) * ((x[rows].abs() @ A[a].double().abs()) @ sB.abs().T)
    return y, tol * (1 + U) + U * y.abs()


def _check(lc, X, weight, W, ad=None, **kw):
    N, o = X.shape[0], W.shape[0]
    Y = torch.full((N, o), float("nan"), dtype=torch.bfloat16, device="cuda")
    if ad is not None:
        A, B, scale, ids = ad
        kw["adapters"] = lc.AdapterSet(A.shape[0], X.shape[1], o, A.shape[2]).pack(A, B, scale)
        kw["plan"] = lc.AdapterPlan(ids, A.shape[0])
    lc.loca_q4_apply(X, weight, Y, **kw)
    torch.cuda.synchronize()
    assert lc.loca_device_status() == 0
    y, tol = _reference(X, W, ad)
    off = (Y.double() - y).abs()
    assert bool((off <= tol + 1e-37).all()), float((off / (tol + 1e-37)).nan_to_num(1e30).max())
    return Y


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,o,d,group", [
    (1, 1, 32, 32), (1, 16, 64, 64), (2, 17, 128, 128), (3, 33, 96, 32), (7, 31, 192, 64), (8, 64, 256, 128),
    (9, 100, 416, 32), (16, 129, 640, 128), (17, 48, 1056, 32), (32, 200, 320, 64), (33, 65, 256, 32), (64, 500, 384, 128),
    (65, 40, 160, 32), (200, 96, 128, 64),
])
def test_matches_definition(lc, N, o, d, group, dtype, zeros):
    codes, scales, z, W = _weight(o, d, group, dtype, zeros)
    _check(lc, _tokens(N, d), lc.Q4Weight(codes, scales, zeros=z), W)


@pytest.mark.parametrize("N,o,d,group", [
    (1, 3584, 3584, 128), (1, 20480, 5120, 64), (5, 40001, 2048, 32), (64, 9000, 4096, 128), (1, 64, 65536, 64), (130, 2000, 8192, 32),
])
def test_large(lc, N, o, d, group):
    """Every number of warps on the same rows, blocks past one round of the SMs, long rows, several token blocks."""
    codes, scales, z, W = _weight(o, d, group, torch.bfloat16, True)
    _check(lc, _tokens(N, d), lc.Q4Weight(codes, scales, zeros=z), W)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,o,d,k,n", [
    (1, 8, 64, 1, 1), (1, 3584, 3584, 16, 4), (5, 72, 128, 4, 3), (13, 200, 512, 33, 2), (40, 328, 1024, 64, 40),
    (64, 1000, 256, 12, 7), (70, 136, 320, 16, 3), (150, 264, 128, 8, 5),
])
def test_adapters(lc, N, o, d, k, n, dtype):
    codes, scales, z, W = _weight(o, d, 64, torch.bfloat16, True)
    _check(lc, _tokens(N, d), lc.Q4Weight(codes, scales, zeros=z), W, _adapters(lc, N, d, o, k, n, dtype))


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("N,o,d,group,k,n", [
    (17, 136, 256, 128, 4, 2), (32, 64, 65536, 64, 0, 0), (33, 128, 128, 32, 8, 1), (100, 264, 2048, 128, 8, 3),
    (128, 2000, 1152, 128, 0, 0), (129, 8, 512, 128, 33, 5), (300, 392, 640, 128, 16, 4), (257, 1000, 256, 64, 0, 0),
])
def test_many_tokens(lc, N, o, d, group, k, n, zeros):
    """Every width of the tokens' tiles and of the clusters on the same rows, several tiles of tokens, ragged ones."""
    codes, scales, z, W = _weight(o, d, group, torch.bfloat16 if zeros else torch.float32, zeros)
    ad = _adapters(lc, N, d, o, k, n, torch.bfloat16) if n else None
    _check(lc, _tokens(N, d), lc.Q4Weight(codes, scales, zeros=z), W, ad)


@pytest.mark.parametrize("ids", [-1, 0])
def test_all_tokens_without_or_with_one_adapter(lc, ids):
    codes, scales, z, W = _weight(264, 512, 128, torch.float32, False)
    ad = list(_adapters(lc, 20, 512, 264, 16, 2, torch.float32))
    ad[3] = torch.full_like(ad[3], ids)
    X, weight = _tokens(20, 512), lc.Q4Weight(codes, scales)
    Y = _check(lc, X, weight, W, ad)
    if ids < 0:
        assert torch.equal(Y, _check(lc, X, weight, W))


def test_each_code_and_zero(lc):
    """One column at a time through a unit token: every code against every zero comes out exactly."""
    d, o = 64, 16
    codes = (torch.arange(16, device="cuda", dtype=torch.int32)[:, None] * 17).expand(16, d // 2).to(torch.uint8).contiguous()
    X = torch.eye(d, device="cuda").to(torch.bfloat16)
    for z in range(16):
        zeros = torch.full((o, 2), z, dtype=torch.uint8, device="cuda")
        scales = torch.tensor([0.5, 2.0], device="cuda").repeat(o, 1).contiguous()
        Y = torch.empty((d, o), dtype=torch.bfloat16, device="cuda")
        lc.loca_q4_apply(X, lc.Q4Weight(codes, scales, zeros=zeros), Y)
        want = (torch.arange(16, device="cuda") - z).float()[None, :] * torch.tensor([0.5, 2.0], device="cuda").repeat_interleave(32)[:, None]
        assert torch.equal(Y.float(), want), z


def test_columns_in_their_places(lc):
    """Codes that name their own column and row: nothing is exchanged by the packed order."""
    o, d = 37, 224
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    q = torch.randint(0, 16, (o, d), generator=g, device="cuda", dtype=torch.int32)
    codes = (q[:, 0::2] | q[:, 1::2] << 4).to(torch.uint8).contiguous()
    scales = torch.ones((o, d // 32), device="cuda")
    X = torch.eye(d, device="cuda").to(torch.bfloat16)
    Y = torch.empty((d, o), dtype=torch.bfloat16, device="cuda")
    lc.loca_q4_apply(X, lc.Q4Weight(codes, scales), Y)
    assert torch.equal(Y.float().T, (q - 8).float())


@pytest.mark.parametrize("N", [3, 70])
def test_tokens_apart_stay_apart(lc, N):
    codes, scales, z, W = _weight(136, 256, 64, torch.bfloat16, True)
    weight, X = lc.Q4Weight(codes, scales, zeros=z), _tokens(N, 256)
    clean = _check(lc, X, weight, W)
    X2 = X.clone()
    X2[1], X2[2, 7] = float("nan"), float("inf")
    Y = torch.empty_like(clean)
    lc.loca_q4_apply(X2, weight, Y)
    keep = [i for i in range(N) if i not in (1, 2)]
    assert torch.equal(Y[keep], clean[keep]) and bool(Y[1].isnan().all()) and not bool(Y[2].isfinite().any() and (Y[2].isfinite() & (W[:, 7] != 0)).any())


def test_an_adapter_that_is_not_finite(lc):
    """It spoils its own tokens' outputs, all of them, and nobody else's."""
    N, o, d = 12, 136, 256
    codes, scales, z, W = _weight(o, d, 64, torch.bfloat16, True)
    weight, X = lc.Q4Weight(codes, scales, zeros=z), _tokens(N, d)
    A, B, scale, _ = _adapters(lc, N, d, o, 8, 3, torch.float32)
    ids = (torch.arange(N, device="cuda") % 4 - 1).to(torch.int32)
    clean = _check(lc, X, weight, W, (A, B, scale, ids))
    A[1, 5, 2] = float("inf")
    Y = torch.empty_like(clean)
    lc.loca_q4_apply(X, weight, Y, adapters=lc.AdapterSet(3, d, o, 8).pack(A, B, scale), plan=lc.AdapterPlan(ids, 3))
    mine = ids == 1
    assert bool(Y[mine].isnan().all()) and torch.equal(Y[~mine], clean[~mine])


@pytest.mark.parametrize("N", [2, 40])
def test_spaced_rows(lc, N):
    o, d = 131, 192
    codes, scales, z, W = _weight(o, d, 64, torch.float32, True)
    weight, X = lc.Q4Weight(codes, scales, zeros=z), _tokens(N, d)
    want = _check(lc, X, weight, W)
    xs = torch.full((N, d + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    xs[:, 8:8 + d] = X
    ys = torch.full((N, o + 10), 7.0, dtype=torch.bfloat16, device="cuda")
    lc.loca_q4_apply(xs[:, 8:8 + d], weight, ys[:, 3:3 + o])
    assert torch.equal(ys[:, 3:3 + o], want) and bool((ys[:, :3] == 7).all()) and bool((ys[:, 3 + o:] == 7).all())


def test_the_source_arrays_are_not_needed(lc):
    codes, scales, z, W = _weight(200, 256, 32, torch.bfloat16, True)
    weight, X = lc.Q4Weight(codes, scales, zeros=z), _tokens(10, 256)
    first = _check(lc, X, weight, W)
    codes.zero_()
    scales.zero_()
    z.zero_()
    assert torch.equal(first, _check(lc, X, weight, W))


def test_no_tokens(lc):
    codes, scales, z, _ = _weight(40, 64, 32, torch.bfloat16, False)
    Y = torch.empty((0, 40), dtype=torch.bfloat16, device="cuda")
    lc.loca_q4_apply(_tokens(0, 64), lc.Q4Weight(codes, scales), Y)


def test_python_refusals(lc):
    codes, scales, z, _ = _weight(40, 64, 32, torch.bfloat16, True)
    weight, X = lc.Q4Weight(codes, scales, zeros=z), _tokens(4, 64)
    Y = torch.empty((4, 40), dtype=torch.bfloat16, device="cuda")
    for bad in ((codes.int(), scales, z), (codes, scales.half(), z), (codes, scales, z.int()), (codes[:, ::2], scales, z)):
        with pytest.raises((TypeError, ValueError)):
            lc.Q4Weight(bad[0], bad[1], zeros=bad[2])
    with pytest.raises(ValueError):
        lc.Q4Weight(codes, scales[:20].contiguous())
    with pytest.raises(ValueError):
        lc.Q4Weight(codes, scales, zeros=z[:, :1].contiguous())
    with pytest.raises(lc.LocaError, match="group"):
        lc.Q4Weight(codes, scales.repeat(1, 2).contiguous())  # groups of 16
    with pytest.raises(ValueError):
        lc.loca_q4_apply(X[:, :32].contiguous(), weight, Y)
    with pytest.raises(ValueError):
        lc.loca_q4_apply(X, weight, Y[:, :32])
    with pytest.raises(ValueError, match="together"):
        lc.loca_q4_apply(X, weight, Y, adapters=lc.AdapterSet(1, 64, 40, 4))
    with pytest.raises(ValueError, match="plan"):
        ids = torch.zeros((5,), dtype=torch.int32, device="cuda")
        lc.loca_q4_apply(X, weight, Y, adapters=lc.AdapterSet(1, 64, 40, 4), plan=lc.AdapterPlan(ids, 1))
    sq = lc.Q4Weight(*_weight(64, 64, 32, torch.bfloat16, False)[:2])
    with pytest.raises(lc.LocaError, match="overlap"):
        lc.loca_q4_apply(X, sq, X)
