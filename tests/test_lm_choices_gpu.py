"""Head loss, adapters and clipping where a size decides how they are computed.

The references and tolerances are those of the operators' own tests (derived there): the choices below
change the order of sums, not what a sum is or how it is rounded.
"""

import math

import pytest
import test_adapter_gpu as adapter
import test_grad_clip_gpu as clip
import test_head_loss_gpu as head
import torch

pytestmark = pytest.mark.gpu
lc = head.lc  # the fixture


# rows in several tiles of which a few, one or none hold a live row: the k ranges of dH are the device's
# choice, within one piece and across pieces of rows and of the vocabulary
@pytest.mark.parametrize("N,d,V,live,dw", [
    (2600, 328, 5003, 0.05, True), (2600, 72, 20001, 0.4, False), (1300, 1024, 3001, 0.0, True),
    (9000, 72, 70001, 0.03, False), (4100, 136, 1100, 0.9, False),
])
def test_few_live_rows(lc, N, d, V, live, dw):
    H, W, y, w, gl = head._inputs(N, d, V)
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    y[torch.rand((N,), generator=g, device="cuda") >= live] = -1
    keep = y >= 0
    ref = head._reference(H[keep], W, y[keep], w[keep], gl[keep], None, 0.5)
    full = {k: torch.zeros((N,) + tuple(ref[k].shape[1:]), dtype=torch.float64, device="cuda") for k in ("loss", "lse", "dH")}
    for k in full:
        full[k][keep] = ref[k]
    full.update(dW=ref["dW"], zmax=ref["zmax"])
    out = head._run(lc, H, W, y, w, gl, None, 0.5, dw=dw)
    head._check(out, full, w)
    assert torch.all(out["dH"][~keep] == 0)
    again = head._run(lc, H, W, y, w, gl, None, 0.5, dw=dw)
    assert all(torch.equal(out[k], again[k]) for k in out)


# up to 128 tokens: the vocabulary decides the tiles' width
@pytest.mark.parametrize("N", [1, 9, 128])
@pytest.mark.parametrize("V", [63, 65, 1000, 9731, 19457, 40001])
def test_few_tokens_and_any_vocabulary(lc, N, V):
    H, W, y, w, gl = head._inputs(N, 136, V)
    cols = torch.unique(torch.tensor([V - 1, 0, V // 2], device="cuda")).to(torch.int32)
    ref = head._reference(H, W, y, w, gl, cols, 1.0)
    head._check(head._run(lc, H, W, y, w, gl, cols, 1.0), ref, w)


# single tokens: rows of s B beforehand for all, some and few of a CTA's tokens; batches in one tile of
# tokens and in several, the k axis in one range and in up to eight; the last sizes of either way
@pytest.mark.parametrize("N,d,o,k,n,ids", [
    (20, 64, 136, 64, 40, "mixed"), (300, 64, 264, 32, 300, "mixed"), (40, 200, 136, 48, 64, "mixed"),
    (512, 72, 200, 16, 512, "mixed"), (513, 72, 200, 16, 513, "mixed"), (64, 3584, 1032, 16, 64, "mixed"),
    (200, 4104, 520, 16, 2, "runs"), (512, 1032, 1320, 12, 3, "runs"), (256, 2048, 2056, 24, 6, "runs"),
    (1000, 520, 264, 32, 40, "runs"), (130, 72, 4104, 8, 1, "last"), (16, 5120, 128, 64, 1, "last"),
])
def test_few_tokens_of_adapters(lc, N, d, o, k, n, ids):
    v = adapter._inputs(N, d, o, k, n, ids)
    ref, low = adapter._reference(v)
    got = adapter._run(lc, v)
    adapter._check(got, ref, low)
    again = adapter._run(lc, v)
    assert all(torch.equal(got[key], again[key]) for key in got)


# gradients joined from one range and from many
@pytest.mark.parametrize("N,d,o,k,n", [(199, 1160, 592, 64, 7), (9000, 72, 136, 4, 1), (9000, 136, 72, 33, 2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ranges_of_adapter_gradients(lc, N, d, o, k, n, dtype):
    v = adapter._inputs(N, d, o, k, n, "runs", dtype)
    ref, low = adapter._reference(v)
    adapter._check(adapter._run(lc, v), ref, low)


# an output any number of elements off its input's 16-byte boundary, over several chunks and in less than
# a vector
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [3, 9, 17, 8193, 20001])
def test_clipped_off_the_boundary(lc, dtype, size):
    per = 16 // torch.empty((), dtype=dtype).element_size()
    pairs = [(i, j) for i in range(per) for j in range(per)]
    pitch = (size + 63) // 32 * 32
    base = clip._tensors([pitch * len(pairs)], [dtype])[0]
    into = torch.full_like(base, 5.0)
    grads = [base[pitch * p + i:pitch * p + i + size] for p, (i, _) in enumerate(pairs)]
    out = [into[pitch * p + j:pitch * p + j + size] for p, (_, j) in enumerate(pairs)]
    clip._check(lc, grads, 0.25, out=out)
    touched = torch.zeros((base.numel(),), dtype=torch.bool, device="cuda")
    for p, (_, j) in enumerate(pairs):
        touched[pitch * p + j:pitch * p + j + size] = True
    assert torch.all(into[~touched] == 5.0)


# the norm over fp32's range, and factors on both sides of one
@pytest.mark.parametrize("power", [-36, -20, -1, 0, 1, 17, 35])
@pytest.mark.parametrize("ratio", [1e-3, 0.4999, 0.9999, 1.0001, 50.0])
def test_norm_and_factor_over_the_range(lc, power, ratio):
    g = torch.full((1000,), 1.5, device="cuda")
    g[::3] = 0.7
    grads = [g * 10.0 ** power]
    norm = math.sqrt(math.fsum(float(x) ** 2 for x in grads[0].double().tolist()))
    clip._check(lc, grads, ratio * norm, out=[torch.empty_like(grads[0])])
