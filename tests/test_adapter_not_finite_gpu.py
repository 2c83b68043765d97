"""An adapter with a value that is not finite: NaN in every output of its own tokens and in its own
gradients, in each way the low-rank term is computed, and nothing of it elsewhere."""

import pytest
import test_adapter_gpu as adapter
import torch

pytestmark = pytest.mark.gpu
lc = adapter.lc  # the fixture


# token by token, one tile by slots, few tokens in several tiles, many tokens
@pytest.mark.parametrize("N,d,o,k,n,ids", [(40, 200, 136, 16, 64, "mixed"), (100, 200, 136, 8, 3, "mixed"),
                                           (300, 72, 136, 8, 3, "mixed"), (1500, 264, 520, 12, 4, "runs")])
@pytest.mark.parametrize("where", ["A", "B", "scale", "scale times B"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_it_spoils_all_of_its_own_and_nothing_else(lc, N, d, o, k, n, ids, where, dtype):
    v = adapter._inputs(N, d, o, k, n, ids, dtype)
    used = int(v["ids"][(v["ids"] >= 0) & (v["ids"] < n)][0])
    ref, low = adapter._reference(v)
    if where == "A":
        v["A"][used, d - 1, k - 1] = float("nan")
    elif where == "B":
        v["B"][used, 3, 0] = float("-inf")
    elif where == "scale":
        v["scale"][used] = float("inf")
    else:  # both finite, not their product
        v["B"][used, o - 1, k - 1] = 3e38
        v["scale"][used] = 100.0
    got = adapter._run(lc, v)
    mine = v["ids"] == used
    for key in ("Y", "dX"):
        assert torch.isnan(got[key][mine].float()).all(), key
        adapter._check({key: got[key][~mine]}, {key: ref[key][~mine]}, {key: low[key][~mine]})
    rest = [a for a in range(n) if a != used]
    for key in ("dA", "dB"):
        assert torch.isnan(got[key][used].float()).all(), key
        adapter._check({key: got[key][rest]}, {key: ref[key][rest]}, {})


@pytest.mark.parametrize("N,n", [(40, 64), (700, 3)])
def test_repacked_with_finite_values_it_is_right_again(lc, N, n):
    v = adapter._inputs(N, 136, 264, 8, n, "mixed")
    ref, low = adapter._reference(v)
    ad = lc.AdapterSet(n, 136, 264, 8)
    plan = lc.AdapterPlan(v["ids"], n)
    bad = v["A"].clone()
    bad[:, 0, 0] = float("inf")
    ad.pack(bad, v["B"], v["scale"])
    ad.pack(v["A"], v["B"], v["scale"])
    Y = torch.empty((N, 264), dtype=torch.bfloat16, device="cuda")
    lc.loca_adapter_apply(v["X"], v["W"], ad, plan, Y)
    torch.cuda.synchronize()
    adapter._check({"Y": Y}, {"Y": ref["Y"]}, {"Y": low["Y"]})
