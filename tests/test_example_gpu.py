"""The example that fits, serves and polishes adapters: the loss falls at each stage, and the last
forward pass equals the definition in 64 bits."""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_adapt_and_serve():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_03020_gb300 import _build

    _build.build()
    spec = importlib.util.spec_from_file_location("adapt_and_serve", os.path.join(ROOT, "examples", "adapt_and_serve.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.run(verbose=False)
    frozen, fitted, polished = (value for _, value in got["told"])
    assert fitted < frozen and polished < fitted
    X, A, B = got["X"].double(), got["A"].double(), got["B"].double()
    H = X @ got["W"].double().T
    for a in range(A.shape[0]):
        rows = got["ids"] == a
        H[rows] += (X[rows] @ A[a]) @ B[a].T
    live = got["y"] >= 0
    want = torch.nn.functional.cross_entropy(H[live] @ got["head"].double().T, got["y"][live].long(), reduction="none")
    # H is rounded to bf16 on the way: 2^-8 of its size moves a loss of order one by about that
    assert abs(float(got["loss"][live].double().mean()) - float(want.mean())) <= 2.0 ** -8 * float(want.mean())
