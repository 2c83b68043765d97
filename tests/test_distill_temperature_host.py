"""Temperatures at the lower end: the exponentials of the logits are taken to the base 2, with a factor of
log2(e) / tau, which has to be finite as 1 / tau has (no GPU needed: the calls fail, or have no position)."""

import ctypes

import pytest

P = ctypes.c_void_p
F = ctypes.c_float


@pytest.fixture(scope="module")
def L():
    from paper_2608_03020_gb300 import _build
    from paper_2608_03020_gb300 import loca

    _build.build()
    return loca.lib()


def _calls(L, tau, N):
    at = [P((i + 1) << 24) for i in range(8)]  # never dereferenced
    return (L.loca_head_distill(at[0], 64, N, 64, at[1], 10, at[2], at[3], 3, F(tau), None, at[4], at[5], at[6], 1 << 40, None),
            L.loca_head_distill_backward(at[0], 64, N, 64, at[1], 10, at[2], at[3], 3, F(tau), None, at[4], None, F(1.0),
                                         at[5], 64, None, at[6], 1 << 40, None))


# 1 / 3e-39 = 3.3e38 is finite in fp32, 1.44 times as much is not
@pytest.mark.parametrize("tau", [3e-39, 3.5e-39, 4.2e-39])
def test_factors_that_are_not_finite(L, tau):
    for N in (4, 0):
        assert _calls(L, tau, N) == (1, 1)


@pytest.mark.parametrize("tau", [4.3e-39, 1e-38, 1e-20, 1.0, 1e19])
def test_factors_that_are(L, tau):
    assert _calls(L, tau, 0) == (0, 0)
