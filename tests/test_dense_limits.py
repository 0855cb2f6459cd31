"""Limits of the dense operators' C entries, on the host: no call here launches
anything."""
import pytest

from paper_2412_00119_amd import bmlp as B

P = 1 << 20   # an aligned address that no call uses


def loss(tau, n=4):
    return B.lib().bmlp_distill(1, n, 100, P, 100, 5, P, P, 1, None, None, tau, P, P, 100, None)


@pytest.mark.parametrize("tau", [1e-45, 1e-42, 1e-39, 4.2e-39])
def test_temperatures_without_a_finite_reciprocal(tau):
    """exp((z - max) / tau) would be exp(0 * inf): refused, and not answered with NaN."""
    assert loss(tau) == B.BMLP_EINVAL
    assert loss(tau, n=0) == B.BMLP_EINVAL


@pytest.mark.parametrize("tau", [4.3e-39, 1e-38, 1.0, 3e38])
def test_temperatures_with_one(tau):
    assert loss(tau, n=0) == B.BMLP_OK
