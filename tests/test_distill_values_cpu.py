"""Temperatures that the loss's factors T^2 and 1 / T do not hold are refused, on the host."""

import os

import pytest

from paper_2301_09830_amd import build as buildmod
from paper_2301_09830_amd import optcc
from test_experts_abi_cpu import SHAPE, VALUE, distill


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(buildmod.LIB):
        buildmod.build()
    return optcc.lib()


@pytest.mark.parametrize("T", [1e-45, 1e-39, 1.1e-38, 1e-30, 2.0 ** -63 * 0.99, 2.0 ** 64, 1e38,
                               float("inf"), float("nan"), 0.0, -0.0, -2.0, -1e-30])
def test_temperatures_out_of_range(L, T):
    for fn in (L.occ_distill_fwd, L.occ_distill_bwd):
        assert fn(distill(temperature=T), None) == VALUE


@pytest.mark.parametrize("T", [2.0 ** -63, 1e-3, 1.0, 1e4, 2.0 ** 63])
def test_temperatures_in_range(L, T):
    """A refusal that comes after the temperature's."""
    for fn in (L.occ_distill_fwd, L.occ_distill_bwd):
        assert fn(distill(temperature=T, lds=99), None) == SHAPE
