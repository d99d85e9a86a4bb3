"""Calls on rows at the edges of what the documentation allows: alignment, batches without rows, shapes."""
import pytest
import torch

import paper_2607_18002_b200 as moe
from paper_2607_18002_b200 import build as moe_build


@pytest.fixture(scope="module")
def lib():
    moe_build.build()
    return moe.lib()


P = 1 << 20          # stands for an aligned device address: a call that is refused does not look at it


@pytest.mark.parametrize("at", [0, 1, 2, 6])
@pytest.mark.parametrize("off", [1, 2])
def test_the_routers_gradient_refuses_addresses_between_elements(lib, at, off):
    args = [P, P, P, 4, 8, 2, P, None]
    args[at] += off
    assert lib.moe_route_grad(*args) == moe.MOE_EINVAL
