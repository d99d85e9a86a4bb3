"""Routers by scores: sums of many scores, of which most are next to nothing beside one another."""
import math

import pytest
import torch

import paper_2607_18002_b200 as moe

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E", [256, 512, 1024])
@pytest.mark.parametrize("stride", [4, 1])
def test_many_small_scores_beside_a_large_one(E, stride):
    """Thirty-two logits of 0, one for each lane of the warp that has the row (neighbours or every fourth, as rows are read one by one or by four), and all others just too small to
    change a sum of 1 by themselves: added to it one after the other they would all be lost, 31 half steps of 2^-23 at 1024 experts."""
    z = torch.full((3, E + 1), math.log(0.98 * 2.0 ** -24), device="cuda")
    z[:, 0:32 * stride:stride] = 0.0
    z = z[:, :E] if stride == 1 else z[:, :E].contiguous()                 # (rows of an odd stride are read one by one)
    p = torch.softmax(z.double(), 1)
    ids, w = moe.choose_experts(z, 8, scores="softmax", renormalize=False)
    assert torch.equal(ids.long().cpu(), (stride * torch.arange(8)).expand(3, 8))
    # half steps: a lane's additions in four parts and their joins, five across the warp; the reciprocal, the product; exp(0) is 1, and what exp loses of the others (their share of the
    # sum is 2^-18 at most) is less than one
    bound = (E // 32 // 4 - 1 + 2 + 5 + 2 + 1) * 2.0 ** -24
    want = p.gather(1, ids.long())
    assert ((w.double() - want).abs() <= bound * want).all(), ((w.double() - want).abs() / want).max().item() * 2 ** 24
    d = torch.zeros(3, 8, device="cuda")
    d[:, 0] = 1.0
    dz = moe.choose_experts_grad(z, ids, d, scores="softmax", renormalize=False).double()
    first = want[:, :1]
    # (a product of two such probabilities, 1 minus one of them, and three roundings)
    assert ((dz[:, stride:2 * stride:stride] + first * first).abs() <= (2 * bound + 3 * 2.0 ** -24) * first * first).all()
    assert ((dz[:, :1] - first * (1 - first)).abs() <= (2 * bound + 3 * 2.0 ** -24) * first).all()
