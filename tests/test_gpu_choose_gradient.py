"""The gradient of a router's weights, entry by entry against roundings that are counted for each."""
import numpy as np
import pytest
import torch

import paper_2607_18002_b200 as moe
from tests import scaled_util as su

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -24
EXP, QUOTIENT = 4, 4                  # half steps of fp32: exp and a quotient by approximation are off by two steps at most
SIGMOID = EXP + 1 + QUOTIENT          # 1 / (1 + exp(-z))


def _bound(z, ids, d, kind, renormalize, scale):
    """fp64 [T, E]: what fp32 may lose of every entry of the gradient, all experts' ids in range."""
    T, E = z.shape
    k = ids.shape[1]
    g = np.abs(scale * d)                                            # rounded once
    zc = np.take_along_axis(z, ids, 1)
    out = np.zeros((T, E))
    rows = np.arange(T)[:, None]
    if renormalize:
        n = su.weights_of(z, ids, kind, True, 1.0)
        # a score relative to the largest: exp of a rounded argument, for sigmoid over 1 + exp(-|z|)
        x = np.abs(zc - zc.max(1, keepdims=True)) if kind == "softmax" else np.abs(np.minimum(zc, 0) - np.minimum(zc.max(1, keepdims=True), 0))
        own = EXP + x + (0 if kind == "softmax" else EXP + 1 + QUOTIENT)
        share = own + (n * own).sum(1, keepdims=True) + 5 + QUOTIENT        # over the sum of the chosen, added in five steps
        mean = (n * g).sum(1, keepdims=True)
        mean_loss = (n * g * (share + 2)).sum(1, keepdims=True) + 5 * mean
        v = n * (g + mean)
        loss = v * (share + 3) + n * mean_loss
        if kind == "sigmoid":
            s = su.scores_of(-zc.reshape(T, k), "sigmoid")
            v, loss = v * s, (loss + v * (SIGMOID + 1)) * s
    elif kind == "sigmoid":
        s = su.scores_of(zc, kind) * su.scores_of(-zc, kind)
        v = s * g
        loss = v * (2 * SIGMOID + 3)
    else:
        v, loss = g, g
    np.add.at(out, (rows, ids), loss + (k if k > 1 else 0) * v)      # slots of one expert are added up
    if kind == "softmax" and not renormalize:
        s = su.scores_of(z, kind)
        x = np.abs(z - z.max(1, keepdims=True))
        # the sum: 14 additions at most for a term, each off by its exp (approximate: two steps and 1.3 |x|)
        total = 14 + (s * (4 + 2.6 * x)).sum(1, keepdims=True) + 1
        share = EXP + x + total + 1
        pc, pl = np.take_along_axis(s, ids, 1), np.take_along_axis(share, ids, 1)
        mean = (pc * g).sum(1, keepdims=True)
        mean_loss = (pc * g * (pl + 2)).sum(1, keepdims=True) + 5 * mean
        size = np.zeros((T, E))
        np.add.at(size, (rows, ids), g)
        out = s * (out + mean_loss + (size + mean) * (share + 2))
    return out * HALF


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("T,E,k,sigma", [(300, 40, 5, 1.5), (64, 257, 32, 3.0), (9, 1024, 6, 1.5), (500, 64, 6, 8.0), (3, 1, 1, 1.0), (100, 384, 8, 1.5)])
def test_every_entry_to_its_own_roundings(kind, renormalize, T, E, k, sigma):
    rng = np.random.default_rng([T, E])
    z = torch.from_numpy((sigma * rng.standard_normal((T, E))).astype(np.float32)).cuda()
    d = rng.standard_normal((T, k)).astype(np.float32)
    z64 = su.to_numpy(z)
    for ids in (np.argsort(rng.random((T, E)), 1)[:, :k], np.argsort(-z64, 1)[:, :k], rng.integers(0, E, (T, k))):        # any, the best, some twice
        dz = moe.choose_experts_grad(z, torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(d).cuda(), scores=kind, renormalize=renormalize, scale=2.5)
        ref = su.weights_gradient(z64, ids, d.astype(np.float64), kind, renormalize, 2.5)
        bound = _bound(z64, ids, d.astype(np.float64), kind, renormalize, 2.5) + 2.0 ** -120
        err = np.abs(su.to_numpy(dz) - ref)
        assert np.all(err <= bound), (err / bound).max()
