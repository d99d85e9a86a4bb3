"""The 4-bit products beyond one turn of their rings and one tile a block, in both heights of tiles.

A stage holds 256 columns and a block has three or four of them, so rings turn over beyond 1 024 columns.  Low tiles (96 rows) are walked by 148 blocks, high
ones (192 rows, more than 256 rows an expert) by 148 blocks or, for gate/up, by 74 pairs: every launch here has more than two tiles for each of them where it
says so.  Operands are small multiples of common powers of two, so fp32 sums are exact in any order (up to 4 096 terms of at most 2^11.2 steps)."""
import numpy as np
import pytest
import torch

import paper_2607_18002_b200 as moe

from rows_util import gpu, values_of
from test_gpu_mx import _bf16, _check_swiglu, _exact_operand, _offsets, _product64

pytestmark = pytest.mark.gpu

LOW = [200, 250, 1, 0, 480, 95, 97, 700]
HIGH = [2600, 300, 0, 1500]


def _is_high(counts):
    return sum(counts) > 256 * len(counts)


def _tiles(counts, cols, step):
    rows = 192 if _is_high(counts) else 96
    return sum(-(-c // rows) for c in counts) * -(-cols // step)


def _reference(x, w, off, R):
    """fp64 products on the GPU."""
    xv, out = torch.from_numpy(values_of(*x)).cuda(), torch.zeros(R, w[0].shape[1], dtype=torch.float64, device="cuda")
    for e in range(w[0].shape[0]):
        if off[e + 1] > off[e]:
            out[off[e]:off[e + 1]] = xv[off[e]:off[e + 1]] @ torch.from_numpy(values_of(w[0][e], w[1][e])).cuda().T
    return out.cpu().numpy()


def _gate_up(counts, I, K, seed):
    x, w = _exact_operand((sum(counts),), K, seed, 0), _exact_operand((len(counts), 2 * I), K, seed + 1, 1)
    x[1][:] = 120                                                    # gate values of a few units
    return x, w


@pytest.mark.parametrize("K", [2304, 2432, 4096])                   # 9 stages, 9 and a half (scales by words), 16
@pytest.mark.parametrize("counts", [LOW, HIGH], ids=["low tiles", "high tiles on pairs"])
def test_gate_up_over_turns_of_the_ring_and_many_tiles(counts, K):
    I, off = 1792, _offsets(counts)
    assert _is_high(counts) == (counts is HIGH)
    assert _tiles(counts, I, 256 if _is_high(counts) else 128) > 2 * (74 if _is_high(counts) else 148)
    x, w = _gate_up(counts, I, K, 51)
    h = _reference(x, w, off, sum(counts))
    args = gpu(*x, *w, off)
    first = moe.mx_swiglu(*args)
    _check_swiglu(first, h[:, :I], h[:, I:])
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(moe.mx_swiglu(*args), first))


@pytest.mark.parametrize("N,K", [(4096, 2304), (4101, 2432), (4096, 4096)])
@pytest.mark.parametrize("counts", [LOW, HIGH], ids=["low tiles", "high tiles"])
def test_product_over_turns_of_the_ring_and_many_tiles(counts, N, K):
    off = _offsets(counts)
    assert _tiles(counts, N, 256) > 2 * 148
    x, w = _exact_operand((sum(counts),), K, 53), _exact_operand((len(counts), N), K, 54)
    assert torch.equal(moe.mx_product(*gpu(*x, *w, off)).cpu(), _bf16(_reference(x, w, off, sum(counts))))


@pytest.mark.parametrize("I", [96, 640])
@pytest.mark.parametrize("K", [256, 2304])
def test_nan_blocks_in_high_tiles(I, K):
    """A row, a gate column and an up column that are NaN: their blocks of the result, and nothing else; the same of the plain product."""
    counts = [620, 30]
    assert _is_high(counts)
    x, w = _exact_operand((650,), K, 7), _exact_operand((2, 2 * I), K, 8)
    x[1][4, 3] = x[1][200, K // 32 - 1] = 255
    w[1][1, 40, 0] = w[1][1, I + 95, 1] = 255
    args = gpu(*x, *w, _offsets(counts))
    scales = moe.mx_swiglu(*args)[1].cpu().numpy()
    want = np.zeros(scales.shape, bool)
    want[[4, 200]] = True
    want[620:, [1, 2]] = True
    assert np.array_equal(scales == 255, want)
    bad = torch.isnan(moe.mx_product(*args)).cpu().numpy()
    want = np.zeros(bad.shape, bool)
    want[[4, 200]] = True
    want[620:, [40, I + 95]] = True
    assert np.array_equal(bad, want)


@pytest.mark.parametrize("lead", [0, 5])
def test_rows_of_no_expert_are_zero_beside_high_tiles(lead):
    counts, K, I = [900, 0, 500], 512, 160
    R = lead + 1400 + 17
    assert R > 256 * 3
    x, w = _gate_up([R], I, K, 61)[0], _gate_up(counts, I, K, 61)[1]
    off = _offsets(counts, lead)
    h = _product64(values_of(*x), values_of(*w), off, R)
    args = gpu(*x, *w, off)
    got = moe.mx_product(*args).cpu()
    assert torch.equal(got, _bf16(h)) and (got[:lead] == 0).all() and (got[lead + 1400:] == 0).all()
    codes, scales = moe.mx_swiglu(*args)
    for t in (codes, scales):
        assert (t[:lead] == 0).all() and (t[lead + 1400:] == 0).all()
    on = slice(lead, lead + 1400)
    _check_swiglu((codes[on], scales[on]), h[on, :I], h[on, I:])


def test_rows_of_high_tiles_do_not_depend_on_their_neighbours():
    """A row's outputs are the same bits beside other rows, at another place of its segment and in every run (sums that round: scales over 13 powers of two)."""
    K, N = 2304, 640
    w = gpu(*_exact_operand((3, N), K, 13, 6))
    x, other = gpu(*_exact_operand((960,), K, 14, 6)), gpu(*_exact_operand((960,), K, 15, 6))
    off = gpu(_offsets([850, 0, 110]))
    assert _is_high([850, 0, 110])
    calls = {"product": lambda r: (moe.mx_product(*r, *w, off),), "gate/up": lambda r: moe.mx_swiglu(*r, *w, off)}
    moves = ((0, 849), (191, 192), (500, 3), (849, 95), (850, 959), (900, 850))
    mixed = tuple(t.clone() for t in other)
    for a, b in moves:
        for t, f in zip(mixed, x):
            t[b] = f[a]
    for call in calls.values():
        here, there = call(x), call(mixed)
        assert all(torch.equal(p, q) for p, q in zip(call(x), here))
        for a, b in moves:
            assert all(torch.equal(p[a], q[b]) for p, q in zip(here, there))


@pytest.mark.parametrize("shift", [4, 8])
@pytest.mark.parametrize("K", [768, 2432])
def test_scales_that_are_aligned_to_words_only_in_high_tiles(K, shift):
    counts, I = [700, 0, 300], 160
    assert _is_high(counts)
    x, w = _gate_up(counts, I, K, 71)
    off = _offsets(counts)

    def moved(t):
        buf = torch.full((t.numel() + shift,), 255, dtype=torch.uint8, device="cuda")
        buf[shift:] = t.reshape(-1)
        return buf[shift:].view(t.shape)

    dx, dxs, dw, dws, doff = gpu(*x, *w, off)
    h = _product64(values_of(*x), values_of(*w), off, sum(counts))
    assert torch.equal(moe.mx_product(dx, moved(dxs), dw, moved(dws), doff).cpu(), _bf16(h))
    _check_swiglu(moe.mx_swiglu(dx, moved(dxs), dw, moved(dws), doff), h[:, :I], h[:, I:])
