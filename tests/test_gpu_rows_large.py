"""Rows sorted and merged where there are enough of them for the forms with several accesses a thread, by every width of access, against evaluations in 64 bits.

From 148 * 2048 * 4 accesses on a thread makes several: cases are chosen past that line for the widest access that their addresses, strides and lengths allow
(bf16 and fp16: 2 048 columns 16 bytes, 1 004 eight, 1 002 four, 1 003 two; fp32: 2 048 and 1 004, 1 002, 1 003 columns 16, 8 and 4).  More than 592 tokens give the
gradient of merge its columns in two goes.

Tolerances count roundings: one of the output type (half_step), k of fp32 in a sum of k terms; a dot product is a chain of at most max(32, H/256 + 8) multiply-adds in
a thread (a group of 32 to 256 threads shares a token's columns, each with at most four accesses of eight elements while the group can still grow, and an even
share of them in a group of 256), 5 additions over lanes and 8 over warps."""
import numpy as np
import pytest
import torch

import paper_2607_18002_b200 as moe

from rows_util import EPS_FP32, gpu, half_step, routing, tiny

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


def _rows(n, H, dtype, seed, pad=0, shift=0):
    """N(0, 1) rows as a view of a buffer with rows `pad` elements further apart, the first one `shift` elements in."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((n * (H + pad) + shift,), 7.0, dtype=dtype, device="cuda")
    v = torch.as_strided(buf, (n, H), (H + pad, 1), shift)
    v.copy_(torch.randn(n, H, generator=g, device="cuda"))
    return v


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("T,k,H,pad,shift,rejected", [
    (1500, 2, 1003, 0, 0, 0), (1500, 5, 1003, 0, 0, 40), (2500, 3, 1002, 0, 0, 0), (2500, 1, 1002, 0, 0, 0), (5000, 2, 1004, 0, 0, 0), (5000, 1, 2048, 0, 0, 0),
    (5000, 2, 2048, 0, 0, 300), (5000, 3, 2048, 0, 0, 0), (5000, 6, 2048, 0, 0, 0), (5000, 2, 2048, 8, 0, 0), (5000, 2, 2048, 4, 4, 0), (5000, 2, 2048, 3, 1, 9),
    (700, 2, 1024, 0, 0, 0), (700, 1, 256, 0, 0, 0), (700, 2, 1023, 0, 0, 0), (700, 9, 520, 0, 0, 77), (600, 2, 8200, 0, 0, 0), (593, 4, 8201, 0, 0, 0)])
def test_many_rows_against_64_bits(T, k, H, pad, shift, rejected, dtype):
    ids, w, offsets, s2f, f2s = routing(T, 16, k, 31, rejected)
    ds2f, df2s, dw_ = gpu(s2f, f2s, w)
    x, rows, dy = (_rows(n, H, dtype, seed, pad, shift) for n, seed in ((T, 1), (T * k, 2), (T, 3)))
    eps, small = half_step(dtype), tiny(dtype)
    owned, has = ds2f >= 0, df2s >= 0                                  # rows of a token, slots with a row
    token, at = torch.where(owned, ds2f, 0).long() // k, torch.where(has, df2s, 0).long()

    xs = moe.sort_rows(x, ds2f, df2s, k)
    assert torch.equal(xs, torch.where(owned[:, None], x[token], 0))

    picked = torch.where(has[:, None], rows[at].double(), 0.0).view(T, k, H)
    terms = picked * dw_.double()[..., None]
    for got, t in ((moe.sort_rows_grad(rows, df2s, k), picked), (moe.merge_rows(rows, df2s, dw_), terms)):
        ref, mag = t.sum(1), t.abs().sum(1)
        assert ((got.double() - ref).abs() <= eps * ref.abs() + (1 + eps) * k * EPS_FP32 * mag + small).all()
    del terms

    drows, dw = moe.merge_rows_grad(dy, rows, ds2f, df2s, dw_)
    wrow = torch.where(owned, dw_.view(-1)[torch.where(owned, ds2f, 0).long()], 0.0).double()
    ref = dy[token].double() * wrow[:, None]
    assert ((drows.double() - ref).abs() <= (eps + 2 * EPS_FP32) * ref.abs() + small).all()
    prods = picked * dy.double()[:, None]
    ref, mag = prods.sum(-1), prods.abs().sum(-1)
    assert ((dw.double() - ref).abs() <= (max(32, H / 256 + 8) + 14) * EPS_FP32 * mag).all()
    assert (dw[~has.view(T, k)] == 0).all()
    again = moe.merge_rows_grad(dy, rows, ds2f, df2s, dw_)
    assert torch.equal(again[0], drows) and torch.equal(again[1], dw)


@pytest.mark.parametrize("T,H", [(1500, 1003), (2500, 1002), (5000, 1004), (2500, 4104), (5000, 4112)])
def test_many_codes_of_one_byte_are_sorted(T, H):
    k = 3
    ids, w, offsets, s2f, f2s = routing(T, 16, k, 33, 5)
    ds2f, df2s = gpu(s2f, f2s)
    x = torch.from_numpy(np.random.default_rng(T).integers(0, 256, (T, H), np.uint8)).cuda()
    want = torch.where((ds2f >= 0)[:, None], x[torch.where(ds2f >= 0, ds2f, 0).long() // k], 0)
    assert torch.equal(moe.sort_rows(x, ds2f, df2s, k), want)
