"""The C entry points with outputs wherever their documentation allows them to lie, between bytes that have to stay as they are."""
import math

import numpy as np
import pytest
import torch

import paper_2607_18002_b200 as moe

from rows_util import gpu, quantised, routing, scale_bytes, values_of
from test_gpu_mx import _bf16, _check_swiglu, _exact_operand, _offsets, _product64

pytestmark = pytest.mark.gpu


class Guarded:
    """A tensor `shift` bytes behind a 256-byte boundary, with 256 bytes or more of 0xA5 on either side."""

    def __init__(self, shape, dtype, shift):
        n = math.prod(shape) * dtype.itemsize
        self.buf = torch.full((n + shift + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        self.lo, self.hi = 256 + shift, 256 + shift + n
        self.t = self.buf[self.lo:self.hi].view(dtype).view(shape)

    def intact(self):
        return bool((self.buf[:self.lo] == 0xA5).all() and (self.buf[self.hi:] == 0xA5).all())


def _call(name, *args):
    rc = getattr(moe.lib(), name)(*(a.t.data_ptr() if isinstance(a, Guarded) else a.data_ptr() if isinstance(a, torch.Tensor) else a for a in args),
                                  torch.cuda.current_stream().cuda_stream)
    assert rc == moe.MOE_OK


@pytest.mark.parametrize("counts", [[40, 0, 3, 97], [900, 0, 3, 397]], ids=["low tiles", "high tiles"])
@pytest.mark.parametrize("shift", [0, 2, 8, 14])
@pytest.mark.parametrize("N", [264, 300, 129])
def test_products(counts, shift, N):
    R, E, K = sum(counts), len(counts), 384
    x, w = _exact_operand((R,), K, 81), _exact_operand((E, N), K, 82)
    off, out = _offsets(counts), Guarded((R, N), torch.bfloat16, shift)
    _call("moe_mx_product", *gpu(*x, *w, off), R, E, N, K, out)
    assert torch.equal(out.t.cpu(), _bf16(_product64(values_of(*x), values_of(*w), off, R))) and out.intact()


@pytest.mark.parametrize("counts", [[40, 0, 3, 97], [900, 0, 3, 397]], ids=["low tiles", "high tiles"])
@pytest.mark.parametrize("shift,scale_shift", [(0, 1), (4, 3), (8, 0), (12, 2)])
def test_gate_up(counts, shift, scale_shift):
    R, E, K, I = sum(counts), len(counts), 384, 160
    x, w = _exact_operand((R,), K, 83, 0), _exact_operand((E, 2 * I), K, 84, 1)
    x[1][:] = 120                                                    # gate values of a few units
    off, codes, scales = _offsets(counts), Guarded((R, I // 2), torch.uint8, shift), Guarded((R, I // 32), torch.uint8, scale_shift)
    _call("moe_mx_swiglu", *gpu(*x, *w, off), R, E, I, K, codes, scales)
    h = _product64(values_of(*x), values_of(*w), off, R)
    _check_swiglu((codes.t, scales.t), h[:, :I], h[:, I:])
    assert codes.intact() and scales.intact()


@pytest.mark.parametrize("shift", [0, 4, 8, 12])
@pytest.mark.parametrize("H", [64, 1003])
def test_rows(shift, H):
    """fp32 rows of whole numbers: sums and products are exact."""
    T, k = 37, 3
    ids, w, offsets, s2f, f2s = routing(T, 8, k, 7, 11)
    rng = np.random.default_rng(H)
    x, rows, dy = (rng.integers(-8, 9, (n, H)).astype(np.float32) for n in (T, T * k, T))
    w = rng.integers(-3, 4, (T, k)).astype(np.float32)
    ds2f, df2s, dx, drows, ddy, dw = gpu(s2f, f2s, x, rows, dy, w)
    own, has = s2f >= 0, (f2s >= 0).reshape(T, k)
    at = np.where(own, s2f, 0)
    picked = np.where(has[..., None], rows[np.where(f2s >= 0, f2s, 0)].reshape(T, k, H), 0)
    xs, sx, y, gr, gw = (Guarded(s, torch.float32, shift) for s in ((T * k, H), (T, H), (T, H), (T * k, H), (T, k)))
    f32 = moe.MOE_DTYPE_FP32
    _call("moe_sort_rows", dx, H, f32, T, k, H, ds2f, df2s, xs)
    _call("moe_sort_rows_grad", drows, H, f32, T, k, H, df2s, sx)
    _call("moe_merge_rows", drows, H, f32, dw, T, k, H, df2s, y)
    _call("moe_merge_rows_grad", ddy, H, drows, H, f32, dw, T, k, H, ds2f, df2s, gr, gw)
    for got, want in ((xs, np.where(own[:, None], x[at // k], 0)), (sx, picked.sum(1)), (y, (picked * w[..., None]).sum(1)),
                      (gr, np.where(own[:, None], dy[at // k] * w.reshape(-1)[at][:, None], 0)), (gw, (picked * dy[:, None]).sum(-1))):
        assert np.array_equal(got.t.cpu().numpy(), want) and got.intact()


@pytest.mark.parametrize("shift", [0, 4, 8, 12])
@pytest.mark.parametrize("E", [7, 40])
def test_router_gradient(shift, E):
    T, k = 19, 3
    ids = np.random.default_rng(E).integers(0, E, (T, k)).astype(np.int32)
    w, dw = np.tile(np.float32([0.5, 0.25, 0.25]), (T, 1)), np.random.default_rng(1).integers(-8, 9, (T, k)).astype(np.float32)      # exact
    dz = np.zeros((T, E), np.float32)
    np.add.at(dz, (np.arange(T)[:, None], ids), w * (dw - (w * dw).sum(1, keepdims=True)))
    out = Guarded((T, E), torch.float32, shift)
    _call("moe_route_grad", *gpu(ids, w, dw), T, E, k, out)
    assert np.array_equal(out.t.cpu().numpy(), dz) and out.intact()


@pytest.mark.parametrize("scale_shift", [0, 1, 2, 7])
@pytest.mark.parametrize("K", [32, 160])
def test_quantise_and_back(scale_shift, K):
    T, k = 21, 4
    ids, w, offsets, s2f, f2s = routing(T, 16, k, 9)
    x = np.random.default_rng(K).standard_normal((T, K)).astype(np.float32)
    codes, scales = Guarded((T * k, K // 2), torch.uint8, 16), Guarded((T * k, K // 32), torch.uint8, scale_shift)
    dx, ds2f, df2s = gpu(x, s2f, f2s)
    _call("moe_mx_quantize", dx, K, moe.MOE_DTYPE_FP32, T, k, K, ds2f, df2s, codes, scales)
    x64 = x.astype(np.float64)[s2f // k]
    assert np.array_equal(scales.t.cpu().numpy(), scale_bytes(x64)) and np.array_equal(values_of(codes.t.cpu(), scales.t.cpu()), quantised(x64))
    assert codes.intact() and scales.intact()
    for dtype, code in ((torch.float32, moe.MOE_DTYPE_FP32), (torch.bfloat16, moe.MOE_DTYPE_BF16)):
        back = Guarded((T * k, K), dtype, 16)
        _call("moe_mx_dequantize", codes, scales, T * k, K, code, back)
        assert torch.equal(back.t.cpu(), torch.from_numpy(quantised(x64)).to(dtype)) and back.intact()
