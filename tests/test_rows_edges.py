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


@pytest.mark.parametrize("s2f,f2s", [(None, None), (P, None), (None, P), (P, P)])
def test_a_batch_without_tokens_needs_no_permutation(lib, s2f, f2s):
    """Arrays of no entries have no address: quantise-and-sort of no tokens is nothing to do whatever k is."""
    for dtype in (moe.MOE_DTYPE_BF16, moe.MOE_DTYPE_FP16, moe.MOE_DTYPE_FP32):
        assert lib.moe_mx_quantize(None, 64, dtype, 0, 8, 64, s2f, f2s, None, None, None) == moe.MOE_OK


@pytest.mark.gpu
@pytest.mark.parametrize("k", [1, 8])
def test_quantise_and_sort_of_a_batch_without_tokens(k):
    x, e = torch.empty(0, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    one = torch.zeros(1, dtype=torch.int32, device="cuda")           # (a plan without rows has arrays of one entry)
    for s2f, f2s in ((e, e), (one, one), (e, one)):
        codes, scales = moe.mx_quantize(x, s2f, f2s, k)
        assert codes.shape == (0, 64) and scales.shape == (0, 4)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(0, 128, 256), (4, 0, 64), (0, 0, 32), (2, 3, 0, 96), (1, 2, 3, 64)])
def test_quantise_of_more_dimensions_without_elements(shape):
    """A rank without experts, experts without rows."""
    x = torch.ones(shape, dtype=torch.bfloat16, device="cuda")
    codes, scales = moe.mx_quantize(x)
    assert codes.shape == (*shape[:-1], shape[-1] // 2) and scales.shape == (*shape[:-1], shape[-1] // 32)
    values = moe.mx_dequantize(codes, scales)
    assert values.shape == shape and torch.equal(values, x)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2, 3, 0), (0, 2, 0), (2, 3, 48)])
def test_quantise_of_more_dimensions_refuses_widths(shape):
    with pytest.raises(ValueError):
        moe.mx_quantize(torch.ones(shape, dtype=torch.bfloat16, device="cuda"))


@pytest.mark.gpu
def test_quantise_of_one_dimension_is_a_row():
    x = torch.randn(96, device="cuda")
    codes, scales = moe.mx_quantize(x)
    c2, s2 = moe.mx_quantize(x[None])
    assert codes.shape == (48,) and scales.shape == (3,) and torch.equal(codes, c2[0]) and torch.equal(scales, s2[0])
    assert torch.equal(moe.mx_dequantize(codes, scales, torch.float32), moe.mx_dequantize(c2, s2, torch.float32)[0])
    for bad in (x[::3], x[:48], torch.zeros((), device="cuda"), torch.zeros(0, device="cuda")):
        with pytest.raises(ValueError):
            moe.mx_quantize(bad)
    with pytest.raises(ValueError):
        moe.mx_quantize(x, *[torch.zeros(1, dtype=torch.int32, device="cuda")] * 2)


@pytest.mark.parametrize("T,E,k", [(1, 8, 2), (300, 40, 5), (8192, 300, 8), (2, 1024, 1)])
def test_the_permutation_of_the_documentation_is_a_plans(T, E, k):
    """The three lines of rows.py for permutations of any size, run as they stand there."""
    from paper_2607_18002_b200 import rows
    from rows_util import routing
    ids, w, offsets, s2f, f2s = routing(T, E, k, 17)
    lines = [line.strip() for line in rows.__doc__.splitlines()]
    at = lines.index("order = torch.argsort(topk_ids.flatten(), stable=True)")
    names = dict(torch=torch, topk_ids=torch.from_numpy(ids), n_experts=E)
    exec("\n".join(lines[at:at + 3]), names)
    for name, want in (("s2f", s2f), ("f2s", f2s), ("offsets", offsets)):
        assert names[name].dtype == torch.int32 and names[name].is_contiguous() and torch.equal(names[name], torch.from_numpy(want)), name
