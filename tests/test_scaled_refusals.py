"""What the routers by scores and the calls on e4m3 rows with block scales refuse, found before anything reaches a GPU."""
import pytest
import torch

import paper_2607_18002_b200 as moe
from paper_2607_18002_b200 import build as moe_build

P = 1 << 20          # stands for an aligned device address: a call that is refused does not look at it
GOOD = {
    "moe_choose_experts": (P, 64, 3, P, 4, 64, 6, 8, 3, 2, 1, 1, 1.0, P, P, None),
    "moe_choose_experts_grad": (P, 64, 3, P, P, 4, 64, 6, 1, 1, 1.0, P, None),
    "moe_scaled_quantize": (P, 64, 0, 4, 2, 64, P, P, P, P, None),
    "moe_scaled_quantize_weights": (P, 0, 2, 64, 128, P, P, None),
    "moe_scaled_dequantize": (P, P, 2, 64, 128, 128, 0, P, None),
    "moe_scaled_product": (P, P, P, P, P, 4, 8, 64, 128, 0, P, None),
    "moe_scaled_swiglu": (P, P, P, P, P, 4, 8, 128, 128, P, P, None),
}
BAD = [
    *[("moe_choose_experts", i, v) for i, v in ((0, None), (0, P + 2), (1, 63), (2, 1), (2, 4), (3, P + 2), (4, -1), (5, 0), (5, 1025), (6, 0), (6, 33), (6, 25), (7, 0), (7, 7),
                                                (7, 64), (8, 0), (8, 9), (9, 0), (9, 3), (10, 2), (10, -1), (13, None), (13, P + 1), (14, None), (14, P + 2))],
    *[("moe_choose_experts_grad", i, v) for i, v in ((0, None), (0, P + 1), (1, 63), (2, 1), (3, None), (3, P + 2), (4, None), (4, P + 1), (5, -1), (6, 0), (6, 1025), (7, 0), (7, 33),
                                                     (8, 2), (11, None), (11, P + 2))],
    *[("moe_scaled_quantize", i, v) for i, v in ((0, None), (0, P + 1), (1, 63), (2, 1), (2, 7), (3, -1), (3, 1 << 26), (4, 0), (4, 33), (5, 0), (5, 24), (5, (1 << 30) + 16), (6, None),
                                                 (6, P + 2), (7, None), (8, None), (8, P + 8), (9, None), (9, P + 2))],
    *[("moe_scaled_quantize_weights", i, v) for i, v in ((0, None), (0, P + 8), (1, 1), (2, -1), (3, 0), (3, (1 << 30) + 1), (4, 0), (4, 120), (5, None), (5, P + 8), (6, None), (6, P + 2),
                                                         (2, 1 << 30))],
    *[("moe_scaled_dequantize", i, v) for i, v in ((0, None), (0, P + 8), (1, None), (1, P + 2), (2, -1), (3, -1), (4, 0), (4, 72), (5, 2), (6, 1), (7, None), (7, P + 8), (2, 1 << 30))],
    *[("moe_scaled_product", i, v) for i, v in ((0, None), (0, P + 8), (1, None), (1, P + 2), (2, None), (2, P + 4), (3, None), (3, P + 1), (4, None), (4, P + 2), (5, -1), (5, 1 << 27),
                                                (6, 0), (6, 1025), (7, 0), (7, (1 << 30) + 1), (8, 0), (8, 120), (8, (1 << 30) + 16), (9, 1), (9, 9), (10, None), (10, P + 1))],
    *[("moe_scaled_swiglu", i, v) for i, v in ((0, None), (2, P + 8), (3, None), (4, None), (5, -1), (6, 0), (7, 0), (7, 64), (7, (1 << 29) + 128), (8, 8), (9, None), (9, P + 8),
                                               (10, None), (10, P + 2))],
]


@pytest.fixture(scope="module")
def lib():
    moe_build.build()
    return moe.lib()


@pytest.mark.parametrize("name,at,value", BAD)
def test_the_library_refuses(lib, name, at, value):
    args = list(GOOD[name])
    args[at] = value
    assert getattr(lib, name)(*args) == moe.MOE_EINVAL


@pytest.mark.parametrize("name,at", [("moe_choose_experts", 4), ("moe_choose_experts_grad", 5), ("moe_scaled_quantize", 3), ("moe_scaled_quantize_weights", 2),
                                     ("moe_scaled_dequantize", 2), ("moe_scaled_dequantize", 3), ("moe_scaled_product", 5), ("moe_scaled_swiglu", 5)])
def test_nothing_is_nothing_to_do(lib, name, at):
    args = [None if a == P else a for a in GOOD[name]]
    args[at] = 0
    assert getattr(lib, name)(*args) == moe.MOE_OK


def test_a_permutation_for_quantise_is_both_arrays_or_neither(lib):
    args = list(GOOD["moe_scaled_quantize"])
    args[6] = args[7] = None
    assert lib.moe_scaled_quantize(*args) == moe.MOE_EINVAL              # top_k = 2 without a permutation


def test_one_matrix_alone_needs_no_offsets(lib):
    args = list(GOOD["moe_scaled_product"])
    args[4], args[6] = None, 2
    assert lib.moe_scaled_product(*args) == moe.MOE_EINVAL


@pytest.mark.parametrize("call", [
    lambda: moe.choose_experts(torch.zeros(4, 8), 2),                                        # not on a GPU
    lambda: moe.choose_experts_grad(torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)),
    lambda: moe.scaled_quantize(torch.zeros(4, 128)),
    lambda: moe.scaled_quantize(torch.zeros(2, 4, 128)),
    lambda: moe.scaled_quantize_weights(torch.zeros(4, 128)),
    lambda: moe.scaled_dequantize(torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 1)),
    lambda: moe.scaled_dequantize(torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 1), torch.int32),
    lambda: moe.scaled_dequantize([1], torch.zeros(4, 1)),
    lambda: moe.scaled_product(torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 1), torch.zeros(8, 128, dtype=torch.uint8), torch.zeros(1, 1)),
    lambda: moe.scaled_swiglu(torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 1), torch.zeros(256, 128, dtype=torch.uint8), torch.zeros(2, 1)),
])
def test_tensors_that_are_not_on_a_gpu_are_refused(call):
    with pytest.raises(ValueError):
        call()


@pytest.mark.gpu
@pytest.mark.parametrize("change", [
    dict(logits=torch.int32), dict(bias=7), dict(scores="tanh"), dict(ids=torch.int64), dict(codes=torch.int8), dict(scales=torch.float64), dict(columns=24), dict(offsets=3),
    dict(weights=144), dict(gate=384), dict(top_k=2), dict(dtype=torch.float64), dict(no_offsets=True), dict(turned=True)])
def test_wrong_types_shapes_and_strides_raise(change):
    key, value = next(iter(change.items()))
    z = torch.zeros(6, 8, device="cuda")
    ids, d = torch.zeros(6, 2, dtype=torch.int32, device="cuda"), torch.zeros(6, 2, device="cuda")
    x = torch.zeros(6, 128, device="cuda")
    codes, scales = torch.zeros(6, 128, dtype=torch.uint8, device="cuda"), torch.ones(6, 1, device="cuda")
    w = torch.zeros(2, 256, 128, dtype=torch.uint8, device="cuda"), torch.ones(2, 2, 1, device="cuda")
    offsets = torch.zeros(3, dtype=torch.int32, device="cuda")
    call = {
        "logits": lambda: moe.choose_experts(z.to(torch.int32), 2),
        "bias": lambda: moe.choose_experts(z, 2, bias=torch.zeros(7, device="cuda")),
        "scores": lambda: moe.choose_experts(z, 2, scores="tanh"),
        "ids": lambda: moe.choose_experts_grad(z, ids.long(), d),
        "codes": lambda: moe.scaled_product(codes.view(torch.int8), scales, *w, offsets),
        "scales": lambda: moe.scaled_product(codes, scales.double(), *w, offsets),
        "columns": lambda: moe.scaled_quantize(x[:, :24]),
        "offsets": lambda: moe.scaled_product(codes, scales, *w, offsets[:2]),
        "weights": lambda: moe.scaled_product(codes[:, :112].contiguous(), scales, *w, offsets),
        "gate": lambda: moe.scaled_swiglu(codes, scales, torch.zeros(2, 384, 128, dtype=torch.uint8, device="cuda"), torch.ones(2, 3, 1, device="cuda"), offsets),
        "top_k": lambda: moe.scaled_quantize(x, top_k=2),
        "dtype": lambda: moe.scaled_product(codes, scales, *w, offsets, torch.float64),
        "no_offsets": lambda: moe.scaled_product(codes, scales, *w),
        "turned": lambda: moe.scaled_product(codes.t().contiguous().t(), scales, *w, offsets),
    }[key]
    with pytest.raises(ValueError):
        call()


@pytest.mark.gpu
def test_what_the_library_refuses_raises_its_error():
    z = torch.zeros(6, 8, device="cuda")
    for bad in (dict(top_k=0), dict(top_k=-1), dict(top_k=9), dict(top_k=2, groups=3), dict(top_k=5, groups=4, top_groups=2), dict(top_k=1, group_sum=3)):
        with pytest.raises(moe.MoeError):
            moe.choose_experts(z, **bad)
