"""Sizes past 32 bits: ctypes cuts longer numbers off without a word, so that a call on 2^32 + 5 rows would be one on 5.  What a call on tensors hands to the library fits, or the call
is refused."""
import ctypes

import pytest
import torch

import paper_2607_18002_b200 as moe
from paper_2607_18002_b200 import build as moe_build, rows

BIG = 2 ** 32
BF16, FP32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


class Shaped:
    """As much of a contiguous tensor on cuda:0 as the checks look at, without its elements."""
    is_cuda, device = True, torch.device("cuda", 0)

    def __init__(self, *shape, dtype=BF16, device=None):
        self.shape, self.dtype = torch.Size(shape), dtype

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for d in self.shape:
            n *= d
        return n

    def stride(self):
        out = [1]
        for d in self.shape[:0:-1]:
            out.insert(0, out[0] * max(d, 1))
        return tuple(out)

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def new_empty(self, *shape):
        return Shaped(*shape, dtype=self.dtype)


def _empty(*shape, dtype, device):
    return Shaped(*(shape[0] if isinstance(shape[0], torch.Size) else shape), dtype=dtype)


class Library:
    """Looks at what it is handed."""

    def __init__(self, real):
        self.real, self.calls = real, 0

    def __getattr__(self, name):
        types = getattr(self.real, name).argtypes

        def call(*args):
            self.calls += 1
            for i, (a, t) in enumerate(zip(args, types, strict=True)):
                if t is ctypes.c_int32:
                    assert -2 ** 31 <= a < 2 ** 31, f"{name}: argument {i} is {a}"
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    moe_build.build()
    fake = Library(moe.lib())
    monkeypatch.setattr(moe, "_lib", fake)
    for name, value in (("_Tensor", Shaped), ("_empty", _empty), ("_current_device", lambda: 0), ("_stream", lambda gpu: 0)):
        monkeypatch.setattr(rows, name, value)
    return fake


def _index(n):
    return Shaped(n, dtype=I32)


CALLS = {
    "sort_rows": lambda T=4, k=2, H=64: rows.sort_rows(Shaped(T, H), _index(T * k), _index(T * k), k),
    "sort_rows_grad": lambda T=4, k=2, H=64: rows.sort_rows_grad(Shaped(T * k, H), _index(T * k), k),
    "merge_rows": lambda T=4, k=2, H=64: rows.merge_rows(Shaped(T * k, H), _index(T * k), Shaped(T, k, dtype=FP32)),
    "merge_rows_grad": lambda T=4, k=2, H=64: rows.merge_rows_grad(Shaped(T, H), Shaped(T * k, H), _index(T * k), _index(T * k), Shaped(T, k, dtype=FP32)),
    "route_grad": lambda T=4, k=2, E=8: rows.route_grad(Shaped(T, k, dtype=I32), Shaped(T, k, dtype=FP32), Shaped(T, k, dtype=FP32), E),
    "mx_quantize": lambda T=4, k=2, K=64: rows.mx_quantize(Shaped(T, K), _index(T * k), _index(T * k), k),
    "mx_dequantize": lambda T=4, K=64: rows.mx_dequantize(Shaped(T, K // 2, dtype=U8), Shaped(T, K // 32, dtype=U8)),
    "mx_product": lambda R=4, E=8, n=64, K=128: rows.mx_product(Shaped(R, K // 2, dtype=U8), Shaped(R, K // 32, dtype=U8), Shaped(E, n, K // 2, dtype=U8),
                                                               Shaped(E, n, K // 32, dtype=U8), _index(E + 1)),
    "mx_swiglu": lambda R=4, E=8, n=128, K=128: rows.mx_swiglu(Shaped(R, K // 2, dtype=U8), Shaped(R, K // 32, dtype=U8), Shaped(E, n, K // 2, dtype=U8),
                                                              Shaped(E, n, K // 32, dtype=U8), _index(E + 1)),
    "choose_experts": lambda T=4, E=64, top_k=4, groups=8, top_groups=4, group_sum=2: rows.choose_experts(
        Shaped(T, E), top_k, groups=groups, top_groups=top_groups, group_sum=group_sum),
    "choose_experts_grad": lambda T=4, E=64, k=4: rows.choose_experts_grad(Shaped(T, E), Shaped(T, k, dtype=I32), Shaped(T, k, dtype=FP32)),
    "scaled_quantize": lambda T=4, K=64: rows.scaled_quantize(Shaped(T, K)),
    "scaled_quantize by expert": lambda T=4, k=2, K=64: rows.scaled_quantize(Shaped(T, K), _index(T * k), _index(T * k), k),
    "scaled_quantize_weights": lambda E=2, n=64, K=64: rows.scaled_quantize_weights(Shaped(E, n, K)),
    "scaled_quantize_weights of one": lambda n=64, K=64: rows.scaled_quantize_weights(Shaped(n, K)),
    "scaled_dequantize": lambda D=1, E=2, n=64, K=64: rows.scaled_dequantize(Shaped(D, E, n, K, dtype=U8), Shaped(D, E, n, -(-K // 128), dtype=FP32)),
    "scaled_dequantize of weights": lambda E=2, n=64, K=64: rows.scaled_dequantize(Shaped(E, n, K, dtype=U8), Shaped(E, -(-n // 128), -(-K // 128), dtype=FP32)),
    "scaled_product": lambda R=4, E=8, n=64, K=128: rows.scaled_product(Shaped(R, K, dtype=U8), Shaped(R, -(-K // 128), dtype=FP32), Shaped(E, n, K, dtype=U8),
                                                                       Shaped(E, -(-n // 128), -(-K // 128), dtype=FP32), _index(E + 1)),
    "scaled_product of one": lambda R=4, n=64, K=128: rows.scaled_product(Shaped(R, K, dtype=U8), Shaped(R, -(-K // 128), dtype=FP32), Shaped(n, K, dtype=U8),
                                                                         Shaped(-(-n // 128), -(-K // 128), dtype=FP32)),
    "scaled_swiglu": lambda R=4, E=8, n=256, K=128: rows.scaled_swiglu(Shaped(R, K, dtype=U8), Shaped(R, -(-K // 128), dtype=FP32), Shaped(E, n, K, dtype=U8),
                                                                      Shaped(E, -(-n // 128), -(-K // 128), dtype=FP32), _index(E + 1)),
}
SIZES = [(name, size, value) for name, call in CALLS.items() for size, at in zip(call.__code__.co_varnames, call.__defaults__)
         for value in (BIG + at, BIG // 2 + at - at % 2, BIG) if (name, size) != ("mx_dequantize", "T")]          # (whose rows are counted in 64 bits)


@pytest.mark.parametrize("name", list(CALLS))
def test_ordinary_sizes_reach_the_library(library, name):
    CALLS[name]()
    assert library.calls == 1


@pytest.mark.parametrize("name,size,value", SIZES)
def test_a_size_past_32_bits_is_refused(library, name, size, value):
    with pytest.raises((ValueError, moe.MoeError)):
        CALLS[name](**{size: value})
    assert library.calls == 0


@pytest.mark.parametrize("size", ["top_k", "groups", "top_groups", "group_sum"])
def test_negative_numbers_hide_no_others(library, size):
    """One that becomes an ordinary number when it is cut off, alone and beside others; those that fit are the library's to refuse."""
    for other in ("top_k", "groups", "top_groups", "group_sum"):
        for value, beside in ((1 - BIG, 1), (2 - BIG, 2 + BIG), (4 + BIG, -1), (4 - BIG, -1)):
            with pytest.raises(ValueError):
                rows.choose_experts(Shaped(4, 64), **{"top_k": 4, other: beside, size: value})
    assert library.calls == 0
    rows.choose_experts(Shaped(4, 64), **{"top_k": 4, size: -1})
    assert library.calls == 1


@pytest.mark.gpu
def test_large_tensors_are_refused():
    row = torch.empty(1, BIG + 16, dtype=U8, device="cuda")
    one = torch.zeros(1, dtype=I32, device="cuda")
    with pytest.raises(ValueError):
        moe.sort_rows(row, one, one, 1)
    with pytest.raises(ValueError):
        moe.scaled_dequantize(row, torch.empty(1, -(-row.shape[1] // 128), device="cuda"))
    del row
    logits = torch.empty(1, BIG + 8, dtype=BF16, device="cuda")
    with pytest.raises(ValueError):
        moe.choose_experts(logits, 2)
    with pytest.raises(ValueError):
        moe.choose_experts_grad(logits, torch.zeros(1, 2, dtype=I32, device="cuda"), torch.zeros(1, 2, device="cuda"))
    with pytest.raises(ValueError):
        moe.scaled_quantize(logits[:, :BIG])
    with pytest.raises(ValueError):
        moe.scaled_quantize_weights(logits[:, :BIG])
