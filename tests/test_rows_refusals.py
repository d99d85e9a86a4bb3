"""What the calls on sorted rows and 4-bit experts refuse, found before anything reaches a GPU."""
import pytest
import torch

import paper_2607_18002_b200 as moe
from paper_2607_18002_b200 import build as moe_build


@pytest.fixture(scope="module")
def lib():
    moe_build.build()
    return moe.lib()


P = 1 << 20          # stands for an aligned device address: a call that is refused does not look at it
GOOD = {
    "moe_sort_rows": (P, 64, 0, 4, 2, 64, P, P, P, None),
    "moe_sort_rows_grad": (P, 64, 0, 4, 2, 64, P, P, None),
    "moe_merge_rows": (P, 64, 0, P, 4, 2, 64, P, P, None),
    "moe_merge_rows_grad": (P, 64, P, 64, 0, P, 4, 2, 64, P, P, P, P, None),
    "moe_route_grad": (P, P, P, 4, 8, 2, P, None),
    "moe_mx_quantize": (P, 64, 0, 4, 2, 64, P, P, P, P, None),
    "moe_mx_dequantize": (P, P, 4, 64, 0, P, None),
    "moe_mx_product": (P, P, P, P, P, 4, 8, 64, 128, P, None),
    "moe_mx_swiglu": (P, P, P, P, P, 4, 8, 64, 128, P, P, None),
}
BAD = [
    *[("moe_sort_rows", i, v) for i, v in ((0, None), (0, P + 1), (1, 63), (2, 4), (2, -1), (3, -1), (4, 0), (4, 33), (5, 0), (6, None), (7, None), (7, P + 2), (8, None),
                                           (3, 1 << 26))],
    ("moe_sort_rows", 5, (1 << 30) + 1), ("moe_merge_rows", 6, (1 << 30) + 1), ("moe_mx_quantize", 5, (1 << 30) + 32), ("moe_mx_dequantize", 3, (1 << 30) + 32),
    ("moe_mx_product", 7, (1 << 30) + 1), ("moe_mx_product", 8, (1 << 30) + 128), ("moe_mx_swiglu", 7, (1 << 29) + 32),
    *[("moe_sort_rows_grad", i, v) for i, v in ((0, None), (1, 63), (2, 1), (3, -1), (4, 0), (5, -1), (6, None), (7, None), (7, P + 1))],
    *[("moe_merge_rows", i, v) for i, v in ((0, None), (1, 1), (2, 1), (2, 9), (3, None), (3, P + 2), (4, -5), (5, 33), (6, 0), (7, None), (8, None))],
    *[("moe_merge_rows_grad", i, v) for i, v in ((0, None), (1, 63), (2, None), (3, 63), (4, 1), (5, None), (6, -1), (7, 0), (8, 0), (9, None), (10, None), (11, None),
                                                 (12, None), (12, P + 1))],
    *[("moe_route_grad", i, v) for i, v in ((0, None), (1, None), (2, None), (3, -1), (4, 0), (4, 1025), (5, 0), (5, 9), (6, None))],
    *[("moe_mx_quantize", i, v) for i, v in ((0, None), (0, P + 1), (1, 63), (2, 1), (3, -1), (4, 0), (4, 33), (5, 48), (5, 0), (6, None), (7, None), (8, None), (8, P + 2),
                                             (9, None))],
    *[("moe_mx_dequantize", i, v) for i, v in ((0, None), (1, None), (2, -1), (3, 16), (4, 1), (5, None), (5, P + 8), (2, 1 << 50))],
    *[("moe_mx_product", i, v) for i, v in ((0, None), (0, P + 8), (1, P + 2), (2, P + 8), (3, None), (3, P + 1), (4, None), (5, -1), (5, 1 << 27), (6, 0), (6, 1025), (7, 0),
                                            (8, 64), (8, 192), (9, None), (9, P + 1))],
    *[("moe_mx_swiglu", i, v) for i, v in ((0, None), (2, P + 4), (4, None), (5, -1), (6, 0), (7, 48), (7, 0), (8, 96), (9, None), (9, P + 2), (10, None))],
]


@pytest.mark.parametrize("name,at,value", BAD)
def test_the_library_refuses(lib, name, at, value):
    args = list(GOOD[name])
    args[at] = value
    assert getattr(lib, name)(*args) == moe.MOE_EINVAL


def test_a_permutation_for_quantise_is_both_arrays_or_neither(lib):
    args = list(GOOD["moe_mx_quantize"])
    args[6] = args[7] = None
    assert lib.moe_mx_quantize(*args) == moe.MOE_EINVAL              # top_k = 2 without a permutation


@pytest.mark.parametrize("name,at", [("moe_sort_rows", 3), ("moe_sort_rows_grad", 3), ("moe_merge_rows", 4), ("moe_merge_rows_grad", 6), ("moe_route_grad", 3),
                                     ("moe_mx_quantize", 3), ("moe_mx_dequantize", 2), ("moe_mx_product", 5), ("moe_mx_swiglu", 5)])
def test_no_rows_is_nothing_to_do(lib, name, at):
    args = [None if a == P else a for a in GOOD[name]]
    args[at] = 0
    if name == "moe_mx_quantize":
        args[4] = 1
    assert getattr(lib, name)(*args) == moe.MOE_OK


def test_contexts_compute_in_their_own_types_only(lib):
    for dtype in (moe.MOE_DTYPE_FP16, moe.MOE_DTYPE_FP32):
        with pytest.raises(moe.MoeError):
            moe.moe_workspace_bytes(moe.moe_config_t(8, 2, 256, 128, dtype, 16, 1, 0, 0, 0))


def test_stream_and_device_are_read_the_public_way_where_torch_lacks_the_other(monkeypatch):
    import importlib.util
    import types
    from paper_2607_18002_b200 import rows
    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda gpu: types.SimpleNamespace(cuda_stream=40 + gpu))
    spec = importlib.util.spec_from_file_location("rows_without", rows.__file__)
    again = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(again)
    assert again._current_device is torch.cuda.current_device and again._stream(2) == 42


def test_tensors_on_the_host_are_refused():
    x, i, w = torch.zeros(4, 64), torch.zeros(8, dtype=torch.int32), torch.zeros(4, 2)
    c, s = torch.zeros(8, 64, dtype=torch.uint8), torch.zeros(8, 4, dtype=torch.uint8)
    for call in (lambda: moe.sort_rows(x, i, i, 2), lambda: moe.sort_rows_grad(x, i, 2), lambda: moe.merge_rows(x, i, w),
                 lambda: moe.merge_rows_grad(x, x, i, i, w), lambda: moe.route_grad(i.view(4, 2), w, w, 8), lambda: moe.mx_quantize(x),
                 lambda: moe.mx_dequantize(c, s), lambda: moe.mx_product(c, s, c.view(1, 8, 64), s.view(1, 8, 4), i),
                 lambda: moe.mx_swiglu(c, s, c.view(1, 8, 64), s.view(1, 8, 4), i)):
        with pytest.raises(ValueError):
            call()


def _gpu_calls():
    x = torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda")
    i = torch.arange(8, dtype=torch.int32, device="cuda")
    w = torch.zeros(4, 2, device="cuda")
    c, s = torch.zeros(8, 64, dtype=torch.uint8, device="cuda"), torch.zeros(8, 4, dtype=torch.uint8, device="cuda")
    wc, ws = torch.zeros(2, 128, 64, dtype=torch.uint8, device="cuda"), torch.zeros(2, 128, 4, dtype=torch.uint8, device="cuda")
    o = torch.zeros(3, dtype=torch.int32, device="cuda")
    return {
        "transposed rows": lambda: moe.sort_rows(x.T, i, i, 2), "index of another length": lambda: moe.sort_rows(x[:4], i[:7], i, 2),
        "index of 64 bits": lambda: moe.sort_rows(x[:4], i.long(), i, 2), "rows of doubles": lambda: moe.sort_rows(x[:4].double(), i, i, 2),
        "rows that overlap": lambda: moe.sort_rows(x[:1].expand(4, 64), i, i, 2), "three dimensions": lambda: moe.sort_rows(x.view(2, 4, 64), i, i, 2),
        "one-byte gradient": lambda: moe.sort_rows_grad(c, i, 2), "rows that are no multiple of k": lambda: moe.sort_rows_grad(x, i, 3),
        "weights of another type": lambda: moe.merge_rows(x, i, w.double()), "weights of another size": lambda: moe.merge_rows(x, i, w[:3]),
        "weights with a stride": lambda: moe.merge_rows(x, i, torch.zeros(4, 4, device="cuda")[:, :2]),
        "gradient of another type": lambda: moe.merge_rows_grad(x[:4].float(), x, i, i, w),
        "gradient of another width": lambda: moe.merge_rows_grad(x[:4, :32], x, i, i, w),
        "gradient of another height": lambda: moe.merge_rows_grad(x[:3], x, i, i, w),
        "ids of 64 bits": lambda: moe.route_grad(i.view(4, 2).long(), w, w, 8), "weights of another shape": lambda: moe.route_grad(i.view(4, 2), w, w[:3], 8),
        "48 columns": lambda: moe.mx_quantize(x[:, :48]), "k without a permutation": lambda: moe.mx_quantize(x, top_k=2),
        "half a permutation": lambda: moe.mx_quantize(x[:4], i, None, 2), "scales of another size": lambda: moe.mx_dequantize(c, s[:, :3]),
        "codes with a stride": lambda: moe.mx_dequantize(c[:, :32], s[:, :2]), "values of doubles": lambda: moe.mx_dequantize(c, s, torch.float64),
        "weights of another depth": lambda: moe.mx_product(c, s, wc[..., :32].contiguous(), ws[..., :2].contiguous(), o),
        "offsets of another length": lambda: moe.mx_product(c, s, wc, ws, i), "two-dimensional weights": lambda: moe.mx_product(c, s, wc[0], ws[0], o),
        "gate and up of 48 rows": lambda: moe.mx_swiglu(c, s, wc[:, :96].contiguous(), ws[:, :96].contiguous(), o),
    }


NAMES = ["transposed rows", "index of another length", "index of 64 bits", "rows of doubles", "rows that overlap", "three dimensions", "one-byte gradient",
         "rows that are no multiple of k", "weights of another type", "weights of another size", "weights with a stride", "gradient of another type",
         "gradient of another width", "gradient of another height", "ids of 64 bits", "weights of another shape", "48 columns", "k without a permutation",
         "half a permutation", "scales of another size", "codes with a stride", "values of doubles", "weights of another depth", "offsets of another length",
         "two-dimensional weights", "gate and up of 48 rows"]


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_tensors_that_do_not_fit_are_refused(name):
    calls = _gpu_calls()
    assert sorted(calls) == sorted(NAMES)
    with pytest.raises(ValueError):
        calls[name]()


@pytest.mark.gpu
def test_what_the_library_refuses_raises():
    c, s = torch.zeros(8, 96, dtype=torch.uint8, device="cuda"), torch.zeros(8, 6, dtype=torch.uint8, device="cuda")
    o = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(moe.MoeError) as ei:                          # 192 columns: no multiple of 128
        moe.mx_product(c, s, c.view(1, 8, 96), s.view(1, 8, 6), o)
    assert ei.value.code == moe.MOE_EINVAL
    with pytest.raises(moe.MoeError):
        moe.sort_rows(torch.zeros(1, 64, device="cuda"), *[torch.zeros(33, dtype=torch.int32, device="cuda")] * 2, 33)
