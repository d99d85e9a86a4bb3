"""Products of e4m3 rows in all their forms: tiles shared by four CTAs, of 64, 128 and 256 rows, and what lies at their borders; results past 2^31 elements."""
import numpy as np
import pytest
import torch

import paper_2607_18002_b200 as moe
from tests import rows_util as ru, scaled_util as su
from tests.test_gpu_scaled import DT, _check_product, _check_swiglu, _offsets

pytestmark = pytest.mark.gpu


def _product(offsets, N, K, dtype, seed=0):
    R, E = int(offsets[-1]), len(offsets) - 1
    rng = np.random.default_rng([seed, R, N, K])
    x, w = su.random_rows(R, K, rng), su.random_weights(E, N, K, rng)
    y = moe.scaled_product(*su.on_gpu(*x), *su.on_gpu(*w), ru.gpu(np.asarray(offsets, np.int32)), DT[dtype])
    _check_product(x, w, offsets, DT[dtype], y)


def _swiglu(offsets, I, K, seed=0):
    R, E = int(offsets[-1]), len(offsets) - 1
    rng = np.random.default_rng([seed, R, I, K])
    x, w = su.random_rows(R, K, rng, 1), su.random_weights(E, 2 * I, K, rng)
    codes, scales = moe.scaled_swiglu(*su.on_gpu(*x), *su.on_gpu(*w), ru.gpu(np.asarray(offsets, np.int32)))
    _check_swiglu(x, w, offsets, codes, scales)


# up to eight rows in up to 32 tiles, eight blocks of K at least: four CTAs a tile
@pytest.mark.parametrize("offsets", [[0, 1], [0, 8], [0, 0, 5, 5], [0, 1, 2, 3], [0, 7, 7, 7, 8], [0, 2, 8]])
@pytest.mark.parametrize("N,K", [(256, 1024), (255, 1040), (700, 2160), (128, 4096)])
def test_tiles_that_four_share(offsets, N, K):
    for dtype in DT:
        _product(offsets, N, K, dtype)


@pytest.mark.parametrize("offsets", [[0, 1], [0, 8], [0, 0, 5, 5], [0, 1, 2, 3], [0, 7, 7, 7, 8], [0, 2, 8]])
@pytest.mark.parametrize("I,K", [(128, 1024), (256, 1040), (384, 2304)])
def test_gate_up_tiles_that_four_share(offsets, I, K):
    _swiglu(offsets, I, K)


@pytest.mark.parametrize("R", [8, 9, 32, 33, 64, 65, 127, 128, 129, 384, 385, 512, 513, 641])
def test_rows_at_the_borders_of_tiles_and_forms(R):
    _product([0, R], 384, 640, "bf16")
    _product([0, R], 131, 400, "fp32")
    _swiglu([0, R], 256, 400)


# (tiles of 64 columns up to 37 tiles of 128 rows x 256 columns)
@pytest.mark.parametrize("offsets,N", [([0, 9], 9472), ([0, 9], 9473), ([0, 129], 4608), ([0, 129], 4865), ([0, 5, 9, 9, 30], 2304), ([0, 128, 256, 384], 3000), ([0, 1, 1, 140], 65)])
@pytest.mark.parametrize("K", [16, 128, 400, 1152])
def test_columns_at_the_border_of_narrow_tiles(offsets, N, K):
    _product(offsets, N, K, "bf16")
    _product(offsets, N + 3, K, "fp32")


# (gate/up: 32 outputs a CTA in up to 32 tiles of 128 rows x 128 outputs)
@pytest.mark.parametrize("offsets,I", [([0, 9], 128), ([0, 64], 4096), ([0, 64], 4224), ([0, 129], 2048), ([0, 129], 2176), ([0, 5, 9, 9, 30], 384), ([0, 128, 256, 384], 512),
                                       ([0, 1, 1, 140], 256), ([0, 300], 128)])
@pytest.mark.parametrize("K", [16, 128, 400, 1152])
def test_gate_up_tiles_of_a_quarter(offsets, I, K):
    _swiglu(offsets, I, K)


# (per expert on average: 32 and 384 are the lines between the forms)
@pytest.mark.parametrize("offsets", [[0, 3, 3, 1200, 1201, 1600], [0, 900, 900, 2400], [0, 256, 768, 1280], [0, 1, 2, 1400], [0, 30, 400, 401, 640], [0, 63, 64, 65, 120]])
@pytest.mark.parametrize("K", [128, 272, 1152])
def test_uneven_experts_in_all_forms(offsets, K):
    _product(offsets, 520, K, "fp16")
    _product(offsets, 257, K, "fp32")
    _swiglu(offsets, 384, K)


@pytest.mark.parametrize("N", [1, 2, 63, 64, 65, 127, 129, 191, 255, 257, 383])
@pytest.mark.parametrize("R", [5, 200, 700])
def test_odd_columns_leave_what_lies_behind_them(N, R):
    """Outputs between guards: an odd row length writes its own columns and nothing else."""
    rng = np.random.default_rng(N)
    K = 144
    x, w = su.random_rows(R, K, rng), su.random_weights(1, N, K, rng)
    xg, wg = su.on_gpu(*x), su.on_gpu(*w)
    for dtype, code in ((torch.bfloat16, moe.MOE_DTYPE_BF16), (torch.float32, moe.MOE_DTYPE_FP32)):
        for shift in (0, 1, 8):
            space = torch.full((shift + R * N + 64,), 7.0, dtype=dtype, device="cuda")
            out = space[shift:shift + R * N]
            rc = moe.lib().moe_scaled_product(xg[0].data_ptr(), xg[1].data_ptr(), wg[0].data_ptr(), wg[1].data_ptr(), None, R, 1, N, K, code, out.data_ptr(),
                                              torch.cuda.current_stream().cuda_stream)
            assert rc == moe.MOE_OK
            _check_product(x, w, [0, R], dtype, out.view(R, N))
            assert (space[:shift] == 7).all() and (space[shift + R * N:] == 7).all()


@pytest.mark.parametrize("N", [8, 56, 72, 136, 200, 264, 328])
@pytest.mark.parametrize("per", [100, 400])
def test_boxes_of_outputs_that_columns_and_rows_end_in(N, per):
    """Many experts, whose segments end inside a warp's 32 rows, and row lengths that are whole 16-byte pieces but not whole boxes of 128 bytes; rows of no expert behind
    them."""
    rng = np.random.default_rng([N, per])
    E, K, behind = 24, 144, 40
    offsets = np.concatenate([[0], np.cumsum(per + rng.integers(-33, 34, E))]).astype(np.int32)
    R = int(offsets[-1])
    x, w = su.random_rows(R + behind, K, rng), su.random_weights(E, N, K, rng)
    xg, wg, off = su.on_gpu(*x), su.on_gpu(*w), ru.gpu(offsets)
    x = x[0][:R], x[1][:R]
    for dtype, code in ((torch.bfloat16, moe.MOE_DTYPE_BF16), (torch.float16, moe.MOE_DTYPE_FP16), (torch.float32, moe.MOE_DTYPE_FP32)):
        space = torch.full((8 + (R + behind) * N + 64,), 7.0, dtype=dtype, device="cuda")
        out = space[8:8 + (R + behind) * N]
        rc = moe.lib().moe_scaled_product(xg[0].data_ptr(), xg[1].data_ptr(), wg[0].data_ptr(), wg[1].data_ptr(), off.data_ptr(), R + behind, E, N, K, code, out.data_ptr(),
                                          torch.cuda.current_stream().cuda_stream)
        assert rc == moe.MOE_OK
        _check_product(x, w, offsets, dtype, out.view(R + behind, N)[:R])
        assert (out.view(R + behind, N)[R:] == 0).all() and (space[:8] == 7).all() and (space[8 + (R + behind) * N:] == 7).all()


def test_scales_far_apart():
    """Scales over sixty powers of two in one sum."""
    rng = np.random.default_rng(1)
    for R, K in ((4, 1024), (100, 640), (600, 640)):
        x, w = su.random_rows(R, K, rng), su.random_weights(1, 256, K, rng)
        x = x[0], (x[1] * np.exp2(rng.integers(-30, 31, x[1].shape))).astype(np.float32)
        w = w[0], (w[1] * np.exp2(rng.integers(-30, 31, w[1].shape))).astype(np.float32)
        y = moe.scaled_product(*su.on_gpu(*x), *su.on_gpu(*w), ru.gpu(np.array([0, R], np.int32)), torch.float32)
        _check_product(x, w, [0, R], torch.float32, y)


def test_two_streams_and_captured_forms_at_once():
    """Every form twice, on two streams at the same time and in a graph: nothing is shared between calls."""
    rng = np.random.default_rng(3)
    K, N = 1152, 512
    w, up = su.on_gpu(*su.random_weights(2, N, K, rng)), su.on_gpu(*su.random_weights(2, N, K, rng))
    for R in (6, 50, 300, 900):
        offsets = ru.gpu(np.array([0, R // 3, R], np.int32))
        a, b = su.on_gpu(*su.random_rows(R, K, rng)), su.on_gpu(*su.random_rows(R, K, rng))
        want = [(moe.scaled_product(*x, *w, offsets), *moe.scaled_swiglu(*x, *up, offsets)) for x in (a, b)]
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        got = [[], []]
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for _ in range(5):
            for i, x in enumerate((a, b)):
                got[i].append((moe.scaled_product(*x, *w, offsets, stream=streams[i]), *moe.scaled_swiglu(*x, *up, offsets, stream=streams[i])))
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = (moe.scaled_product(*a, *w, offsets), *moe.scaled_swiglu(*a, *up, offsets))
        for _ in range(3):
            graph.replay()
        got[0].append(out)
        for i in (0, 1):
            for g in got[i]:
                assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(g, want[i]))


def test_results_past_two_to_the_31():
    R, N, K = 70_000, 32_768, 32
    g = torch.Generator("cuda").manual_seed(1)
    x, w = torch.randn(R, K, device="cuda", generator=g), torch.randn(N, K, device="cuda", generator=g)
    xq, wq = moe.scaled_quantize(x), moe.scaled_quantize_weights(w)
    y = moe.scaled_product(*xq, *wq)
    assert y.numel() > 2 ** 31
    rows = torch.tensor([0, 1, 255, 256, 40_000, 65_535, 65_536, 69_998, 69_999], device="cuda")
    ref = moe.scaled_dequantize(xq[0][rows], xq[1][rows], torch.float32).double() @ moe.scaled_dequantize(*wq, torch.float32).double().T
    size = moe.scaled_dequantize(xq[0][rows], xq[1][rows], torch.float32).double().abs() @ moe.scaled_dequantize(*wq, torch.float32).double().abs().T
    assert (y[rows].double() - ref).abs().le((2 * 128 + 3 + 4) * 2.0 ** -24 * size + ref.abs() * 2.0 ** -8 * (1 + 2.0 ** -8)).all()
    del y
    few = torch.tensor([0, R], dtype=torch.int32, device="cuda")
    assert torch.equal(moe.scaled_product(*xq, wq[0][None], wq[1][None], few)[rows], moe.scaled_product(xq[0][rows], xq[1][rows], *wq))


def test_rows_and_weights_past_two_to_the_31():
    T, K = 540_000, 4096
    x = torch.empty(T, K, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(2))
    assert x.numel() > 2 ** 31
    codes, scales = moe.scaled_quantize(x)
    at = torch.tensor([0, 262_143, 262_144, 524_287, 524_288, T - 1], device="cuda")
    some = moe.scaled_quantize(x[at])
    assert torch.equal(codes[at].view(torch.uint8), some[0].view(torch.uint8)) and torch.equal(scales[at], some[1])
    back = moe.scaled_dequantize(codes, scales)
    assert torch.equal(back[at], moe.scaled_dequantize(*some))
    del back
    # rows far down the codes times one small matrix
    w = moe.scaled_quantize_weights(torch.randn(64, K, device="cuda"))
    y = moe.scaled_product(codes, scales, *w)
    tile = slice(T - 300, T)
    assert torch.equal(y[tile], moe.scaled_product(codes[tile].contiguous(), scales[tile].contiguous(), *w))
    del codes, scales, y
    W = x.view(-1, 1000, K)
    codes, scales = moe.scaled_quantize_weights(W)
    last = moe.scaled_quantize_weights(W[-1])
    assert torch.equal(codes[-1].view(torch.uint8), last[0].view(torch.uint8)) and torch.equal(scales[-1], last[1])
    y = moe.scaled_product(*some, codes, scales, torch.tensor([0] * 540 + [6], dtype=torch.int32, device="cuda"))
    assert torch.equal(y, moe.scaled_product(*some, *last))


def test_many_tokens_through_a_router():
    T, E = 300_000, 8192 // 16
    z = torch.randn(T, E, device="cuda", generator=torch.Generator("cuda").manual_seed(4))
    ids, w = moe.choose_experts(z, 8, scores="sigmoid")
    at = torch.tensor([0, 7, 131_071, 131_072, T - 1], device="cuda")
    some = moe.choose_experts(z[at], 8, scores="sigmoid")
    assert torch.equal(ids[at], some[0]) and torch.equal(w[at], some[1])
