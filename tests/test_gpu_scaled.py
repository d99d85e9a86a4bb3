"""e4m3 with block scales: quantising, values, products of sorted rows, and a layer of them."""
import numpy as np
import pytest
import torch

import paper_2607_18002_b200 as moe
from tests import rows_util as ru, scaled_util as su

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _values(shape, seed, dtype, spread=6):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, generator=g) * torch.exp2(torch.randint(-spread, spread + 1, (*shape[:-1], 1), generator=g).float())
    return x.to(DT[dtype])


def _check_quantised(x, codes, scales, rows):
    x64 = su.to_numpy(x)
    want = su.block_scales(x64, rows)
    assert np.array_equal(scales.cpu().numpy(), want, equal_nan=True)
    s = su.spread(want, rows, *x64.shape[-2:])
    on = np.isfinite(s)
    with np.errstate(invalid="ignore"):
        ref = su.nearest_code(np.where(on, x64, 0) / np.where(on, s, 1))
    assert np.array_equal(su.bytes_of(codes)[on], ref[on])


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("T,K", [(1, 16), (1, 4096), (3, 112), (33, 128), (129, 2048), (65, 144), (7, 1008)])
def test_rows_are_quantised_to_the_nearest_code(T, K, dtype):
    x = _values((T, K), T + K, dtype).cuda()
    x[0, :min(K, 128)] = 0
    codes, scales = moe.scaled_quantize(x)
    assert codes.dtype == torch.float8_e4m3fn and scales.shape == (T, -(-K // 128))
    _check_quantised(x, codes, scales, 1)
    back = moe.scaled_dequantize(codes, scales, x.dtype)
    ref = su.values_of(su.bytes_of(codes), scales.cpu().numpy(), 1)
    assert np.all(np.abs(su.to_numpy(back) - ref) <= np.abs(ref) * (torch.finfo(x.dtype).eps / 2 + 2.0 ** -24) + torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("E,n,K", [(1, 1, 16), (2, 127, 128), (3, 129, 144), (1, 300, 1008), (2, 256, 2048), (5, 128, 384)])
def test_weights_are_quantised_to_the_nearest_code(E, n, K, dtype):
    w = _values((E, n, K), E + n + K, dtype).cuda()
    w[0, :min(n, 128), :min(K, 128)] = 0
    codes, scales = moe.scaled_quantize_weights(w)
    assert scales.shape == (E, -(-n // 128), -(-K // 128))
    _check_quantised(w, codes, scales, 128)
    back = moe.scaled_dequantize(codes, scales, torch.float32)
    assert np.array_equal(su.to_numpy(back), su.values_of(su.bytes_of(codes), scales.cpu().numpy(), 128).astype(np.float32).astype(np.float64))
    one = moe.scaled_quantize_weights(w[0])
    assert torch.equal(one[0].view(torch.uint8), codes[0].view(torch.uint8)) and torch.equal(one[1], scales[0])


def test_quotients_next_to_midpoints_are_rounded_as_the_exact_ones():
    """Values whose quotient by the scale lies within a few fp32 steps of the middle of two codes, for scales of many magnitudes."""
    rng = np.random.default_rng(1)
    T, K = 600, 128
    top = (rng.random(T) + 0.5) * np.exp2(rng.integers(-140, 100, T))
    top = np.maximum(top, 448 * 2.0 ** -148).astype(np.float32)
    scale = su.block_scales(top.astype(np.float64)[:, None].repeat(16, 1), 1)[:, 0]
    mid = 0.5 * (su.GRID[1:] + su.GRID[:-1])
    at = (mid[rng.integers(0, 126, (T, K))] * scale[:, None].astype(np.float64)).astype(np.float32)
    x = (at.view(np.int32) + rng.integers(-2, 3, (T, K)).astype(np.int32)).clip(0).view(np.float32) * rng.choice([-1, 1], (T, K)).astype(np.float32)
    x = np.where(np.abs(x) <= top[:, None], x, 0).astype(np.float32)
    x[:, 0] = top
    t = torch.from_numpy(x).cuda()
    _check_quantised(t, *moe.scaled_quantize(t), 1)
    _check_quantised(t[None, :128], *moe.scaled_quantize_weights(t[None, :128].contiguous()), 128)


def test_extremes_and_blocks_with_nan():
    x = torch.zeros(8, 256)
    x[0, 0] = torch.finfo(torch.float32).max
    x[1, 0] = 2.0 ** -149                                  # the smallest number: its scale is held at 2^-126
    x[2, :128] = float("nan"); x[2, 128:] = 1.0
    x[3, 5] = float("inf"); x[4, 200] = -float("inf")
    x[5] = -448.0
    x[6, :] = torch.linspace(-1, 1, 256)
    x = x.cuda()
    codes, scales = moe.scaled_quantize(x)
    _check_quantised(x, codes, scales, 1)
    v = moe.scaled_dequantize(codes, scales, torch.float32)
    assert torch.isnan(v[2, :128]).all() and (v[2, 128:] == 1).all() and torch.isnan(v[3, :128]).all() and (v[3, 128:] == 0).all()
    assert (v[7] == 0).all() and (scales[7] == 1).all()
    # such a row spoils its own outputs and nobody else's
    w = moe.scaled_quantize_weights(torch.randn(64, 256, device="cuda"))
    for n in (1, 40):
        y = moe.scaled_product(codes.repeat(n, 1), scales.repeat(n, 1), *w)
        bad = torch.isnan(y).any(1)
        assert torch.equal(bad, torch.tensor([False, False, True, True, True, False, False, False], device="cuda").repeat(n))


@pytest.mark.parametrize("dtype", list(DT))
def test_rows_with_strides_and_any_alignment(dtype):
    wide = _values((40, 300), 5, dtype).cuda()
    for at in (0, 1, 7, 8):
        x = wide[:, at:at + 272]
        a, b = moe.scaled_quantize(x), moe.scaled_quantize(x.contiguous())
        assert torch.equal(a[0].view(torch.uint8), b[0].view(torch.uint8)) and torch.equal(a[1], b[1])
    three = _values((2, 3, 128), 6, dtype).cuda()
    codes, scales = moe.scaled_quantize(three)
    assert codes.shape == (2, 3, 128) and scales.shape == (2, 3, 1)
    assert torch.equal(codes[1, 2].view(torch.uint8), moe.scaled_quantize(three[1, 2])[0].view(torch.uint8))
    assert moe.scaled_dequantize(*moe.scaled_quantize(three[1, 2])).shape == (128,)


@pytest.mark.parametrize("T,E,k,K,rejected", [(1, 8, 2, 128, 0), (50, 8, 3, 272, 20), (130, 16, 4, 1024, 0), (300, 5, 5, 16, 7)])
def test_sorting_on_the_way(T, E, k, K, rejected):
    _, _, _, s2f, f2s = ru.routing(T, E, k, 3, rejected)
    x = _values((T, K), 7, "bf16").cuda()
    s, f = ru.gpu(s2f, f2s)
    plain = moe.scaled_quantize(x)
    codes, scales = moe.scaled_quantize(x, s, f, k)
    has = s2f >= 0
    token = np.where(has, s2f // k, 0)
    want_codes = np.where(has[:, None], su.bytes_of(plain[0])[token], 0)
    want_scales = np.where(has[:, None], plain[1].cpu().numpy()[token], 1)
    assert np.array_equal(su.bytes_of(codes), want_codes) and np.array_equal(scales.cpu().numpy(), want_scales)


@pytest.mark.parametrize("dtype", list(DT))
def test_every_code_has_its_value(dtype):
    codes = torch.arange(256, dtype=torch.uint8).view(2, 128).cuda()
    scales = torch.tensor([[0.5], [3.0]]).cuda()
    v = moe.scaled_dequantize(codes, scales, DT[dtype])
    ref = torch.from_numpy(su.values_of(codes.cpu().numpy(), scales.cpu().numpy(), 1)).to(DT[dtype])
    assert torch.equal(torch.nan_to_num(v.cpu(), 12345.0), torch.nan_to_num(ref, 12345.0))


def _offsets(R, E, rng, uneven=True):
    cut = np.sort(rng.integers(0, R + 1, E - 1)) if uneven else np.arange(1, E) * R // E
    return np.concatenate([[0], cut, [R]]).astype(np.int32)


def _check_product(x, w, offsets, dtype, got):
    ref, size = su.product_of(su.values_of(*x, 1), su.values_of(*w, 128), offsets)
    bound = su.product_error(x[0].shape[1], size) + np.abs(ref) * torch.finfo(dtype).eps / 2 + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    err = np.abs(su.to_numpy(got) - ref)
    assert np.all(err <= bound), (err - bound).max()


SIZES = [(1, 1, 1, 16), (1, 4, 300, 128), (5, 8, 5, 144), (64, 1, 256, 1008), (65, 1, 257, 512), (200, 3, 128, 2048), (333, 40, 1003, 1008), (700, 2, 255, 640),
         (1300, 5, 513, 384), (257, 1, 64, 4096), (2500, 16, 384, 128), (64 * 9, 9, 640, 1152), (8, 1024, 130, 256)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("R,E,N,K", SIZES)
def test_product_against_64_bits(R, E, N, K, dtype):
    rng = np.random.default_rng(R + N + K)
    offsets = _offsets(R, E, rng)
    x, w = su.random_rows(R, K, rng), su.random_weights(E, N, K, rng)
    y = moe.scaled_product(*su.on_gpu(*x), *su.on_gpu(*w), ru.gpu(offsets), DT[dtype])
    assert y.shape == (R, N) and y.dtype == DT[dtype]
    _check_product(x, w, offsets, DT[dtype], y)
    again = moe.scaled_product(*su.on_gpu(*x), *su.on_gpu(*w), ru.gpu(offsets), DT[dtype])
    assert torch.equal(y, again)


@pytest.mark.parametrize("R,N,K", [(1, 300, 512), (3, 6144, 4096), (17, 1000, 4096), (63, 128, 1008), (1000, 257, 256)])
def test_one_matrix_for_all_rows(R, N, K):
    rng = np.random.default_rng(R)
    x, w = su.random_rows(R, K, rng), su.random_weights(1, N, K, rng)
    codes, scales = su.on_gpu(*w)
    y = moe.scaled_product(*su.on_gpu(*x), codes[0], scales[0], dtype=torch.float32)
    _check_product(x, w, [0, R], torch.float32, y)
    assert torch.equal(y, moe.scaled_product(*su.on_gpu(*x), codes, scales, dtype=torch.float32))
    assert torch.equal(y, moe.scaled_product(*su.on_gpu(*x), codes, scales, ru.gpu(np.array([0, R], np.int32)), dtype=torch.float32))
    u = moe.scaled_product(su.on_gpu(*x)[0].view(torch.uint8), su.on_gpu(*x)[1], codes.view(torch.uint8), scales, dtype=torch.float32)
    assert torch.equal(y, u)


@pytest.mark.parametrize("R,E,N,K", [(40, 3, 300, 1024), (900, 3, 300, 1024), (64, 1, 512, 4096), (300, 1, 512, 4096)])
def test_products_that_fp32_holds_are_exact(R, E, N, K):
    """Codes of small whole numbers, scales that are powers of two over a narrow range: every sum is a whole number of a common power of two below 2^24."""
    rng = np.random.default_rng(K)
    small = np.array([su.nearest_code(np.float64(v)) for v in range(-3, 4)], np.uint8)
    xc, wc = small[rng.integers(0, 7, (R, K))], small[rng.integers(0, 7, (E, N, K))]
    xs = np.exp2(rng.integers(-1, 2, (R, -(-K // 128)))).astype(np.float32)
    ws = np.exp2(rng.integers(-1, 2, (E, -(-N // 128), -(-K // 128)))).astype(np.float32)       # |sum| <= 4096 * 9 * 4 = 147456, in steps of 1/4
    offsets = _offsets(R, E, rng)
    y = moe.scaled_product(*su.on_gpu(xc, xs), *su.on_gpu(wc, ws), ru.gpu(offsets), torch.float32)
    ref, _ = su.product_of(su.values_of(xc, xs, 1), su.values_of(wc, ws, 128), offsets)
    assert np.array_equal(su.to_numpy(y), ref)


@pytest.mark.parametrize("R", [60, 900])
def test_rows_of_no_expert_and_offsets_of_any_content(R):
    rng = np.random.default_rng(R)
    E, N, K = 4, 260, 256
    x, w, up = su.random_rows(R, K, rng), su.random_weights(E, N, K, rng), su.random_weights(E, 512, K, rng)
    offsets = np.array([7, 20, 20, R // 2, R - 5], np.int32)
    y = moe.scaled_product(*su.on_gpu(*x), *su.on_gpu(*w), ru.gpu(offsets), torch.float32)
    _check_product(x, w, offsets, torch.float32, y)
    assert (y[:7] == 0).all() and (y[R - 5:] == 0).all()
    codes, scales = moe.scaled_swiglu(*su.on_gpu(*x), *su.on_gpu(*up), ru.gpu(offsets))
    assert (codes.view(torch.uint8)[:7] == 0).all() and (scales[:7] == 1).all() and (scales[R - 5:] == 1).all()
    for bad in ([0, 0, 0, 0, 0], [-5, 10, 5, 2 ** 31 - 1, 3], [R, 0, R, 0, R], [2 ** 31 - 1] * 5, [-2 ** 31] * 5):
        held = np.maximum.accumulate(np.clip(np.array(bad, np.int64), 0, R))
        y = moe.scaled_product(*su.on_gpu(*x), *su.on_gpu(*w), ru.gpu(np.array(bad, np.int32)), torch.float32)
        _check_product(x, w, held, torch.float32, y)


def _check_swiglu(x, w, offsets, codes, scales):
    """The codes lie between those of the fp64 value moved down and up by the error bound, for the scale that was stored, and so does the scale."""
    I = w[0].shape[1] // 2
    h, size = su.product_of(su.values_of(*x, 1), su.values_of(*w, 128), offsets)
    g, u, eg, eu = h[:, :I], h[:, I:], *np.split(su.product_error(x[0].shape[1], size), 2, 1)
    with np.errstate(over="ignore"):
        silu = g / (1 + np.exp(-g))
    a = silu * u
    # silu' <= 1.1; exp(-g) to 2 + 1.2 |g| steps of 2^-23, reciprocal, product and product one each; below -87 silu counts as 0
    da = 1.1 * eg * (np.abs(u) + eu) + np.abs(silu) * eu + np.abs(a) * (8 + 1.2 * np.abs(g)) * su.STEP + np.abs(u) * 2.0 ** -119
    s = scales.cpu().numpy().astype(np.float64)
    R = a.shape[0]
    top, dtop = (np.abs(v).reshape(R, -1, 128).max(-1) for v in (a, da))
    assert np.all((np.abs(s - top / 448) <= (dtop + 2.0 ** -22 * top) / 448) | (top <= dtop))
    wide = np.repeat(s, 128, 1)
    q, dq = a / wide, da / wide + np.abs(a / wide) * 4 * su.STEP
    got = su.code_values(su.bytes_of(codes))
    lo, hi = su.code_values(su.nearest_code(q - dq)), su.code_values(su.nearest_code(q + dq))
    assert np.all((got >= lo) & (got <= hi))
    same = su.nearest_code(q)
    assert np.mean(su.code_values(same) != got) <= 0.02       # (an interval of two codes is rare: products are off by 2^-20, codes by 2^-4)


@pytest.mark.parametrize("R,E,I,K", [(1, 1, 128, 16), (1, 8, 384, 256), (5, 3, 256, 1008), (33, 1, 128, 512), (64, 1, 640, 1024), (100, 4, 256, 144), (300, 2, 384, 640),
                                     (65, 1, 128, 128), (129, 1, 256, 256), (1500, 7, 256, 384), (600, 40, 128, 272)])
def test_swiglu_against_64_bits(R, E, I, K):
    rng = np.random.default_rng(R + I)
    offsets = _offsets(R, E, rng)
    x, w = su.random_rows(R, K, rng, 1), su.random_weights(E, 2 * I, K, rng)
    codes, scales = moe.scaled_swiglu(*su.on_gpu(*x), *su.on_gpu(*w), ru.gpu(offsets))
    assert codes.shape == (R, I) and scales.shape == (R, I // 128)
    _check_swiglu(x, w, offsets, codes, scales)


@pytest.mark.parametrize("R", [10, 400])
def test_swiglu_of_gates_far_from_zero_and_of_zeros(R):
    K, I = 128, 256
    x = torch.ones(R, K)
    x[3] = 0
    w = torch.zeros(2 * I, K)
    w[:I, 0] = torch.linspace(-300, 300, I)
    w[I:, 1] = 1.0
    q, wq = moe.scaled_quantize(x.cuda()), moe.scaled_quantize_weights(w.cuda())
    codes, scales = moe.scaled_swiglu(*q, *wq)
    host = lambda t: (su.bytes_of(t[0]), t[1].cpu().numpy())
    v = su.values_of(*host((codes, scales)), 1)
    assert np.isfinite(v).all() and (v[3] == 0).all() and (scales[3] == 1).all()
    wc, ws = host(wq)
    keep = np.arange(R) != 3
    _check_swiglu((host(q)[0][keep], host(q)[1][keep]), (wc[None], ws[None]), [0, R - 1], codes[torch.from_numpy(keep).cuda()], scales[torch.from_numpy(keep).cuda()])


@pytest.mark.parametrize("T,E,k,H,I", [(1, 16, 4, 256, 128), (40, 8, 2, 512, 256), (300, 4, 2, 512, 384), (129, 64, 8, 256, 256)])
def test_a_layer_and_its_graph(T, E, k, H, I):
    """choose -> sort and quantise -> gate/up -> down -> merge, eagerly and replayed on new inputs, against 64 bits."""
    gen = torch.Generator().manual_seed(T)
    x, z = torch.randn(T, H, generator=gen).bfloat16().cuda(), torch.randn(T, E, generator=gen).cuda()
    w1 = moe.scaled_quantize_weights((torch.randn(E, 2 * I, H, generator=gen) * H ** -0.5).cuda())
    w2 = moe.scaled_quantize_weights((torch.randn(E, H, I, generator=gen) * I ** -0.5).cuda())
    bias = (0.1 * torch.randn(E, generator=gen)).cuda()

    def layer(x, z):
        ids, w = moe.choose_experts(z, k, scores="sigmoid", bias=bias, scale=1.5)
        order = torch.argsort(ids.flatten(), stable=True)
        s2f, f2s = order.int(), torch.argsort(order).int()
        offsets = (ids.flatten()[None] < torch.arange(E + 1, device="cuda")[:, None]).sum(1).int()
        a = moe.scaled_swiglu(*moe.scaled_quantize(x, s2f, f2s, k), *w1, offsets)
        d = moe.scaled_product(*a, *w2, offsets)
        return moe.merge_rows(d, f2s, w), ids, w

    def check(x, out):
        y, ids, w = out
        q = moe.scaled_quantize(x)
        x64 = su.values_of(su.bytes_of(q[0]), q[1].cpu().numpy(), 1)
        v1, v2 = (su.values_of(su.bytes_of(c), s.cpu().numpy(), 128) for c, s in (w1, w2))
        ref = np.zeros((T, H))
        for t in range(T):
            for j in range(k):
                e = ids[t, j].item()
                h = v1[e] @ x64[t]
                a = (h[:I] / (1 + np.exp(-h[:I])) * h[I:])[None]
                s = su.block_scales(a.astype(np.float32).astype(np.float64), 1)
                wide = su.spread(s, 1, 1, I)
                ref[t] += w[t, j].item() * (v2[e] @ (su.code_values(su.nearest_code(a / wide)) * wide)[0])
        # bf16 twice (2^-9 of rms each on average), and a code here and there that fell on the other side (2^-4 of one of I terms)
        assert np.linalg.norm(su.to_numpy(y) - ref) <= (2 * 2.0 ** -8 + 2.0 ** -8) * np.linalg.norm(ref)

    want = layer(x, z)
    check(x, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(x, z)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    x.copy_(torch.randn(T, H, generator=gen).bfloat16())
    z.copy_(torch.randn(T, E, generator=gen))
    graph.replay()
    check(x, out)


def test_gradient_to_the_rows_is_a_product_with_the_transposed_weights():
    rng = np.random.default_rng(5)
    R, E, N, K = 150, 3, 272, 384
    offsets = _offsets(R, E, rng)
    w = su.random_weights(E, N, K, rng)
    codes, scales = su.on_gpu(*w)
    turned = codes.view(torch.uint8).transpose(1, 2).contiguous(), scales.transpose(1, 2).contiguous()
    dy = su.random_rows(R, N, rng)
    dx = moe.scaled_product(*su.on_gpu(*dy), *turned, ru.gpu(offsets), torch.float32)
    v, dv = su.values_of(*w, 128), su.values_of(*dy, 1)
    for e in range(E):
        r = slice(offsets[e], offsets[e + 1])
        bound = su.product_error(N, np.abs(dv[r]) @ np.abs(v[e])) + 2.0 ** -24 * np.abs(dv[r] @ v[e])
        assert np.all(np.abs(su.to_numpy(dx)[r] - dv[r] @ v[e]) <= bound)


def test_no_rows_and_another_stream():
    w = moe.scaled_quantize_weights(torch.randn(2, 256, 128, device="cuda"))
    none = moe.scaled_quantize(torch.empty(0, 128, device="cuda"))
    assert none[0].shape == (0, 128) and none[1].shape == (0, 1)
    offsets = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert moe.scaled_product(*none, *w, offsets).shape == (0, 256)
    assert moe.scaled_swiglu(*none, *w, offsets)[1].shape == (0, 1)
    assert moe.scaled_dequantize(*none).shape == (0, 128)
    x = torch.randn(500, 128, device="cuda")
    offsets = torch.tensor([0, 100, 500], dtype=torch.int32, device="cuda")
    want = moe.scaled_product(*moe.scaled_quantize(x), *w, offsets)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q = moe.scaled_quantize(x, stream=side)
    y = moe.scaled_product(*q, *w, offsets, stream=side)
    mine = moe.scaled_product(*moe.scaled_quantize(x), *w, offsets)      # two at a time
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(want, y) and torch.equal(want, mine)
