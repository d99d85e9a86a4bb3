"""4-bit rows: quantisation, values, and products with the experts' matrices, against evaluations in 64 bits.

Quantisation and values are exact operations with one defined rounding: equality.  Products whose terms are small multiples of a common power of
two are exact in fp32, whatever the order of the additions: there the bf16 outputs have to be equal too.  Where terms are of any size, K terms of fp32
accumulation are off by at most K steps of 2^-23 of the sum of magnitudes."""
import numpy as np
import pytest
import torch

import paper_2607_18002_b200 as moe

from rows_util import EPS_FP32, gpu, half_step, quantised, round_to_grid, routing, scale_bytes, values_of

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


def _special(dtype):
    """Rows of 64 columns with values at and next to every border of the format, block maxima next to powers of two, zeros, and the
    smallest and largest numbers of the type."""
    g = torch.Generator().manual_seed(7)
    rows = []
    mids = [0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.0, 7.5]
    near = []
    for m in mids:
        v = torch.tensor(m).to(dtype)
        near += [v, torch.nextafter(v.float(), torch.tensor(9.0)).to(dtype) if dtype == torch.float32 else (v.float() * (1 + torch.finfo(dtype).eps)).to(dtype),
                 torch.nextafter(v.float(), torch.tensor(-1.0)).to(dtype) if dtype == torch.float32 else (v.float() * (1 - torch.finfo(dtype).eps / 2)).to(dtype)]
    near = torch.stack(near)
    for e in (0, 3, -4):
        row = torch.zeros(64, dtype=dtype)
        row[:51] = near[:51] * 2.0 ** e
        row[:25:2] *= -1
        row[51] = row[31] = 7 * 2.0 ** e                              # fixes the scale of both blocks
        rows.append(row)
    top = torch.finfo(dtype).max
    for amax in (1.0, 1.0 - torch.finfo(dtype).eps / 2, 2.0, 1.99, 3.0, 6.0, top, torch.finfo(dtype).tiny, torch.finfo(dtype).tiny * torch.finfo(dtype).eps,
                 torch.finfo(dtype).tiny * 2, torch.finfo(dtype).tiny * 8):
        row = (torch.rand(64, generator=g) * 2 - 1).double() * amax
        row[5], row[40] = amax, -amax
        rows.append(row.to(dtype))
    rows.append(torch.zeros(64, dtype=dtype))
    rows.append(torch.full((64,), -0.0).to(dtype))
    rows.append(torch.cat([torch.zeros(32), torch.ones(32)]).to(dtype))
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_borders_of_the_format(dtype):
    x = _special(dtype)
    codes, scales = moe.mx_quantize(x.cuda())
    x64 = x.double().numpy()
    assert np.array_equal(scales.cpu().numpy(), scale_bytes(x64))
    assert np.array_equal(values_of(codes.cpu(), scales.cpu()), quantised(x64))


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("T,K,pad,shift", [(1, 32, 0, 0), (7, 96, 0, 0), (129, 2048, 0, 0), (33, 160, 8, 0), (33, 160, 3, 0), (20, 256, 0, 1), (1000, 64, 0, 0)])
def test_quantise(dtype, T, K, pad, shift):
    g = torch.Generator().manual_seed(T + K)
    x = (torch.randn(T, K, generator=g) * torch.exp2(torch.randint(-9, 9, (T, 1), generator=g).float())).to(dtype)
    buf = torch.zeros(T * (K + pad) + shift, dtype=dtype, device="cuda")
    v = torch.as_strided(buf, (T, K), (K + pad, 1), shift)
    v.copy_(x)
    codes, scales = moe.mx_quantize(v)
    x64 = x.double().numpy()
    assert codes.shape == (T, K // 2) and scales.shape == (T, K // 32)
    assert np.array_equal(scales.cpu().numpy(), scale_bytes(x64))
    assert np.array_equal(values_of(codes.cpu(), scales.cpu()), quantised(x64))
    for out in DTYPES:
        got = moe.mx_dequantize(codes, scales, out).cpu()
        assert got.dtype == out and torch.equal(got, torch.from_numpy(quantised(x64)).to(out))


def test_quantise_of_more_dimensions_is_by_rows():
    w = torch.randn(3, 5, 96, device="cuda")
    codes, scales = moe.mx_quantize(w)
    assert codes.shape == (3, 5, 48) and scales.shape == (3, 5, 3)
    c2, s2 = moe.mx_quantize(w.view(15, 96))
    assert torch.equal(codes.view(15, 48), c2) and torch.equal(scales.view(15, 3), s2)
    assert torch.equal(moe.mx_dequantize(codes, scales).view(15, 96), moe.mx_dequantize(c2, s2))


def test_blocks_with_nan_or_infinity_are_nan():
    x = torch.ones(3, 128)
    x[0, 40], x[1, 0], x[2, 127] = float("nan"), float("inf"), -float("inf")
    for dtype in DTYPES:
        codes, scales = moe.mx_quantize(x.to(dtype).cuda())
        want = np.full((3, 4), 125)
        want[0, 1] = want[1, 0] = want[2, 3] = 255
        assert np.array_equal(scales.cpu().numpy(), want)
        for out in DTYPES:
            v = moe.mx_dequantize(codes, scales, out).cpu().float().numpy()
            assert np.array_equal(np.isnan(v), np.repeat(want == 255, 32, axis=1)) and np.all(v[~np.isnan(v)] == 1.0)


def test_every_code_and_scale_has_its_value():
    codes = torch.arange(256, dtype=torch.uint8).view(1, 256).expand(256, 256).contiguous()
    scales = torch.arange(256, dtype=torch.uint8).view(256, 1).expand(256, 16).contiguous()
    ref = values_of(codes, scales)
    got = moe.mx_dequantize(codes.cuda(), scales.cuda(), torch.float32).cpu()
    with np.errstate(over="ignore"):
        want = torch.from_numpy(ref.astype(np.float32))
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


@pytest.mark.parametrize("T,E,k,K,rejected", [(1, 8, 2, 128, 0), (40, 8, 3, 96, 0), (33, 16, 8, 2048, 5), (9, 32, 32, 64, 10 ** 6)])
def test_quantise_and_sort(T, E, k, K, rejected):
    ids, w, offsets, s2f, f2s = routing(T, E, k, 2, rejected)
    x = torch.randn(T, K).to(torch.bfloat16).cuda()
    codes, scales = moe.mx_quantize(x, *gpu(s2f, f2s), k)
    c0, s0 = moe.mx_quantize(x)
    assert torch.equal(codes, moe.sort_rows(c0, *gpu(s2f, f2s), k)) and torch.equal(scales, moe.sort_rows(s0, *gpu(s2f, f2s), k))


# ------------------------------------------------------------------ products

def _offsets(counts, lead=0):
    return np.concatenate([[lead], lead + np.cumsum(counts)]).astype(np.int32)


def _exact_operand(shape, K, seed, spread=1):
    """Codes of any value with scales of a few powers of two."""
    rng = np.random.default_rng(seed)
    return rng.integers(0, 256, (*shape, K // 2)).astype(np.uint8), (127 + rng.integers(-spread, spread + 1, (*shape, K // 32))).astype(np.uint8)


def _product64(x, w, offsets, R):
    out = np.zeros((R, w.shape[1]))
    for e in range(w.shape[0]):
        out[offsets[e]:offsets[e + 1]] = x[offsets[e]:offsets[e + 1]] @ w[e].T
    return out


def _bf16(a):
    return torch.from_numpy(a.astype(np.float32)).to(torch.bfloat16)       # exact in fp32 where it is used


COUNTS = {
    "one row": [1], "none at all but one": [0, 0, 3, 0], "odd": [5, 0, 17, 1, 33, 0, 2, 64], "around a tile": [31, 32, 33, 0, 65],
    "dense": [300], "large": [191, 192, 193, 385, 0, 7], "mid": [64, 65, 63, 40, 130, 20],
    "tall": [577, 192, 0, 390], "tall and one": [1100, 1, 33],            # more than 256 rows an expert, up to 64, and between: three heights of tiles
}


@pytest.mark.parametrize("counts", list(COUNTS.values()), ids=list(COUNTS))
@pytest.mark.parametrize("N,K", [(256, 256), (1000, 384), (64, 128), (1, 640), (513, 2048), (392, 512)])
def test_product_is_exact_where_fp32_is(counts, N, K):
    """|terms| <= 36 * 4, multiples of 2^-4: sums of up to 2048 of them take 18 + 4 bits."""
    E, R = len(counts), sum(counts)
    x, w = _exact_operand((R,), K, 1), _exact_operand((E, N), K, 2)
    off = _offsets(counts)
    got = moe.mx_product(*gpu(*x, *w, off)).cpu()
    ref = _product64(values_of(*x), values_of(*w), off, R)
    assert torch.equal(got, _bf16(ref))


def test_rows_of_no_expert_are_zero_and_segments_need_not_start_at_the_first_row():
    counts, K, N, lead, R = [3, 0, 40], 256, 300, 5, 60
    x, w = _exact_operand((R,), K, 3), _exact_operand((3, N), K, 4)
    off = _offsets(counts, lead)
    ref = _product64(values_of(*x), values_of(*w), off, R)
    got = moe.mx_product(*gpu(*x, *w, off)).cpu()
    assert torch.equal(got, _bf16(ref)) and (got[:lead] == 0).all() and (got[lead + 43:] == 0).all()
    codes, scales = moe.mx_swiglu(*gpu(*x, w[0][:, :256].copy(), w[1][:, :256].copy(), off))
    for t in (codes, scales):
        assert (t[:lead] == 0).all() and (t[lead + 43:] == 0).all() and t[lead:lead + 43].any()
    nobody = np.zeros(4, np.int32)
    assert (moe.mx_product(*gpu(*x, *w, nobody)) == 0).all()


def test_offsets_out_of_order_stay_inside_their_rows():
    """What the documentation forbids is not an access out of bounds: offsets count as the largest so far, inside [0, R]."""
    R, K, N, E = 40, 256, 128, 5
    x, w = _exact_operand((R,), K, 31), _exact_operand((E, N), K, 32)
    for off, held in (([-7, 10, 4, 30, 20, 90], [0, 10, 10, 30, 30, 40]), ([2 ** 31 - 1, 0, -2 ** 31, 5, 6, 7], [40] * 6), ([0, 40, 0, 40, 0, 40], [0, 40, 40, 40, 40, 40])):
        got = moe.mx_product(*gpu(*x, *w, np.array(off, np.int64).astype(np.int32))).cpu()
        assert torch.equal(got, _bf16(_product64(values_of(*x), values_of(*w), np.array(held), R)))


@pytest.mark.parametrize("E", [31, 32, 33, 64, 200, 1024])
def test_many_experts(E):
    """Every expert's segment is found, whatever its place in the scan over the experts."""
    rng = np.random.default_rng(E)
    counts = rng.integers(0, 4, E)
    R, K, N = int(counts.sum()), 128, 40
    x, w = _exact_operand((R,), K, 33), _exact_operand((E, N), K, 34)
    off = _offsets(counts)
    assert torch.equal(moe.mx_product(*gpu(*x, *w, off)).cpu(), _bf16(_product64(values_of(*x), values_of(*w), off, R)))


def test_product_of_any_scales():
    """Scales over forty powers of two: rounding of the accumulation, K steps of 2^-23 of the magnitudes at most."""
    counts, K, N = [70, 3, 0, 130], 1024, 320
    R, E = sum(counts), len(counts)
    rng = np.random.default_rng(8)
    x, w = _exact_operand((R,), K, 5), _exact_operand((E, N), K, 6)
    xs, ws = (127 + rng.integers(-20, 21, x[1].shape)).astype(np.uint8), (127 + rng.integers(-20, 21, w[1].shape)).astype(np.uint8)
    off = _offsets(counts)
    got = moe.mx_product(*gpu(x[0], xs, w[0], ws, off)).cpu().double().numpy()
    xv, wv = values_of(x[0], xs), values_of(w[0], ws)
    ref, mag = _product64(xv, wv, off, R), _product64(np.abs(xv), np.abs(wv), off, R)
    err = K * 2.0 ** -23 * mag
    assert np.all(np.abs(got - ref) <= half_step(torch.bfloat16) * np.abs(ref) + 2 * err)


def test_nan_blocks_reach_their_outputs_only():
    counts, K, N = [20, 30], 256, 256
    x, w = _exact_operand((50,), K, 7), _exact_operand((2, N), K, 8)
    x[1][4, 3] = 255
    w[1][1, 17, 0] = 255
    got = moe.mx_product(*gpu(*x, *w, _offsets(counts))).cpu()
    bad = torch.isnan(got)
    want = torch.zeros_like(bad)
    want[4] = True
    want[20:, 17] = True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("counts", [[20, 30], [420, 30]], ids=["low tiles", "high tiles"])
def test_nan_blocks_make_their_swiglu_blocks_nan(counts):
    K, I = 256, 96
    x, w = _exact_operand((sum(counts),), K, 7), _exact_operand((2, 2 * I), K, 8)
    x[1][4, 3] = 255                                                # a row
    w[1][1, 40, 0] = 255                                            # expert 1, gate column 40
    w[1][1, I + 95, 1] = 255                                        # ... and up column 95
    codes, scales = (t.cpu().numpy() for t in moe.mx_swiglu(*gpu(*x, *w, _offsets(counts))))
    want = np.zeros(scales.shape, bool)
    want[4] = True
    want[counts[0]:, 1:] = True
    assert np.array_equal(scales == 255, want)


def _swiglu_bounds(g, u):
    """silu(g) u, and how far off fp32 may be: exp to 2 + 1.2 |g| steps of 2^-23, a sum, a quotient to two steps, a product."""
    a = g / (1.0 + np.exp(-g)) * u
    return a, np.abs(a) * (2 + 1.2 * np.abs(g) + 1 + 2 + 1 + 1) * 2.0 ** -23


def _check_swiglu(got, g, u):
    codes, scales = (t.cpu().numpy() for t in got)
    a, d = _swiglu_bounds(g, u)
    lo, hi = np.abs(a) - d, np.abs(a) + d
    assert np.all((scales == scale_bytes(lo)) | (scales == scale_bytes(hi)))
    s = np.repeat(np.ldexp(1.0, scales.astype(np.int64) - 127), 32, axis=-1)
    v = values_of(codes, scales)
    mag = np.abs(v) / s
    assert np.all((mag >= round_to_grid(lo / s)) & (mag <= round_to_grid(hi / s)))
    assert np.all((v == 0) | (np.sign(v) == np.sign(a)))


@pytest.mark.parametrize("counts", list(COUNTS.values()), ids=list(COUNTS))
@pytest.mark.parametrize("I,K", [(32, 128), (128, 256), (160, 384), (512, 1024)])
def test_swiglu(counts, I, K):
    E, R = len(counts), sum(counts)
    x, w = _exact_operand((R,), K, 9, 0), _exact_operand((E, 2 * I), K, 10, 1)
    x[1][:] = 120                                                    # gate values of a few units
    off = _offsets(counts)
    got = moe.mx_swiglu(*gpu(*x, *w, off))
    h = _product64(values_of(*x), values_of(*w), off, R)
    _check_swiglu(got, h[:, :I], h[:, I:])


def test_swiglu_far_from_zero():
    """Gates of hundreds to thousands either way: silu is the gate itself, or nothing."""
    K, I = 256, 64
    x, w = _exact_operand((40,), K, 11, 0), _exact_operand((1, 2 * I), K, 12, 0)
    off = _offsets([40])
    codes, scales = moe.mx_swiglu(*gpu(*x, *w, off))
    h = _product64(values_of(*x), values_of(*w), off, 40)
    assert np.abs(h[:, :I]).max() > 200
    with np.errstate(over="ignore"):
        _check_swiglu((codes, scales), h[:, :I], h[:, I:])


def test_results_do_not_depend_on_the_run_or_on_neighbours():
    """A row's outputs are the same bits whatever other rows its tile holds, and in every run."""
    K, N = 512, 384
    w = gpu(*_exact_operand((3, N), K, 13, 6))
    x = gpu(*_exact_operand((400,), K, 14, 6))
    off = _offsets([150, 0, 250])
    all_rows = moe.mx_product(*x, *w, gpu(off))
    for _ in range(3):
        assert torch.equal(moe.mx_product(*x, *w, gpu(off)), all_rows)
    for at in (0, 149, 150, 399):
        one = moe.mx_product(x[0][at:at + 1], x[1][at:at + 1], *w, gpu(_offsets([1, 0, 0] if at < 150 else [0, 0, 1])))
        assert torch.equal(one[0], all_rows[at])


@pytest.mark.parametrize("T,E,k,H,I", [(1, 8, 2, 256, 128), (5, 64, 8, 512, 256), (100, 16, 4, 384, 384), (700, 8, 2, 256, 128), (1500, 8, 2, 384, 160 * 4)])
def test_a_layer_as_it_is_used(T, E, k, H, I):
    """route -> plan -> quantise and sort -> gate/up -> down -> merge, eagerly and as a captured graph that is replayed on new tokens."""
    rng = np.random.default_rng([T, E])
    w1 = moe.mx_quantize(torch.from_numpy(rng.standard_normal((E, 2 * I, H), dtype=np.float32) * H ** -0.5).to(torch.bfloat16).cuda())
    w2 = moe.mx_quantize(torch.from_numpy(rng.standard_normal((E, H, I), dtype=np.float32) * I ** -0.5).to(torch.bfloat16).cuda())
    plan = [torch.full((n,), -1, dtype=torch.int32, device="cuda") for n in (E, E + 1, T * k, T * k)]
    x = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    z = torch.empty(T, E, device="cuda")

    def layer():
        ids, wt = moe.route(z, k)
        moe.moe_plan_static(ids.data_ptr(), T, k, E, *(o.data_ptr() for o in plan), torch.cuda.current_stream().cuda_stream)
        a = moe.mx_quantize(x, plan[2], plan[3], k)
        h = moe.mx_swiglu(*a, *w1, plan[1])
        d = moe.mx_product(*h, *w2, plan[1])
        return ids, wt, a, h, d, moe.merge_rows(d, plan[3], wt)

    def fill(seed):
        r = np.random.default_rng(seed)
        x.copy_(torch.from_numpy(r.standard_normal((T, H), dtype=np.float32)).to(torch.bfloat16))
        z.copy_(torch.from_numpy(r.standard_normal((T, E), dtype=np.float32)))

    def check(out):
        ids, wt, a, h, d, y = (tuple(t.cpu() for t in o) if isinstance(o, tuple) else o.cpu() for o in out)
        flat = ids.numpy().reshape(-1)
        order = np.argsort(flat, kind="stable")
        off = _offsets(np.bincount(flat, minlength=E))
        xq = quantised(x.cpu().double().numpy())[order // k]
        assert np.array_equal(values_of(*a), xq)
        W1, W2 = values_of(w1[0].cpu(), w1[1].cpu()), values_of(w2[0].cpu(), w2[1].cpu())
        p, m = _product64(xq, W1, off, T * k), _product64(np.abs(xq), np.abs(W1), off, T * k)
        g, u, dg, du = p[:, :I], p[:, I:], H * 2.0 ** -23 * m[:, :I], H * 2.0 ** -23 * m[:, I:]
        # the intermediate: within one code of the 64-bit one where the products' roundings leave a choice
        sig = 1.0 / (1.0 + np.exp(-g))
        act, err = g * sig * u, _swiglu_bounds(g, u)[1]
        slack = err + dg * np.abs(u) * 1.1 + du * np.abs(g * sig)          # |silu'| <= 1.1
        hv = values_of(*h)
        s = np.repeat(np.ldexp(1.0, h[1].numpy().astype(np.int64) - 127), 32, axis=-1)
        assert np.all(np.abs(hv) / s >= round_to_grid(np.maximum(np.abs(act) - slack, 0) / s))
        assert np.all(np.abs(hv) / s <= round_to_grid((np.abs(act) + slack) / s))
        dref, dmag = _product64(hv, W2, off, T * k), _product64(np.abs(hv), np.abs(W2), off, T * k)
        assert np.all(np.abs(d.double().numpy() - dref) <= half_step(torch.bfloat16) * np.abs(dref) + 2 * I * 2.0 ** -23 * dmag)
        f2s = np.argsort(order)
        terms = d.double().numpy()[f2s].reshape(T, k, H) * wt.double().numpy()[..., None]
        ref, mag = terms.sum(1), np.abs(terms).sum(1)
        assert np.all(np.abs(y.double().numpy() - ref) <= half_step(torch.bfloat16) * np.abs(ref) + 2 * k * EPS_FP32 * mag)

    fill(1)
    check(layer())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = layer()
    for seed in (2, 3):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        check(out)


@pytest.mark.parametrize("counts", [[100, 20, 0, 180], [900, 20, 0, 380]], ids=["low tiles", "high tiles"])
def test_two_streams_at_once(counts):
    """Products on two streams share nothing: both are what they are alone."""
    K, N = 512, 512
    a = [gpu(*_exact_operand((sum(counts),), K, s), *_exact_operand((4, N), K, s + 1), _offsets(counts)) for s in (20, 30)]
    both = lambda v, s=None: (moe.mx_product(*v, stream=s), *moe.mx_swiglu(*v, stream=s))
    want = [both(v) for v in a]
    streams = [torch.cuda.Stream() for _ in a]
    torch.cuda.synchronize()
    got = [[both(v, s) for v, s in zip(a, streams)] for _ in range(10)]
    torch.cuda.synchronize()
    for pair in got:
        for x, y in zip(pair, want):
            assert all(torch.equal(p, q) for p, q in zip(x, y))


@pytest.mark.parametrize("K", [128, 256, 384, 768, 1024])
@pytest.mark.parametrize("shift", [4, 8])
def test_scales_that_are_aligned_to_words_only(K, shift):
    counts, N = [50, 0, 300], 200
    R = sum(counts)
    x, w = _exact_operand((R,), K, 41), _exact_operand((3, N), K, 42)
    off = _offsets(counts)
    def moved(t):
        buf = torch.full((t.numel() + shift,), 255, dtype=torch.uint8, device="cuda")
        buf[shift:] = t.reshape(-1)
        return buf[shift:].view(t.shape)
    dx, dxs, dw, dws, doff = gpu(*x, *w, off)
    ref = _bf16(_product64(values_of(*x), values_of(*w), off, R))
    assert torch.equal(moe.mx_product(dx, moved(dxs), dw, moved(dws), doff).cpu(), ref)
    assert torch.equal(moe.mx_product(dx, dxs, dw, moved(dws), doff).cpu(), ref)


def test_weights_past_four_gigabytes():
    """Addresses of codes and scales beyond 32 bits."""
    E, N, K = 9, 1 << 18, 4096                                      # 4.8 GB of codes, 0.3 GB of scales
    codes = torch.zeros(E, N, K // 2, dtype=torch.uint8, device="cuda")
    scales = torch.full((E, N, K // 32), 127, dtype=torch.uint8, device="cuda")
    codes[8, N - 3:] = 0x22                                         # ones
    scales[8, N - 1] = 128
    x = torch.full((2, K // 2), 0x22, dtype=torch.uint8, device="cuda")
    xs = torch.full((2, K // 32), 127, dtype=torch.uint8, device="cuda")
    out = moe.mx_product(x, xs, codes, scales, gpu(_offsets([1] + [0] * 7 + [1])))
    assert (out[0] == 0).all() and (out[1, :N - 3] == 0).all()
    assert out[1, N - 3:].tolist() == [K, K, 2 * K]


def test_results_past_four_giga_elements():
    """Sorted codes of more than 2^32 bytes; products of more than 2^32 outputs, stored both ways (rows aligned to 16 bytes, and not)."""
    T, k, K = 1 << 17, 8, 8448
    ids, w, offsets, s2f, f2s = routing(T, 16, k, 3)
    ds2f, df2s = gpu(s2f, f2s)
    x = torch.randn(T, K, device="cuda").to(torch.bfloat16)
    codes, scales = moe.mx_quantize(x, ds2f, df2s, k)
    c0, s0 = moe.mx_quantize(x)
    token = (ds2f // k).long()
    for at in (0, K // 4 + 3, K // 2 - 1):
        assert torch.equal(codes[:, at], c0[token, at])
    for at in (0, K // 32 - 1):
        assert torch.equal(scales[:, at], s0[token, at])
    R = T * k
    rows, rows_scales = codes[:, :64].contiguous(), torch.full((R, 4), 127, dtype=torch.uint8, device="cuda")
    del codes, scales, c0, s0, x
    for N in (4104, 4101):
        wc, ws = _exact_operand((2, N), 128, 5)
        out = moe.mx_product(rows, rows_scales, *gpu(wc, ws), gpu(np.array([0, R // 2 + 5, R], np.int32)))
        at = np.array([0, 1, R // 2 + 4, R // 2 + 5, R - 2, R - 1])
        xv, wv = values_of(rows[at].cpu(), rows_scales[at].cpu()), values_of(wc, ws)
        ref = np.stack([xv[i] @ wv[0 if at[i] < R // 2 + 5 else 1].T for i in range(len(at))])
        assert torch.equal(out[at].cpu(), _bf16(ref))
        whole = torch.cat([out[: 1 << 16], out[-(1 << 16):]])
        near = torch.cat([moe.mx_product(rows[: 1 << 16], rows_scales[: 1 << 16], *gpu(wc, ws), gpu(np.array([0, 1 << 16, 1 << 16], np.int32))),
                          moe.mx_product(rows[-(1 << 16):], rows_scales[-(1 << 16):], *gpu(wc, ws), gpu(np.array([0, 0, 1 << 16], np.int32)))])
        assert torch.equal(whole, near)
        del out, whole, near


def test_empty_batches():
    x = torch.empty(0, 128, dtype=torch.bfloat16, device="cuda")
    codes, scales = moe.mx_quantize(x)
    assert codes.shape == (0, 64) and scales.shape == (0, 4) and moe.mx_dequantize(codes, scales).shape == (0, 128)
    w = gpu(*_exact_operand((2, 64), 128, 1))
    off = gpu(np.zeros(3, np.int32))
    assert moe.mx_product(codes, scales, *w, off).shape == (0, 64)
    a, b = moe.mx_swiglu(codes, scales, *w, off)
    assert a.shape == (0, 16) and b.shape == (0, 1)
