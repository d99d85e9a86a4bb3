"""Rows sorted by expert and merged again, their gradients and the router's, against evaluations in 64 bits.

Tolerances count roundings: an output is rounded once (half_step), a sum of k terms in fp32 is off by at most k roundings of the sum
of magnitudes; a dot product over H columns is a chain of at most H/256 + 8 additions per thread, 5 over lanes and 16 over warps."""
import numpy as np
import pytest
import torch

import paper_2607_18002_b200 as moe

from gpu_util import assert_close, bind_ops, make_ctx, weights_to
from workloads import synth

from rows_util import EPS_FP32, gpu, half_step, plan, routing, tiny

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


def _rows(n, H, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(n, H, generator=g).to(dtype)


def _wide(t, pad, shift):
    """The same rows as a view of a wider buffer: row stride H + pad, first element `shift` elements in."""
    n, H = t.shape
    buf = torch.full((n * (H + pad) + shift,), 7.0, dtype=t.dtype, device="cuda")
    v = torch.as_strided(buf, (n, H), (H + pad, 1), shift)
    v.copy_(t)
    return v


def _sorted64(x, s2f, k):
    """fp64 rows by expert; rows of no token are 0."""
    on = s2f >= 0
    return np.where(on[:, None], x[np.where(on, s2f, 0) // k], 0.0)


def _picked(rows, f2s, T, k):
    on = f2s >= 0
    return np.where(on[:, None], rows[np.where(on, f2s, 0)], 0.0).reshape(T, k, -1), on.reshape(T, k)


def _check_all(T, E, k, H, dtype, seed=1, rejected=0, pad=0, shift=0):
    ids, w, offsets, s2f, f2s = routing(T, E, k, seed, rejected)
    ds2f, df2s, dw_ = gpu(s2f, f2s, w)
    eps, small = half_step(dtype), tiny(dtype)
    x, rows, dy = _rows(T, H, dtype, 1), _rows(T * k, H, dtype, 2), _rows(T, H, dtype, 3)
    put = (lambda t: _wide(t, pad, shift)) if pad or shift else (lambda t: t.cuda())
    f64 = lambda t: t.cpu().double().numpy()

    xs = moe.sort_rows(put(x), ds2f, df2s, k)
    assert np.array_equal(f64(xs), _sorted64(f64(x), s2f, k))

    picked, on = _picked(f64(rows), f2s, T, k)
    dx = f64(moe.sort_rows_grad(put(rows), df2s, k))
    ref, mag = picked.sum(1), np.abs(picked).sum(1)
    assert np.all(np.abs(dx - ref) <= eps * np.abs(ref) + (1 + eps) * k * EPS_FP32 * mag + small)

    terms = picked * w.astype(np.float64)[..., None]
    y = f64(moe.merge_rows(put(rows), df2s, dw_))
    ref, mag = terms.sum(1), np.abs(terms).sum(1)
    assert np.all(np.abs(y - ref) <= eps * np.abs(ref) + (1 + eps) * k * EPS_FP32 * mag + small)

    drows, dw = moe.merge_rows_grad(put(dy), put(rows), ds2f, df2s, dw_)
    drows, dw = f64(drows), f64(dw)
    wrow = np.where(s2f >= 0, w.reshape(-1)[np.where(s2f >= 0, s2f, 0)], 0.0).astype(np.float64)
    ref = _sorted64(f64(dy), s2f, k) * wrow[:, None]
    assert np.all(np.abs(drows - ref) <= (eps + 2 * EPS_FP32) * np.abs(ref) + small)
    assert np.all(drows[s2f < 0] == 0)
    prods = picked * f64(dy)[:, None]
    ref, mag = prods.sum(-1), np.abs(prods).sum(-1)
    assert np.all(np.abs(dw - ref) <= (H / 256 + 29) * EPS_FP32 * mag)
    assert np.all(dw[~on] == 0)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("T,E,k,H", [(1, 8, 2, 256), (1, 256, 8, 6144), (3, 5, 5, 1), (37, 40, 5, 1003), (64, 16, 4, 33), (5, 32, 32, 520),
                                     (130, 24, 11, 96), (2, 4, 1, 8), (300, 64, 8, 2048), (17, 12, 9, 7)])
def test_against_64_bits(T, E, k, H, dtype):
    _check_all(T, E, k, H, dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("rejected", [1, 40, 10 ** 6])
def test_rejected_ids(dtype, rejected):
    """Slots without a row contribute nothing, rows without a token are zero -- also where no slot is left."""
    _check_all(33, 8, 3, 264, dtype, rejected=rejected)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("H,pad,shift", [(256, 8, 0), (256, 3, 0), (256, 0, 1), (1003, 5, 2), (512, 512, 8), (40, 4, 4)])
def test_strides_and_alignment(dtype, H, pad, shift):
    _check_all(21, 8, 3, H, dtype, pad=pad, shift=shift)


@pytest.mark.parametrize("H", [1, 2, 5, 16, 48, 6144])
def test_codes_of_one_byte_are_sorted(H):
    T, k = 19, 4
    ids, w, offsets, s2f, f2s = routing(T, 16, k, 3)
    x = torch.randint(0, 256, (T, H), dtype=torch.uint8)
    xs = moe.sort_rows(x.cuda(), *gpu(s2f, f2s), k)
    assert torch.equal(xs.cpu(), x[torch.from_numpy(s2f // k).long()])
    x8 = x.view(torch.float8_e4m3fn)
    xs8 = moe.sort_rows(x8.cuda(), *gpu(s2f, f2s), k)
    assert xs8.dtype == x8.dtype and torch.equal(xs8.view(torch.uint8), xs)


def test_many_rows_take_four_accesses_a_thread():
    _check_all(4096, 64, 4, 2560, torch.bfloat16)


def test_infinities_and_nan_stay_in_their_tokens():
    T, k, H = 12, 3, 264
    ids, w, offsets, s2f, f2s = routing(T, 8, k, 5)
    rows = _rows(T * k, H, torch.float32, 2)
    rows[f2s[4 * k + 1], 5] = float("inf")
    rows[f2s[7 * k], 9] = float("nan")
    y = moe.merge_rows(rows.cuda(), *gpu(f2s, w)).cpu()
    bad = ~torch.isfinite(y)
    assert bad.sum() == 2 and bad[4, 5] and bad[7, 9]
    ids, w, offsets, s2f, f2s = routing(T, 8, k, 5, rejected=6)
    rows = _rows(T * k, H, torch.float32, 4)
    rows[torch.from_numpy(s2f < 0)] = float("nan")                 # rows that no token names are not read
    y = moe.merge_rows(rows.cuda(), *gpu(f2s, w))
    drows, dw = moe.merge_rows_grad(torch.ones(T, H).cuda(), rows.cuda(), *gpu(s2f, f2s, w))
    for t in (y, drows, dw):
        assert torch.isfinite(t).all()


def test_rows_far_into_a_large_buffer():
    """Row strides whose products pass 32 bits."""
    T, k, H = 5, 2, 40
    ids, w, offsets, s2f, f2s = routing(T, 4, k, 8)
    stride = (1 << 29) + 8                                        # 10 rows of 2^29 bf16: 10 GB
    buf = torch.empty((T * k - 1) * stride + H, dtype=torch.bfloat16, device="cuda")
    rows = _rows(T * k, H, torch.bfloat16, 2)
    v = torch.as_strided(buf, (T * k, H), (stride, 1))
    v.copy_(rows)
    near = rows.cuda()
    args = gpu(s2f, f2s, w)
    dy = _rows(T, H, torch.bfloat16, 3).cuda()
    assert torch.equal(moe.merge_rows(v, *args[1:]), moe.merge_rows(near, *args[1:]))
    for a, b in zip(moe.merge_rows_grad(dy, v, *args), moe.merge_rows_grad(dy, near, *args)):
        assert torch.equal(a, b)
    far = torch.as_strided(buf, (T, H), (stride, 1))
    far.copy_(dy)
    assert torch.equal(moe.sort_rows(far, *args[:2], k), moe.sort_rows(dy, *args[:2], k))


def test_results_of_more_than_four_giga_elements():
    """R * H beyond 2^32: every row is where it belongs, checked on the GPU by two columns of every row and by sums."""
    T, k, H, E = 8192, 32, 16512, 64
    ids, w, offsets, s2f, f2s = routing(T, E, k, 6)
    ds2f, df2s, dw = gpu(s2f, f2s, w)
    x = torch.randint(-8, 9, (T, H), device="cuda", dtype=torch.int8).to(torch.bfloat16)
    xs = moe.sort_rows(x, ds2f, df2s, k)
    token = (ds2f // k).long()
    for c in (0, H // 2 + 1, H - 1):
        assert torch.equal(xs[:, c], x[token, c])
    y = moe.merge_rows(xs, df2s, torch.ones_like(dw))              # whole numbers up to 256: exact
    assert torch.equal(y.float(), (k * x.float()))
    assert torch.equal(moe.sort_rows_grad(xs, df2s, k), y)
    drows, dwt = moe.merge_rows_grad(x, xs, ds2f, df2s, torch.ones_like(dw))
    for c in (0, H // 2 + 1, H - 1):
        assert torch.equal(drows[:, c], x[token, c])
    want = (x.float() ** 2).sum(1, keepdim=True).expand(T, k)      # whole numbers below 2^24: exact in any order
    assert torch.equal(dwt, want)


def test_results_do_not_depend_on_the_run():
    T, k, H = 700, 8, 2048
    ids, w, offsets, s2f, f2s = routing(T, 64, k, 9)
    rows, dy = _rows(T * k, H, torch.bfloat16, 2).cuda(), _rows(T, H, torch.bfloat16, 3).cuda()
    args = gpu(s2f, f2s, w)
    first = moe.merge_rows_grad(dy, rows, *args)
    for _ in range(5):
        for a, b in zip(moe.merge_rows_grad(dy, rows, *args), first):
            assert torch.equal(a, b)


# ------------------------------------------------------------------ the router's gradient

def _route_grad64(ids, w, dw, E):
    T, k = ids.shape
    dz, mag = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        on = [j for j in range(k) if 0 <= ids[t, j] < E]
        mean = sum(float(w[t, i]) * float(dw[t, i]) for i in on)
        amean = sum(abs(float(w[t, i]) * float(dw[t, i])) for i in on)
        for j in on:
            dz[t, ids[t, j]] += float(w[t, j]) * (float(dw[t, j]) - mean)
            mag[t, ids[t, j]] += float(w[t, j]) * (abs(float(dw[t, j])) + amean)
    return dz, mag


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 256, 8), (60, 40, 5), (33, 1024, 32), (7, 5, 5), (129, 63, 2), (9, 30, 11)])
def test_router_gradient(T, E, k):
    ids, w, *_ = routing(T, E, k, 11)
    dw = np.random.default_rng(T).standard_normal((T, k)).astype(np.float32)
    got = moe.route_grad(*gpu(ids, w, dw), E).cpu().double().numpy()
    ref, mag = _route_grad64(ids, w, dw, E)
    # w dw, six additions over lanes, a difference, a product
    assert np.all(np.abs(got - ref) <= 10 * EPS_FP32 * mag)
    assert np.all(got[mag == 0] == 0)


def test_router_gradient_of_repeated_and_rejected_ids():
    T, E, k = 50, 9, 6
    rng = np.random.default_rng(4)
    ids = rng.integers(-1, E + 1, (T, k)).astype(np.int32)            # -1 and E name no expert; repeats are many
    w, dw = rng.random((T, k)).astype(np.float32), rng.standard_normal((T, k)).astype(np.float32)
    got = moe.route_grad(*gpu(ids, w, dw), E).cpu().double().numpy()
    ref, mag = _route_grad64(ids, w, dw, E)
    assert np.all(np.abs(got - ref) <= (10 + k) * EPS_FP32 * mag)
    assert np.all(got[mag == 0] == 0)


def test_gradients_against_differences():
    """A loss through router, sort and merge, differentiated by differences of a 64-bit evaluation.

    Central differences with step h of a smooth loss are off by O(h^2) of its third derivatives and by the roundings of the loss over h; both
    are measured here by a second step twice as large: the two estimates differ by three quarters of the h^2 part."""
    T, E, k, H = 6, 8, 3, 16
    rng = np.random.default_rng(21)
    z, x, scale = rng.standard_normal((T, E)), rng.standard_normal((T, H)), rng.standard_normal((E, H))
    target = rng.standard_normal((T, H))
    z32, x32 = z.astype(np.float32), x.astype(np.float32)
    ids, w = moe.route(gpu(z32), k)
    hids = ids.cpu().numpy()
    offsets, s2f, f2s = plan(hids, E)
    expert = np.repeat(np.arange(E), np.diff(offsets))
    s = gpu(scale[expert].astype(np.float32))
    xs = moe.sort_rows(gpu(x32), *gpu(s2f, f2s), k)
    rows = xs * s                                                     # the "experts": a scale per column
    y = moe.merge_rows(rows, gpu(f2s), w)
    dy = y - gpu(target.astype(np.float32))
    drows, dw = moe.merge_rows_grad(dy, rows, *gpu(s2f, f2s), w)
    dx = moe.sort_rows_grad(drows * s, gpu(f2s), k).cpu().double().numpy()
    dz = moe.route_grad(ids, w, dw, E).cpu().double().numpy()

    def loss(zz, xx):
        total = 0.0
        for t in range(T):
            e = hids[t]
            p = np.exp(zz[t, e] - zz[t, e].max())
            p /= p.sum()
            total += 0.5 * np.sum(((p[:, None] * scale[e] * xx[t]).sum(0) - target[t]) ** 2)
        return total

    def differences(which, h):
        out = np.zeros((z if which == 0 else x).shape)
        for i in np.ndindex(*out.shape):
            d = np.zeros(out.shape)
            d[i] = h
            hi = loss(z + d, x) if which == 0 else loss(z, x + d)
            lo = loss(z - d, x) if which == 0 else loss(z, x - d)
            out[i] = (hi - lo) / (2 * h)
        return out

    for which, got in ((0, dz), (1, dx)):
        fine, coarse = differences(which, 1e-4), differences(which, 2e-4)
        # fp32 inputs, a dozen roundings on the way, sums of k (dx) and H (dw) terms
        tol = 2 * np.abs(fine - coarse) + 200 * EPS_FP32 * (np.abs(fine).max() + 1)
        assert np.all(np.abs(got - fine) <= tol)


# ------------------------------------------------------------------ as a program uses them

def test_with_the_librarys_own_route_and_plan():
    """route -> plan -> sort -> merge on the device, with experts that do nothing: every token comes back."""
    T, E, k, H = 200, 16, 4, 512
    z = torch.from_numpy(np.random.default_rng(12).standard_normal((T, E), dtype=np.float32)).cuda()
    ids, w = moe.route(z, k)
    outs = [torch.full((n,), -1, dtype=torch.int32, device="cuda") for n in (E, E + 1, T * k, T * k)]
    moe.moe_plan_static(ids.data_ptr(), T, k, E, *(o.data_ptr() for o in outs), torch.cuda.current_stream().cuda_stream)
    counts, offsets, s2f, f2s = outs
    x = _rows(T, H, torch.bfloat16, 1).cuda()
    xs = moe.sort_rows(x, s2f, f2s, k)
    hids = ids.cpu().numpy()
    order = np.argsort(hids.reshape(-1), kind="stable")
    assert torch.equal(xs.cpu(), x.cpu()[torch.from_numpy(order // k)])
    y = moe.merge_rows(xs, f2s, w)
    err = (y.double() - x.double()).abs()
    assert (err <= (half_step(torch.bfloat16) + (k + 8) * EPS_FP32) * x.double().abs() + tiny(torch.bfloat16)).all()


def test_a_contexts_plan_with_experts_of_the_callers_own():
    """The permutation of moe_plan serves both: experts computed here between sort and merge give what moe_run gives."""
    spec = synth.Spec("rows", synth.Shape(8, 2, 512, 256), ((synth.PREFILL, 150),), "zipf", 1.0, 1.0, -1.0, 61)
    W, (op,) = synth.make_weights(spec), synth.make_ops(spec)
    ctx, Wd = make_ctx(spec), weights_to(W)
    (b,) = bind_ops(ctx, [op], Wd)
    ctx.plan(0, b)
    ctx.run([0], fuse_combine=True)
    ctx.check()
    xs = moe.sort_rows(b.x, b.sorted_to_flat, b.flat_to_sorted, 2).float()
    o = b.offsets.tolist()
    rows = torch.empty(300, 512, dtype=torch.bfloat16, device="cuda")
    for e in range(8):
        h = xs[o[e]:o[e + 1]] @ Wd.w_gate_up[e].float().T
        a = (torch.nn.functional.silu(h[:, :256]) * h[:, 256:]).to(torch.bfloat16).float()
        rows[o[e]:o[e + 1]] = (a @ Wd.w_down[e].float().T).to(torch.bfloat16)
    y = moe.merge_rows(rows, b.flat_to_sorted, b.topk_w)
    assert_close(b.y.float().cpu().numpy(), y.float().cpu().numpy())


def test_streams_graphs_and_several_batches():
    """Captured once, replayed on new inputs in the same buffers; two captured steps share nothing; direct calls on another stream."""
    T, k, H = 90, 4, 640
    side = torch.cuda.Stream()
    cases = []
    for seed in (1, 2):
        ids, w, offsets, s2f, f2s = routing(T, 16, k, seed)
        cases.append(dict(s2f=gpu(s2f), f2s=gpu(f2s), w=gpu(w), x=_rows(T, H, torch.bfloat16, seed).cuda(), dy=_rows(T, H, torch.bfloat16, 9 + seed).cuda()))

    def step(c):
        xs = moe.sort_rows(c["x"], c["s2f"], c["f2s"], k)
        y = moe.merge_rows(xs, c["f2s"], c["w"])
        drows, dw = moe.merge_rows_grad(c["dy"], xs, c["s2f"], c["f2s"], c["w"])
        return xs, y, drows, dw, moe.sort_rows_grad(drows, c["f2s"], k)

    want = [[t.clone() for t in step(c)] for c in cases]
    graphs, outs = [], []
    for c in cases:
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(step(c))
        graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for o, ref in zip(outs, want):
            for a, b in zip(o, ref):
                assert torch.equal(a, b)
    fresh = _rows(T, H, torch.bfloat16, 77).cuda()
    cases[0]["x"].copy_(fresh)
    graphs[0].replay()
    assert torch.equal(outs[0][0], moe.sort_rows(fresh, cases[0]["s2f"], cases[0]["f2s"], k))
    side.wait_stream(torch.cuda.current_stream())
    got = moe.merge_rows(want[1][0], cases[1]["f2s"], cases[1]["w"], stream=side)
    side.synchronize()
    assert torch.equal(got, want[1][1])


def test_empty_batches():
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.empty(0, 4, device="cuda")
    for i in (e, one):
        assert moe.sort_rows(x, i, i, 4).shape == (0, 64)
        assert moe.sort_rows_grad(x, i, 4).shape == (0, 64)
        assert moe.merge_rows(x, i, w).shape == (0, 64)
        drows, dw = moe.merge_rows_grad(x, x, i, i, w)
        assert drows.shape == (0, 64) and dw.shape == (0, 4)
    assert moe.route_grad(torch.empty(0, 4, dtype=torch.int32, device="cuda"), w, w, 8).shape == (0, 8)
