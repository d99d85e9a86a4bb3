"""Routers by scores: the choice as 64 bits decide it, the weights and their gradient."""
import numpy as np
import pytest
import torch

import paper_2607_18002_b200 as moe
from tests import scaled_util as su

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _logits(T, E, seed, dtype="fp32", sigma=1.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, E, generator=g) * sigma).to(DT[dtype]).cuda()


def _check(z, k, kind="sigmoid", bias=None, groups=1, top_groups=1, group_sum=2, renormalize=True, scale=1.0):
    ids, w = moe.choose_experts(z, k, scores=kind, bias=bias, groups=groups, top_groups=top_groups, group_sum=group_sum, renormalize=renormalize, scale=scale)
    z64 = su.to_numpy(z)
    want = su.chosen(z64, k, kind, None if bias is None else bias.cpu().numpy(), groups, top_groups, group_sum)
    assert np.array_equal(ids.cpu().numpy(), want)
    ref = su.weights_of(z64, want, kind, renormalize, scale)
    err = np.abs(su.to_numpy(w) - ref)
    assert np.all(err <= su.weights_error(z64, want, kind) * np.abs(ref) + abs(scale) * 2.0 ** -120), err.max()
    return ids, w


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T,E,k,groups,top_groups,dtype", [
    (1, 1, 1, 1, 1, "fp32"), (1, 256, 8, 8, 4, "fp32"), (9, 5, 5, 1, 1, "bf16"), (8, 40, 5, 4, 2, "fp16"), (777, 40, 5, 1, 1, "fp32"),
    (333, 256, 8, 8, 3, "bf16"), (65, 257, 7, 1, 1, "fp32"), (64, 264, 32, 8, 2, "fp32"), (130, 1024, 32, 32, 1, "fp32"), (77, 1000, 9, 5, 4, "bf16"),
    (50, 12, 2, 12, 3, "fp32"), (513, 64, 6, 2, 1, "fp32"), (31, 96, 4, 3, 2, "fp16"), (4099, 160, 6, 8, 3, "fp32")])
def test_choice_and_weights(kind, T, E, k, groups, top_groups, dtype):
    z = _logits(T, E, T + E, dtype)
    bias = torch.randn(E, generator=torch.Generator().manual_seed(E)).cuda() * 0.1
    for b in (None, bias):
        for group_sum in (1, 2) if groups > 1 else (2,):
            _check(z, k, kind, b, groups, top_groups, group_sum, renormalize=group_sum == 2, scale=2.5 if b is None else 1.0)
    _check(z, k, kind, bias, groups, top_groups, renormalize=False, scale=0.5)


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,k,groups,top_groups", [(256, 8, 1, 1), (64, 6, 8, 3), (257, 32, 1, 1), (1024, 20, 4, 2)])
def test_values_that_fp32_cannot_tell_apart(kind, E, k, groups, top_groups):
    """A bias that makes all sums equal but for the rounding of the bias itself: the order is that of errors of 2^-25."""
    T = 40
    z = _logits(T, E, 3)
    bias = torch.from_numpy((0.75 - su.scores_of(su.to_numpy(z[:1]), kind)[0]).astype(np.float32)).cuda()
    z = z[:1] + 0 * z                       # every token the same,
    z[T // 2:] = _logits(T - T // 2, E, 4)  # and others that are not close
    _check(z.contiguous(), k, kind, bias, groups, top_groups)


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("bias", [None, 0.0, 0.25])
def test_ties_go_to_the_lower_index(kind, bias):
    b = None if bias is None else torch.full((64,), bias, device="cuda")
    for dtype in DT:
        z = torch.round(_logits(200, 64, 5, dtype).float() * 2).to(DT[dtype]) / 2        # some dozen different values
        for groups, top in ((1, 1), (8, 3), (16, 16)):
            _check(z, 8, kind, b, groups, top)
        _check(torch.zeros_like(z), 8, kind, b, 8, 2)


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
def test_padded_tokens_between_others(kind):
    """Rows of equal logits (and of nothing but -inf) among others, for k up to 32, with and without a bias and groups."""
    for E in (40, 64, 256, 300, 1024):
        z = _logits(50, E, 6)
        z[::3] = 0.0
        z[1::9] = -2.5
        z[4::9] = -float("inf")
        z[7, :] = 1.0; z[7, E - 1] = 1.0 + 2.0 ** -23
        z[10, :] = 1.0; z[10, 3] = 1.0 - 2.0 ** -24
        bias = 0.1 * torch.randn(E, device="cuda", generator=torch.Generator("cuda").manual_seed(E))
        for b in (None, bias, torch.zeros_like(bias), torch.full_like(bias, 0.3)):
            for k in (1, 8, 31, 32):
                _check(z, k, kind, b)
            _check(z, 8, kind, b, 4, 2)
            _check(z, 2, kind, b, 10 if E % 10 == 0 else 32 if E % 32 == 0 else 1, 1)


def test_signed_zeros_are_equal():
    z = torch.zeros(3, 8, device="cuda")
    z[:, ::2] = -0.0
    assert moe.choose_experts(z, 4)[0].tolist() == [[0, 1, 2, 3]] * 3


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_masked_experts_and_rows_without_any(kind, renormalize):
    z = _logits(6, 40, 7)
    z[0] = -float("inf")                                   # nothing left
    z[1, :] = -float("inf"); z[1, 33] = 0.5                # one left
    z[2, 3:] = -float("inf")                               # fewer than k
    z[3, ::2] = torch.finfo(torch.float32).min             # the lowest number instead
    bias = 0.1 * torch.randn(40, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    closed = bias.clone(); closed[::2] = -float("inf")
    for b in (None, bias, closed):
        ids, w = _check(z, 5, kind, b, 8, 8, renormalize=renormalize)
        assert (w[0] == 0).all() and (w[1][ids[1] != 33] == 0).all()
    d = torch.randn(6, 5, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    dz = moe.choose_experts_grad(z, ids, d, scores=kind, renormalize=renormalize)
    assert torch.isfinite(dz).all() and (dz[0] == 0).all()


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
def test_scores_that_are_tiny_alike_have_weights(kind):
    z = _logits(20, 64, 8) - 300.0
    ids, w = _check(z, 6, kind)
    assert torch.allclose(w.sum(1), torch.ones(20, device="cuda"), atol=1e-5)


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("scale_of", [30.0, 3e3, 3e38])
def test_wide_logits(kind, scale_of):
    z = (torch.rand(64, 48, generator=torch.Generator().manual_seed(9)) * 2 - 1).cuda() * scale_of
    _check(z, 6, kind)
    _check(z, 6, kind, renormalize=False)


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
def test_nan_and_infinite_logits_give_ids_in_range(kind):
    z = _logits(5, 64, 10)
    z[0, 7] = float("nan"); z[1] = float("nan"); z[2, 5] = float("inf")
    bias = torch.zeros(64, device="cuda")
    for b, groups in ((None, 1), (bias, 1), (bias, 8)):
        ids, w = moe.choose_experts(z, 6, scores=kind, bias=b, groups=groups, top_groups=min(groups, 4))
        assert ((ids >= 0) & (ids < 64)).all()
        assert all(len(set(r)) == 6 for r in ids.tolist())
        assert torch.isnan(w[0]).any() and torch.isnan(w[1]).all()
        assert torch.isfinite(w[3:]).all()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("E,pad,at", [(64, 4, 0), (64, 3, 1), (40, 8, 4), (257, 1, 0)])
def test_rows_with_strides(dtype, E, pad, at):
    wide = _logits(33, E + pad + at, 11, dtype)
    z = wide[:, at:at + E]
    assert z.stride(0) == E + pad + at
    ids, w = _check(z, 5)
    d = torch.randn(33, 5, device="cuda")
    assert torch.equal(moe.choose_experts_grad(z, ids, d, scores="sigmoid"), moe.choose_experts_grad(z.contiguous(), ids, d, scores="sigmoid"))


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("T,E,k,dtype", [(1, 256, 8, "fp32"), (777, 40, 5, "bf16"), (64, 257, 32, "fp32"), (9, 1024, 6, "fp16"), (3, 1, 1, "fp32"), (4099, 64, 6, "fp32")])
def test_gradient_against_its_formula(kind, renormalize, T, E, k, dtype):
    z = _logits(T, E, T, dtype)
    rng = np.random.default_rng(T)
    d = rng.standard_normal((T, k)).astype(np.float32)
    ids = np.argsort(rng.random((T, E)), 1)[:, :k].astype(np.int32)       # any, not the best alone
    if T > 2:
        ids[0, :] = ids[0, 0]                 # one expert in all slots
        ids[1, 0], ids[2, -1] = -1, E
    dz = moe.choose_experts_grad(z, torch.from_numpy(ids).cuda(), torch.from_numpy(d).cuda(), scores=kind, renormalize=renormalize, scale=2.5)
    assert dz.dtype == z.dtype
    z64 = su.to_numpy(z)
    ref = su.weights_gradient(z64, ids, d.astype(np.float64), kind, renormalize, 2.5)
    # each term is a product of scores and differences; what cancels in them is bounded by the sum of the magnitudes
    s = su.scores_of(z64, kind)
    safe = np.clip(ids, 0, E - 1)
    p = np.take_along_axis(s, safe, 1)
    n = su.weights_of(z64, safe, kind, True, 1.0) if renormalize else p
    size = 2.5 * np.abs(d).max(1, keepdims=True) * k * 2 * (n.max(1, keepdims=True) if renormalize or kind == "sigmoid" else p.max(1, keepdims=True))
    rel = (2 * 44 + 4 * np.abs(z64).max() + 40) * 2.0 ** -24
    bound = rel * size + np.abs(ref) * torch.finfo(z.dtype).eps / 2 + torch.finfo(z.dtype).smallest_normal * torch.finfo(z.dtype).eps
    assert np.all(np.abs(su.to_numpy(dz) - ref) <= bound)
    outside = np.ones((T, E), bool)
    for t in range(T):
        outside[t, [i for i in ids[t] if 0 <= i < E]] = False
    if renormalize or kind == "sigmoid":
        assert (su.to_numpy(dz)[outside] == 0).all()


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_gradient_against_differences(kind, renormalize):
    T, E, k, h = 4, 12, 3, 1e-5
    z = _logits(T, E, 21)
    ids, _ = moe.choose_experts(z, k, scores=kind, renormalize=renormalize, scale=1.5)
    d = torch.randn(T, k, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    dz = su.to_numpy(moe.choose_experts_grad(z, ids, d, scores=kind, renormalize=renormalize, scale=1.5))
    z64, i, d64 = su.to_numpy(z), ids.cpu().numpy(), su.to_numpy(d)
    loss = lambda v: (su.weights_of(v, i, kind, renormalize, 1.5) * d64).sum(1)
    for e in range(E):
        step = np.zeros((T, E)); step[:, e] = h
        diff = (loss(z64 + step) - loss(z64 - step)) / (2 * h)
        # the differences' own error: h^2 / 6 times a third derivative (of products of up to three scores: below 6 sum |d| scale), and 2^-52 / h
        bound = (h * h + 2.0 ** -51 / h) * 6 * 1.5 * np.abs(d64).sum(1) + 200 * 2.0 ** -24 * 1.5 * np.abs(d64).sum(1)
        assert np.all(np.abs(dz[:, e] - diff) <= bound)


def test_agrees_with_route_where_both_say_the_same():
    z = _logits(300, 64, 30)
    ids, w = moe.route(z, 6)
    mine, v = moe.choose_experts(z, 6, scores="softmax")
    assert torch.equal(ids, mine) and torch.allclose(w, v, rtol=1e-6, atol=0)
    d = torch.randn(300, 6, device="cuda")
    assert torch.allclose(moe.route_grad(ids, w, d, 64), moe.choose_experts_grad(z, ids, d), rtol=1e-4, atol=1e-6)


def test_no_tokens_another_stream_and_a_graph():
    z = _logits(50, 64, 31)
    b = torch.zeros(64, device="cuda")
    ids, w = moe.choose_experts(z[:0], 4)
    assert ids.shape == (0, 4) and w.shape == (0, 4)
    assert moe.choose_experts_grad(z[:0], ids, w).shape == (0, 64)
    want = moe.choose_experts(z, 4, scores="sigmoid", bias=b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = moe.choose_experts(z, 4, scores="sigmoid", bias=b, stream=side)
    grad = moe.choose_experts_grad(z, got[0], got[1], scores="sigmoid", stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ids, w = moe.choose_experts(z, 4, scores="sigmoid", bias=b)
        dz = moe.choose_experts_grad(z, ids, w, scores="sigmoid")
    graph.replay()
    assert torch.equal(ids, want[0]) and torch.equal(w, want[1]) and torch.equal(dz, grad)
    z.copy_(_logits(50, 64, 32))
    graph.replay()
    want = moe.choose_experts(z, 4, scores="sigmoid", bias=b)
    assert torch.equal(ids, want[0]) and torch.equal(w, want[1])


@pytest.mark.parametrize("kind", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,groups,top_groups", [(260, 1, 1), (384, 8, 4), (511, 7, 3), (512, 8, 4), (512, 4, 1), (512, 32, 5), (513, 1, 1)])
def test_some_hundred_experts(kind, E, groups, top_groups):
    test_choice_and_weights(kind, 70, E, 8, groups, top_groups, "fp32")
    zero = torch.zeros(E, device="cuda")
    for sigma in (0.0, 1e-3, 40.0):       # equal by their inputs, hardly different, far apart with most scores tiny: more that are close than a warp has lanes
        z = _logits(40, E, E, sigma=sigma)
        _check(z, 8, kind, zero, groups, top_groups)
        _check(z, 8, kind, None, groups, top_groups, group_sum=1)
    for renormalize in (True, False):
        test_gradient_against_its_formula(kind, renormalize, 33, E, 8, "bf16")


def test_sizes_that_do_not_fit_32_bits_are_refused():
    z = torch.zeros(6, 8, device="cuda")
    for bad in (dict(top_k=2, groups=2**32 + 1), dict(top_k=2, groups=2, top_groups=2**32 + 1), dict(top_k=2, group_sum=2**32 + 1), dict(top_k=2**32 + 1)):
        with pytest.raises(ValueError):
            moe.choose_experts(z, **bad)
    z = torch.empty(2**31, 1, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        moe.choose_experts(z, 1)
