"""Shared by the tests of routers by scores and of e4m3 with block scales: evaluations in 64 bits on the CPU that share no code with the library."""
import numpy as np
import torch

SUBNORMAL = 2.0 ** -9
GRID = np.concatenate([np.arange(8) * SUBNORMAL] + [(8 + np.arange(8)) * 2.0 ** (e - 3) for e in range(-6, 9)])[:127]      # code 0 .. 126
STEP = 2.0 ** -23


def to_numpy(t):
    return t.detach().cpu().double().numpy()


# ------------------------------------------------------------------ routers

def scores_of(z, kind):
    """fp64 [T, E]; a row of nothing above -inf has scores 0."""
    with np.errstate(all="ignore"):
        if kind == "sigmoid":
            return np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))
        top = z.max(1, keepdims=True)
        e = np.exp(z - np.where(np.isneginf(top), 0, top))
        total = e.sum(1, keepdims=True)
        return np.where(total == 0, 0, e / np.where(total == 0, 1, total))


def chosen(z, k, kind, bias=None, groups=1, top_groups=1, group_sum=2):
    """ids [T, k] of the definition, by stable sorts of fp64 values."""
    T, E = z.shape
    c = scores_of(z, kind) + (0 if bias is None else bias.astype(np.float64))
    order = z.copy() if bias is None else c.copy()
    out = np.zeros((T, E), bool)
    if top_groups < groups:
        best = -np.sort(-c.reshape(T, groups, E // groups), axis=2)[:, :, :group_sum].sum(2)
        kept = np.argsort(-best, axis=1, kind="stable")[:, :top_groups]
        out[:] = True
        for t in range(T):
            for g in kept[t]:
                out[t, g * (E // groups):(g + 1) * (E // groups)] = False
    # kept experts first, each kind in order
    return np.stack([np.lexsort((np.arange(E), -order[t], out[t]))[:k] for t in range(T)])


def weights_of(z, ids, kind, renormalize, scale):
    if renormalize:                            # relative to the largest of the chosen
        p = np.take_along_axis(z, ids, 1)
        top = p.max(1, keepdims=True)
        with np.errstate(all="ignore"):
            top = np.where(np.isneginf(top), 0, top)
            shift = np.minimum(top, 0) if kind == "sigmoid" else top
            n = np.exp(p - shift) / (1 + np.exp(p)) if kind == "sigmoid" else np.exp(p - shift)
            n = np.where(p > 0, 1 / (1 + np.exp(-p)), n) if kind == "sigmoid" else n
            total = n.sum(1, keepdims=True)
            return scale * np.where(total == 0, 0, n / np.where(total == 0, 1, total))
    return scale * np.take_along_axis(scores_of(z, kind), ids, 1)


def weights_error(z, ids, kind):
    """Relative bound for fp32 weights, in steps of 2^-24: the argument of exp is off by half a step of its magnitude (z - top, at most the spread of what counts), exp by
    two steps of 2^-23, sums of E or k terms by the lanes' and the shuffles' additions (32 + 5, or 32), three quotients and products; numerator and denominator alike."""
    p = np.take_along_axis(z, ids, 1)
    p, z = np.where(np.isneginf(p), -1e300, p), np.where(np.isneginf(z), -1e300, z)      # (weights of 0: any bound will do)
    spread = np.where(np.isfinite(p), np.abs(p - p.max(1, keepdims=True)), 0) if kind == "softmax" else np.zeros_like(p)
    far = np.where(np.isfinite(p), np.abs(p - z.max(1, keepdims=True)), 0) if kind == "softmax" else np.minimum(np.abs(p), 110)
    return (2 * (4 + 37 + 3) + spread + far + spread.max(1, keepdims=True)) * 2.0 ** -24


def weights_gradient(z, ids, d, kind, renormalize, scale):
    """[T, E] by the formula; ids outside [0, E) are left out."""
    T, E = z.shape
    out = np.zeros((T, E))
    s = scores_of(z, kind)
    for t in range(T):
        on = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < E]
        if not on:
            continue
        i = ids[t, on]
        g = scale * d[t, on]
        if renormalize:
            n = weights_of(z[t:t + 1], i[None], kind, True, 1.0)[0]
            v = n * (g - (n * g).sum())
            if kind == "sigmoid":
                v = v * scores_of(-z[t:t + 1, i], "sigmoid")[0]
            np.add.at(out[t], i, v)
        elif kind == "sigmoid":
            np.add.at(out[t], i, g * s[t, i] * scores_of(-z[t:t + 1, i], "sigmoid")[0])
        else:
            np.add.at(out[t], i, g * s[t, i])
            out[t] -= s[t] * (g * s[t, i]).sum()
    return out


# ------------------------------------------------------------------ e4m3 with block scales

def block_scales(x, rows):
    """fp64 [..., n, K] (fp32 numbers) -> fp32 scales of blocks of `rows` x 128, NaN where a block holds NaN or infinity."""
    n, K = x.shape[-2:]
    pad = [(0, 0)] * (x.ndim - 2) + [(0, -n % rows), (0, -K % 128)]
    b = np.pad(np.abs(x), pad)
    b = b.reshape(*x.shape[:-2], b.shape[-2] // rows, rows, b.shape[-1] // 128, 128)
    top = b.max((-1, -3))
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.maximum(top.astype(np.float32) * (np.float32(1.0) / np.float32(448.0)), np.float32(2.0 ** -126))
    s = np.where(top == 0, np.float32(1), s)
    return np.where(np.isfinite(top), s, np.float32(np.nan)).astype(np.float32)


def spread(s, rows, n, K):
    return np.repeat(np.repeat(s.astype(np.float64), rows, -2)[..., :n, :], 128, -1)[..., :K]


def nearest_code(q):
    """fp64 quotients -> code bytes, ties to the even code, saturating.  (A 24-bit number over another is a midpoint or off by more than fp64 rounds.)"""
    a = np.abs(q)
    mid = 0.5 * (GRID[1:] + GRID[:-1])
    up = np.searchsorted(mid, a, side="left")
    tie = (up < 126) & (a == mid[np.minimum(up, 125)])
    up = np.where(tie & (up % 2 == 1), up + 1, up)
    return (up + 128 * np.signbit(q)).astype(np.uint8)


def code_values(codes):
    codes = np.asarray(codes, np.uint8)
    m = codes & 127
    return np.where(m == 127, np.nan, GRID[np.minimum(m, 126)]) * np.where(codes & 128, -1.0, 1.0)


def values_of(codes, scales, rows):
    codes = np.asarray(codes)
    return code_values(codes) * spread(scales, rows, *codes.shape[-2:])


def bytes_of(t):
    return t.view(torch.uint8).cpu().numpy()


def random_rows(R, K, rng, spread_of=3):
    """Codes and scales of N(0, 1) rows of different magnitudes, as tensors."""
    x = rng.standard_normal((R, K)) * np.exp2(rng.integers(-spread_of, spread_of + 1, (R, 1)))
    x = x.astype(np.float32).astype(np.float64)
    s = block_scales(x, 1)
    return nearest_code(x / spread(s, 1, R, K)), s


def random_weights(E, N, K, rng):
    w = (rng.standard_normal((E, N, K)) * K ** -0.5).astype(np.float32).astype(np.float64)
    s = block_scales(w, 128)
    return nearest_code(w / spread(s, 128, N, K)), s


def on_gpu(codes, scales):
    return torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn), torch.from_numpy(scales).cuda()


def product_of(x, w, offsets):
    """fp64 rows times matrices by expert, and the same of the magnitudes; rows of no expert are 0."""
    out = np.zeros((x.shape[0], w.shape[1]))
    size = np.zeros_like(out)
    for e in range(w.shape[0]):
        r = slice(offsets[e], offsets[e + 1])
        out[r] = x[r] @ w[e].T
        size[r] = np.abs(x[r]) @ np.abs(w[e]).T
    return out, size


def product_error(K, size):
    """fp32 bound: a block's 128 products (exact) are added with a loss of a step of 2^-23 each at most, scaled by a rounded product of scales, and the
    blocks added with half a step each."""
    return (2 * 128 + 2 + -(-K // 128)) * 2.0 ** -24 * size
