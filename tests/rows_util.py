"""Shared by the tests of sorted rows and 4-bit experts: routings, and evaluations in 64 bits on the CPU that share no code with the library."""
import numpy as np
import torch

EPS_FP32 = 2.0 ** -24
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def half_step(dtype):
    """Largest relative error of one rounding to dtype."""
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """Largest error of one rounding below the normal numbers."""
    return torch.finfo(dtype).tiny * torch.finfo(dtype).eps / 2


def routing(T, E, k, seed, rejected=0):
    """ids [T, k] int32 (some replaced by -1), w [T, k], offsets [E + 1], s2f, f2s [T k] as the plan defines them."""
    rng = np.random.default_rng([seed, T, E, k])
    ids = np.argsort(rng.random((T, E)), axis=1)[:, :k].astype(np.int32)
    if rejected:
        flat = ids.reshape(-1)
        flat[rng.choice(flat.size, min(rejected, flat.size), replace=False)] = -1
    w = rng.random((T, k)).astype(np.float32) + 0.1
    w /= w.sum(1, keepdims=True)
    return ids, w, *plan(ids, E)


def plan(ids, E):
    flat = ids.reshape(-1)
    on = np.nonzero(flat >= 0)[0]
    order = on[np.argsort(flat[on], kind="stable")]
    s2f = np.full(flat.size, -1, np.int32)
    f2s = np.full(flat.size, -1, np.int32)
    s2f[:order.size] = order
    f2s[order] = np.arange(order.size)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[on], minlength=E))]).astype(np.int32)
    return offsets, s2f, f2s


def gpu(*arrays):
    out = tuple(torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays)
    return out[0] if len(out) == 1 else out


def values_of(codes, scales):
    """Codes [..., K/2] and scale bytes [..., K/32] -> fp64 values [..., K]."""
    codes, scales = np.asarray(codes, np.uint8), np.asarray(scales, np.int64)
    nib = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = GRID[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    with np.errstate(invalid="ignore"):
        s = np.where(scales == 255, np.nan, np.ldexp(1.0, np.where(scales == 255, 0, scales) - 127))
        return v * np.repeat(s, 32, axis=-1)


def scale_bytes(x):
    """fp64 [..., K] -> scale bytes [..., K/32] of the format's definition."""
    top = np.abs(x).reshape(*x.shape[:-1], -1, 32).max(-1)
    bad = ~np.isfinite(top)
    _, e = np.frexp(np.where(bad, 1.0, top))              # top = m 2^e, m in [0.5, 1): floor(log2 top) = e - 1
    return np.where(bad, 255, np.where(top == 0, 0, np.maximum(e - 1 - 2 + 127, 0)))


def round_to_grid(y):
    """Nearest grid value of fp64 magnitudes y, ties to the even index, saturating."""
    mid = 0.5 * (GRID[1:] + GRID[:-1])
    up = np.searchsorted(mid, y, side="left")             # midpoints below y
    tie = (up < 7) & (y == mid[np.minimum(up, 6)])
    return GRID[np.where(tie & (up % 2 == 1), up + 1, up)]


def quantised(x, bytes_=None):
    """fp64 [..., K] -> the values that the format stores for it."""
    b = scale_bytes(x) if bytes_ is None else bytes_
    s = np.repeat(np.ldexp(1.0, np.where(b == 255, 0, b) - 127), 32, axis=-1)
    with np.errstate(invalid="ignore"):
        v = np.copysign(round_to_grid(np.abs(x) / s), x) * s
        return np.where(np.repeat(b == 255, 32, axis=-1), np.nan, v)
