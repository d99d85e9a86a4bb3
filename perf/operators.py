"""The operators around the experts of a routed layer: rows sorted by expert and back with their gradients, the router's
gradient, and the experts in 4 bits -- each as a plain evaluation with elementary torch operations and as the calls a
program makes of this library.

A case names its operator (`op`):
  sort        rows of tokens -> rows sorted by expert; with `grad` its gradient too (a training step's two directions)
  merge       sorted rows -> weighted sums per token; with `grad` the gradients of rows and weights too
  route_grad  gradient of the router weights -> gradient of the logits
  quantise    rows -> 4-bit codes and block scales, and back to values
  layer       a layer's experts in 4 bits: quantise and sort, gate/up product with SwiGLU, down product, merge
  product     one product of sorted 4-bit rows with the experts' 4-bit matrices

4-bit values are e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign bit), the even column in a byte's low half, with one
power-of-two scale (exponent + 127 in a byte) per 32 columns: the largest power of two not above the block's largest
magnitude, over 4.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_EL = {"bf16": 2, "fp16": 2, "fp32": 4}


def _case(name, op, T, E=1, k=1, H=0, dtype="bf16", I=0, zipf=0.0, grad=False):
    return dict(name=name, op=op, T=T, E=E, k=k, H=H, dtype=dtype, I=I, zipf=zipf, grad=grad)


def listed():
    return [
        # a decode batch laid out by expert: latency
        _case("sort_decode_16", "sort", 16, 256, 8, 6144),
        # a training chunk's tokens sorted by expert, and the gradient back to the tokens
        _case("sort_train_8192", "sort", 8192, 64, 8, 4096, zipf=1.0, grad=True),
        # one user's token put together from its eight experts
        _case("merge_decode_1", "merge", 1, 256, 8, 6144),
        # an odd-sized chunk of a model whose width is no multiple of anything
        _case("merge_train_777_odd", "merge", 777, 40, 5, 1003, "fp16", zipf=0.8, grad=True),
        # a training chunk put together, and the gradients of its rows and router weights
        _case("merge_train_4096", "merge", 4096, 256, 8, 6144, zipf=1.2, grad=True),
        # the router's gradient for a small and a large chunk
        _case("route_grad_60", "route_grad", 60, 40, 5),
        _case("route_grad_16384", "route_grad", 16384, 256, 8),
        # activations of a decode batch to 4 bits and back
        _case("quantise_129_fp32", "quantise", 129, H=2048, dtype="fp32"),
        # an expert layer's weights to 4 bits and back, as when a checkpoint is loaded
        _case("quantise_weights", "quantise", 64 * 1536, H=2048),
        # one token through eight 4-bit experts
        _case("layer_decode_1", "layer", 1, 64, 8, 2048, I=1024),
        # a decode batch that meets most experts: the weight stream
        _case("layer_decode_100", "layer", 100, 128, 8, 4096, I=1792),
        # a prefill chunk
        _case("layer_prefill_8192", "layer", 8192, 64, 8, 4096, I=1792, zipf=0.6),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["sort", "sort", "merge", "merge", "route_grad", "quantise", "layer", "layer", "product", "product"])
    E, k = rng.choice([(8, 2), (16, 4), (40, 5), (64, 6), (64, 8), (128, 8), (256, 8)])
    zipf = round(rng.uniform(0.0, 1.2), 2)
    if op in ("sort", "merge"):
        H = rng.choice([256, 1000, 2048, 4096, 6144, rng.randrange(33, 6000), rng.randrange(16, 700) * 8])
        most = max(64, min(8192, 200_000_000 // (H * k)))
        return dict(op=op, T=_log_int(rng, 1, most), E=E, k=k, H=H, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), I=0, zipf=zipf,
                    grad=rng.random() < 0.6)
    if op == "route_grad":
        return dict(op=op, T=_log_int(rng, 1, 16384), E=E, k=k, H=0, dtype="fp32", I=0, zipf=zipf, grad=False)
    if op == "quantise":
        H = 128 * _log_int(rng, 2, 64)
        return dict(op=op, T=_log_int(rng, 1, 200_000_000 // H), E=1, k=1, H=H, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), I=0, zipf=0.0,
                    grad=False)
    H, I = 128 * _log_int(rng, 2, 32), 128 * _log_int(rng, 1, 12)
    if op == "product":          # I: the experts' output columns, odd ones too
        I = rng.choice([I, I + rng.randrange(1, 128)])
    return dict(op=op, T=_log_int(rng, 1, 4096), E=min(E, 128), k=k, H=H, dtype="bf16", I=I, zipf=round(zipf / 2, 2), grad=False)


# ------------------------------------------------------------------ inputs

def _routing(c, g, dev):
    """Top-k routing with a Zipf(zipf) popularity over a random expert order, its weights and its plan."""
    T, E, k = c["T"], c["E"], c["k"]
    rank = torch.randperm(E, generator=g, device=dev)
    u = torch.rand(T, E, generator=g, device=dev).clamp_(1e-7, 1.0 - 1e-7)
    z = -c["zipf"] * torch.log((rank + 1).float()) - torch.log(-torch.log(u))
    ids = torch.topk(z, k, dim=1).indices
    w = torch.softmax(torch.randn(T, k, generator=g, device=dev), dim=1)
    flat = ids.reshape(-1)
    s2f = torch.argsort(flat, stable=True)
    f2s = torch.empty_like(s2f)
    f2s[s2f] = torch.arange(T * k, device=dev)
    counts = torch.bincount(flat, minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=dev)
    offsets[1:] = torch.cumsum(counts, 0)
    return dict(ids=ids.int(), w=w, s2f=s2f.int(), f2s=f2s.int(), offsets=offsets, most=int(counts.max()))


def _weights(E, N, K, g, dev):
    """Experts' matrices N(0, 1/K) as 4-bit codes [E, N, K/2] and block scales [E, N, K/32]."""
    codes = torch.empty(E, N, K // 2, dtype=torch.uint8, device=dev)
    scales = torch.empty(E, N, K // 32, dtype=torch.uint8, device=dev)
    for e in range(0, E, 8):
        n = min(8, E - e)
        codes[e:e + n], scales[e:e + n] = _quantise(torch.empty(n, N, K, device=dev).normal_(0.0, K ** -0.5, generator=g))
    return codes, scales


def prepare(case, seed):
    c, dev = case, torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    T, E, k, H, I, dt = c["T"], c["E"], c["k"], c["H"], c["I"], _DT[c["dtype"]]

    def rows(n, w=H):
        return torch.empty(n, w, device=dev).normal_(0.0, 1.0, generator=g).to(dt)

    if c["op"] == "quantise":          # rows of different magnitudes
        x = torch.empty(T, H, device=dev).normal_(0.0, 1.0, generator=g)
        return dict(c=c, x=(x * torch.exp2(torch.randint(-6, 7, (T, 1), generator=g, device=dev).float())).to(dt))
    s = _routing(c, g, dev)
    s["c"] = c
    if c["op"] == "sort":
        s["x"] = rows(T)
        if c["grad"]:
            s["dxs"] = rows(T * k)
    elif c["op"] == "merge":
        s["rows"] = rows(T * k)
        if c["grad"]:
            s["dy"] = rows(T)
    elif c["op"] == "route_grad":
        s["dw"] = torch.empty(T, k, device=dev).normal_(0.0, 1.0, generator=g)
    elif c["op"] == "product":
        s["codes"], s["scales"] = _quantise(rows(T * k).float())
        s["w1"] = _weights(E, I, H, g, dev)
    else:
        s["x"] = rows(T)
        s["w1"] = _weights(E, 2 * I, H, g, dev)
        s["w2"] = _weights(E, H, I, g, dev)
    return s


# ------------------------------------------------------------------ plain forms

def _power(byte):
    """2^(byte - 127) by its bits (2^-127 is a subnormal number)."""
    return torch.where(byte > 0, byte << 23, 0x400000).view(torch.float32)


def _quantise(x):
    """fp32 [..., K] -> codes [..., K/2], scales [..., K/32] (finite values)."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = b.abs().amax(-1)
    byte = ((top.view(torch.int32) >> 23) - 2).clamp_(min=0)         # floor(log2) by the exponent field
    b = b * _power(254 - byte)[..., None]
    a = b.abs()
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte()
            + (a > 5.0).byte())                                       # ties to the even code
    code = (code + 8 * torch.signbit(b).byte()).reshape(*x.shape[:-1], -1, 2)
    return code[..., 0] + 16 * code[..., 1], byte.to(torch.uint8)


def _value_table(dev, dtype):
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=dtype, device=dev)
    v = torch.cat([v, -v])
    return torch.stack([v.repeat(16), v.repeat_interleave(16)], -1)   # byte -> (low half, high half)


def _values(codes, scales):
    """The fp32 values of codes [..., K/2] with scales [..., K/32]."""
    v = _value_table(codes.device, torch.float32)[codes.int()].reshape(*scales.shape, 32)
    return (v * _power(scales.int())[..., None]).reshape(*codes.shape[:-1], -1)


def _grouped(x, w, offsets, most):
    """x [R, K] sorted by expert times w [E, N, K]: every expert's rows in a slab of the largest expert's height."""
    R, at = x.shape[0], torch.arange(most, device=x.device)
    index = offsets[:-1, None].long() + at
    slab = x[index.clamp(max=R - 1)]
    y = torch.bmm(slab, w.transpose(1, 2))
    return y[at < (offsets[1:] - offsets[:-1]).long()[:, None]]


def _plain(s):
    c = s["c"]
    op, k = c["op"], c["k"]
    if op == "sort":
        out = dict(xs=s["x"][s["s2f"] // k])
        if c["grad"]:
            out["dx"] = s["dxs"][s["f2s"]].float().reshape(c["T"], k, -1).sum(1).to(s["x"].dtype)
        return out
    if op == "merge":
        picked = s["rows"][s["f2s"]].float().reshape(c["T"], k, -1)
        out = dict(y=(picked * s["w"][..., None]).sum(1).to(s["rows"].dtype))
        if c["grad"]:
            dy = s["dy"].float()
            out["dw"] = (picked * dy[:, None]).sum(-1)
            drows = (s["w"][..., None] * dy[:, None]).reshape(c["T"] * k, -1)
            out["drows"] = drows[s["s2f"]].to(s["rows"].dtype)
        return out
    if op == "route_grad":
        w, dw = s["w"], s["dw"]
        dz = w * (dw - (w * dw).sum(1, keepdim=True))
        return torch.zeros(c["T"], c["E"], device=w.device).scatter_add_(1, s["ids"].long(), dz)
    if op == "quantise":
        return _values(*_quantise(s["x"].float())).to(s["x"].dtype)
    if op == "product":
        return _grouped(_values(s["codes"], s["scales"]), _values(*s["w1"]), s["offsets"], s["most"]).to(torch.bfloat16)
    x = _values(*_quantise(s["x"].float()))[s["s2f"] // k]
    h = _grouped(x, _values(*s["w1"]), s["offsets"], s["most"])
    g, u = h[:, :c["I"]], h[:, c["I"]:]
    a = _values(*_quantise(g / (1.0 + torch.exp(-g)) * u))
    d = _grouped(a, _values(*s["w2"]), s["offsets"], s["most"])
    return (d[s["f2s"]].reshape(c["T"], k, -1) * s["w"][..., None]).sum(1).to(torch.bfloat16)


# ------------------------------------------------------------------ the library's calls

def _library(s):
    import paper_2607_18002_b200 as moe
    c = s["c"]
    op, k = c["op"], c["k"]
    if op == "sort":
        out = dict(xs=moe.sort_rows(s["x"], s["s2f"], s["f2s"], k))
        if c["grad"]:
            out["dx"] = moe.sort_rows_grad(s["dxs"], s["f2s"], k)
        return out
    if op == "merge":
        out = dict(y=moe.merge_rows(s["rows"], s["f2s"], s["w"]))
        if c["grad"]:
            out["drows"], out["dw"] = moe.merge_rows_grad(s["dy"], s["rows"], s["s2f"], s["f2s"], s["w"])
        return out
    if op == "route_grad":
        return moe.route_grad(s["ids"], s["w"], s["dw"], c["E"])
    if op == "quantise":
        return moe.mx_dequantize(*moe.mx_quantize(s["x"]), s["x"].dtype)
    if op == "product":
        return moe.mx_product(s["codes"], s["scales"], *s["w1"], s["offsets"])
    x = moe.mx_quantize(s["x"], s["s2f"], s["f2s"], k)
    a = moe.mx_swiglu(*x, *s["w1"], s["offsets"])
    d = moe.mx_product(*a, *s["w2"], s["offsets"])
    return moe.merge_rows(d, s["f2s"], s["w"])


def run(state):
    return _library(state) if own else _plain(state)


# ------------------------------------------------------------------ the definitions in 64 bits

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest(x):
    """fp64 [..., K]: every value replaced by the nearest multiple of its block's scale that 4 bits can hold."""
    b = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(b.abs().amax(-1, keepdim=True))               # amax = m 2^e, m in [0.5, 1)
    scale = torch.where(m > 0, _two_to((e - 3).clamp(min=-127)), torch.ones_like(m))
    a = (b / scale).abs()
    best = torch.zeros_like(a)
    for i in range(1, 8):                                             # a midpoint goes to the entry of even index
        mid = 0.5 * (_GRID[i - 1] + _GRID[i])
        best = torch.where((a > mid) | ((a == mid) & (i % 2 == 0)), torch.full_like(a, _GRID[i]), best)
    return (torch.copysign(best, b) * scale).flatten(-2)


def _decode(codes, scales):
    grid = torch.tensor(_GRID, dtype=torch.float64, device=codes.device)
    halves = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    v = grid[halves & 7] * (1.0 - 2.0 * (halves >> 3).double())
    return (v.unflatten(-1, (-1, 32)) * _two_to(scales.long() - 127)[..., None]).flatten(-2)


def _by_expert(x, w, offsets):
    """One expert after the other; w: codes and scales."""
    out, o = [], offsets.tolist()
    for e in range(len(o) - 1):
        if o[e + 1] > o[e]:
            out.append(x[o[e]:o[e + 1]] @ _decode(w[0][e], w[1][e]).T)
    return torch.cat(out)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    op, T, k = c["op"], c["T"], c["k"]
    if op == "quantise":
        return _nearest(s["x"].double())
    token = torch.div(s["s2f"].long(), k, rounding_mode="floor")
    f2s, w = s["f2s"].long(), s["w"].double()
    if op == "sort":
        out = dict(xs=torch.index_select(s["x"], 0, token).double())
        if c["grad"]:
            out["dx"] = torch.zeros(T, c["H"], dtype=torch.float64, device=w.device).index_add_(0, token, s["dxs"].double())
        return out
    if op == "merge":
        rows, wrow = s["rows"].double(), w.reshape(-1)[s["s2f"].long()]
        out = dict(y=torch.zeros(T, c["H"], dtype=torch.float64, device=w.device).index_add_(0, token, rows * wrow[:, None]))
        if c["grad"]:
            dyr = torch.index_select(s["dy"], 0, token).double()
            out["drows"] = dyr * wrow[:, None]
            out["dw"] = torch.einsum("rh,rh->r", dyr, rows)[f2s].reshape(T, k)
        return out
    if op == "route_grad":
        jac = torch.diag_embed(w) - w[:, :, None] * w[:, None, :]
        dz = torch.einsum("tij,tj->ti", jac, s["dw"].double())
        return torch.zeros(T, c["E"], dtype=torch.float64, device=w.device).scatter_add_(1, s["ids"].long(), dz)
    if op == "product":
        return _by_expert(_decode(s["codes"], s["scales"]), s["w1"], s["offsets"])
    h = _by_expert(torch.index_select(_nearest(s["x"].double()), 0, token), s["w1"], s["offsets"])
    g, u = h.split(c["I"], dim=1)
    d = _by_expert(_nearest(g * torch.sigmoid(g) * u), s["w2"], s["offsets"])
    return torch.zeros(T, c["H"], dtype=torch.float64, device=w.device).index_add_(0, token, d * w.reshape(-1)[s["s2f"].long()][:, None])


# ------------------------------------------------------------------ what a pass cannot do without

def _active(c):
    """Expected number of experts that T tokens meet, each choosing k without replacement."""
    E, k, T = c["E"], c["k"], c["T"]
    pi = [(r + 1) ** -c["zipf"] for r in range(E)]
    if k == E:
        return float(E)
    lo, hi = 0.0, 1e9
    for _ in range(100):
        mid = 0.5 * (lo + hi)
        lo, hi = (mid, hi) if sum(1.0 - math.exp(-mid * p) for p in pi) < k else (lo, mid)
    return sum(1.0 - math.exp(-T * lo * p) for p in pi)


def work(case):
    c = case
    op, T, E, k, H, I, el = c["op"], c["T"], c["E"], c["k"], c["H"], c["I"], _EL[c["dtype"]]
    R, q = T * k, 17 / 32                                             # q: bytes of a 4-bit value and its share of a scale
    if op == "sort":
        b, f = (T + R) * H * el + 8 * R, 0
        if c["grad"]:
            b, f = b + (T + R) * H * el, R * H
    elif op == "merge":
        b, f = (T + R) * H * el + 8 * R, 2 * R * H
        if c["grad"]:
            b, f = b + (T + R) * H * el + 8 * R, 5 * R * H           # the rows are read once for both directions
    elif op == "route_grad":
        b, f = 12 * R + 4 * T * E, 4 * R
    elif op == "quantise":
        b, f = 2 * T * H * el + 2 * T * H * q, 4 * T * H
    elif op == "product":
        b, f = R * H * q + _active(c) * I * H * q + 2 * R * I, 2 * R * H * I
    else:
        rows = T * H * 2 + 2 * R * H * q + 2 * R * I * q + 4 * R * H + T * H * 2
        b, f = rows + _active(c) * 3 * H * I * q, 6 * R * H * I
    return {"bytes": float(b), "flops": float(f)}
