"""Choosing experts by scores, and experts in e4m3 with a scale for every block of 128 -- each as a plain evaluation with elementary torch
operations and as the calls a program makes of this library.

A case names its operator (`op`):
  choose    logits -> the experts of every token and their weights; with `grad` the gradient of the weights to the logits too
  quantise  rows -> e4m3 codes and a scale per 128 columns, and back to values
  weights   matrices -> e4m3 codes and a scale per 128 x 128 entries, and back to values
  product   rows in e4m3, sorted by expert, with the experts' e4m3 matrices (E = 1: one matrix for all rows)
  layer     a layer's experts in e4m3: quantise and sort, gate/up product with SwiGLU, down product, merge

The scale of a block is amax / 448 in fp32 (1 for a block of zeros, 2^-126 at least); a code is the nearest e4m3 value of the quotient by it.
The score of an expert is the softmax or the sigmoid of its logit; score + bias decides who is chosen, among the groups of neighbouring
experts whose two largest such values add up to most; weights are the scores themselves.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_EL = {"bf16": 2, "fp16": 2, "fp32": 4}
_TOP = 448.0


def _case(name, op, T, E=1, k=1, H=0, dtype="bf16", I=0, zipf=0.0, grad=False, scores="sigmoid", bias=True, groups=1, top_groups=1,
          renormalize=True, scale=1.0):
    c = dict(op=op, T=T, E=E, k=k, H=H, dtype=dtype, I=I, zipf=zipf, grad=grad, scores=scores, bias=bias, groups=groups, top_groups=top_groups,
             renormalize=renormalize, scale=scale)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # one token of a decode batch: latency
        _case("choose_decode_1", "choose", 1, 256, 8, dtype="fp32", groups=8, top_groups=4, scale=2.5),
        # a softmax router of an odd number of experts in training, weights not renormalised: the gradient is dense
        _case("choose_train_777_odd", "choose", 777, 40, 5, dtype="bf16", grad=True, scores="softmax", bias=False, renormalize=False),
        # a training chunk through a sigmoid router with a balancing bias and groups, both directions
        _case("choose_train_16384", "choose", 16384, 256, 8, dtype="fp32", grad=True, groups=8, top_groups=4, scale=2.5),
        # activations of a decode batch to 8 bits and back
        _case("quantise_129_fp32", "quantise", 129, H=2048, dtype="fp32"),
        # an expert layer's weights to 8 bits and back, as when a checkpoint is loaded
        _case("quantise_weights", "weights", 1536, E=64, H=2048),
        # one token through one matrix: a shared expert or a projection while decoding
        _case("product_decode_1", "product", 1, 1, 1, 4096, I=6144),
        # ragged everything: rows an expert, columns, and a last block of 112
        _case("product_777_odd", "product", 777, 40, 5, 1008, I=1003, zipf=0.8),
        # a prefill chunk through one matrix
        _case("product_prefill_8192", "product", 8192, 1, 1, 4096, I=4096),
        # one token through eight experts
        _case("layer_decode_1", "layer", 1, 64, 8, 2048, I=1024),
        # a decode batch that meets most experts: the weight stream
        _case("layer_decode_100", "layer", 100, 128, 8, 4096, I=1792),
        # a prefill chunk
        _case("layer_prefill_8192", "layer", 8192, 64, 8, 4096, I=1792, zipf=0.6),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["choose", "choose", "choose", "quantise", "weights", "product", "product", "product", "layer", "layer"])
    E, k = rng.choice([(8, 2), (16, 4), (40, 5), (64, 6), (64, 8), (128, 8), (256, 8)])
    zipf = round(rng.uniform(0.0, 0.8), 2)
    if op == "choose":
        groups = rng.choice([1, 1, 2, 4, 8])
        top_groups = rng.randrange(1, groups + 1)
        while top_groups * (E // groups) < k:
            top_groups += 1
        return _case(None, op, _log_int(rng, 1, 16384), E, k, dtype=rng.choice(["fp32", "bf16", "fp16"]), grad=rng.random() < 0.6,
                     scores=rng.choice(["sigmoid", "softmax"]), bias=rng.random() < 0.6, groups=groups, top_groups=top_groups,
                     renormalize=rng.random() < 0.6, scale=rng.choice([1.0, 2.5]))
    if op == "quantise":
        H = 16 * _log_int(rng, 8, 512)
        return _case(None, op, _log_int(rng, 1, 200_000_000 // H), H=H, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    if op == "weights":
        H, N = 16 * _log_int(rng, 8, 512), _log_int(rng, 1, 4096)
        return _case(None, op, N, E=_log_int(rng, 1, max(1, min(64, 200_000_000 // (N * H)))), H=H, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    if op == "product":
        one = rng.random() < 0.4
        H, I = 16 * _log_int(rng, 8, 384), _log_int(rng, 64, 6144)
        return _case(None, op, _log_int(rng, 1, 8192 if one else 2048), 1 if one else min(E, 128), 1 if one else k, H, I=I, zipf=0.0 if one else zipf,
                     dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    return _case(None, op, _log_int(rng, 1, 4096), min(E, 128), k, 128 * _log_int(rng, 2, 32), I=128 * _log_int(rng, 1, 14), zipf=zipf)


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
    return dict(w=w, s2f=s2f.int(), f2s=f2s.int(), offsets=offsets, most=int(counts.max()))


def _weights(E, N, K, g, dev):
    """Matrices N(0, 1/K) as codes [E, N, K] and scales [E, N/128, K/128], rounded up."""
    codes = torch.empty(E, N, K, dtype=torch.float8_e4m3fn, device=dev)
    scales = torch.empty(E, -(-N // 128), -(-K // 128), device=dev)
    for e in range(E):
        w = torch.empty(N, K, device=dev).normal_(0.0, K ** -0.5, generator=g)
        s = _block_scales(w, 128)
        codes[e] = (w / _spread(s, 128, N, K)).clamp_(-_TOP, _TOP).to(torch.float8_e4m3fn)
        scales[e] = s
    return codes, scales


def prepare(case, seed):
    c, dev = case, torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    T, E, k, H, I, dt = c["T"], c["E"], c["k"], c["H"], c["I"], _DT[c["dtype"]]
    s = dict(c=c)
    if c["op"] == "choose":
        s["z"] = torch.empty(T, E, device=dev).normal_(0.0, 1.5, generator=g).to(dt)
        s["bias"] = torch.empty(E, device=dev).normal_(0.0, 0.05, generator=g) if c["bias"] else None
        s["dw"] = torch.empty(T, k, device=dev).normal_(0.0, 1.0, generator=g)
        return s
    if c["op"] in ("quantise", "weights"):          # rows of different magnitudes
        n = T * E
        x = torch.empty(n, H, device=dev).normal_(0.0, 1.0, generator=g)
        s["x"] = x.mul_(torch.exp2(torch.randint(-6, 7, (n, 1), generator=g, device=dev).float())).to(dt)
        if c["op"] == "weights":
            s["x"] = s["x"].view(E, T, H)
        return s
    s.update(_routing(c, g, dev))
    x = torch.empty(T * k if c["op"] == "product" else T, H, device=dev).normal_(0.0, 1.0, generator=g)
    if c["op"] == "product":
        sx = _block_scales(x, 1)
        s["codes"], s["scales"] = (x / _spread(sx, 1, T * k, H)).clamp_(-_TOP, _TOP).to(torch.float8_e4m3fn), sx
        s["w1"] = _weights(E, I, H, g, dev)
    else:
        s["x"] = x.to(dt)
        s["w1"] = _weights(E, 2 * I, H, g, dev)
        s["w2"] = _weights(E, H, I, g, dev)
    return s


# ------------------------------------------------------------------ plain forms

def _block_scales(x, rows):
    """fp32 [..., N, K] -> the scales of its blocks of so many rows and 128 columns, those at the edges cut off."""
    N, K = x.shape[-2:]
    x = torch.nn.functional.pad(x.abs(), (0, -K % 128, 0, -N % rows))
    top = x.unflatten(-1, (-1, 128)).unflatten(-3, (-1, rows)).amax((-1, -3))
    return torch.where(top > 0, (top / _TOP).clamp(min=2.0 ** -126), torch.ones_like(top))


def _spread(s, rows, N, K):
    """Scales of blocks -> the scale of every entry."""
    return s.repeat_interleave(rows, -2)[..., :N, :].repeat_interleave(128, -1)[..., :K]


def _nearest(q):
    """fp64 quotients -> the nearest e4m3 values (three bits behind the leading one, steps of 2^-9 at least), as fp32."""
    a = q.abs().clamp_(max=_TOP)
    _, e = torch.frexp(a)
    step = torch.exp2((e - 4).clamp_(min=-9).double())
    return torch.copysign(torch.round(a / step).mul_(step).clamp_(max=_TOP), q).float()


def _quantised(x, rows):
    """The values that codes and scales of x stand for, fp32 (a gigabyte at a time)."""
    N, K = x.shape[-2:]
    s = _block_scales(x.float(), rows)
    flat, out = x.reshape(-1, N, K), torch.empty(x.shape, dtype=torch.float32, device=x.device).reshape(-1, N, K)
    scale = s.reshape(flat.shape[0], *s.shape[-2:])
    step = max(1, (1 << 27) // K // rows * rows)
    for b in range(flat.shape[0]):
        for i in range(0, N, step):
            sc = _spread(scale[b, i // rows:(i + step - 1) // rows + 1], rows, min(step, N - i), K)
            out[b, i:i + step] = _nearest(flat[b, i:i + step].double() / sc.double()) * sc
    return out.reshape(x.shape)


def _grouped(x, w, offsets, most):
    """x [R, K] sorted by expert times w [E, N, K]: every expert's rows in a slab of the largest expert's height."""
    if w.shape[0] == 1:
        return x @ w[0].T
    R, at = x.shape[0], torch.arange(most, device=x.device)
    index = offsets[:-1, None].long() + at
    slab = x[index.clamp(max=R - 1)]
    y = torch.bmm(slab, w.transpose(1, 2))
    return y[at < (offsets[1:] - offsets[:-1]).long()[:, None]]


def _matrices(w):
    codes, scales = w
    return codes.float() * _spread(scales, 128, *codes.shape[-2:])


def _scores(z, c):
    if c["scores"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z))
    e = torch.exp(z - z.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain_choose(s):
    c = s["c"]
    T, E, k, G = c["T"], c["E"], c["k"], c["groups"]
    z = s["z"].float()
    by = _scores(z.double(), c)                                       # who comes first is decided in 64 bits
    if s["bias"] is not None:
        by = by + s["bias"].double()
    if c["top_groups"] < G:
        two = torch.sort(by.view(T, G, E // G), dim=2, descending=True).values[:, :, :2].sum(2)
        kept = torch.sort(two, dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        on = torch.zeros(T, G, dtype=torch.bool, device=z.device)
        on[torch.arange(T, device=z.device)[:, None], kept] = True
        by = torch.where(on.repeat_interleave(E // G, 1), by, -math.inf)
    ids = torch.sort(by, dim=1, descending=True, stable=True).indices[:, :k]
    score = _scores(z, c)
    p = torch.gather(score, 1, ids)
    total = p.sum(1, keepdim=True)
    w = (p / total if c["renormalize"] else p) * c["scale"]
    out = dict(ids=ids.int(), w=w)
    if c["grad"]:
        d = s["dw"] * c["scale"]
        if c["renormalize"]:
            d = (d - (d * p).sum(1, keepdim=True) / total) / total
        ds = torch.zeros_like(score).scatter_(1, ids, d)
        if c["scores"] == "sigmoid":
            dz = ds * score * (1.0 / (1.0 + torch.exp(z)))
        else:
            dz = score * (ds - (ds * score).sum(1, keepdim=True))
            if c["renormalize"]:                                      # the others' terms cancel
                dz = torch.where(torch.zeros_like(score).scatter_(1, ids, 1.0) > 0, dz, 0.0)
        out["dz"] = dz.to(s["z"].dtype)
    return out


def _plain(s):
    c = s["c"]
    op, k = c["op"], c["k"]
    if op == "choose":
        return _plain_choose(s)
    if op in ("quantise", "weights"):
        return _quantised(s["x"], 1 if op == "quantise" else 128).to(s["x"].dtype)
    if op == "product":
        return _grouped(s["codes"].float() * _spread(s["scales"], 1, *s["codes"].shape), _matrices(s["w1"]), s["offsets"], s["most"]).to(_DT[c["dtype"]])
    x = _quantised(s["x"], 1)[s["s2f"] // k]
    h = _grouped(x, _matrices(s["w1"]), s["offsets"], s["most"])
    g, u = h[:, :c["I"]], h[:, c["I"]:]
    a = _quantised(g / (1.0 + torch.exp(-g)) * u, 1)
    d = _grouped(a, _matrices(s["w2"]), s["offsets"], s["most"])
    return (d[s["f2s"]].reshape(c["T"], k, -1) * s["w"][..., None]).sum(1).to(torch.bfloat16)


# ------------------------------------------------------------------ the library's calls

def _library(s):
    import paper_2607_18002_b200 as moe
    c = s["c"]
    op, k = c["op"], c["k"]
    if op == "choose":
        ids, w = moe.choose_experts(s["z"], k, scores=c["scores"], bias=s["bias"], groups=c["groups"], top_groups=c["top_groups"],
                                    renormalize=c["renormalize"], scale=c["scale"])
        out = dict(ids=ids, w=w)
        if c["grad"]:
            out["dz"] = moe.choose_experts_grad(s["z"], ids, s["dw"], scores=c["scores"], renormalize=c["renormalize"], scale=c["scale"])
        return out
    if op == "quantise":
        return moe.scaled_dequantize(*moe.scaled_quantize(s["x"]), s["x"].dtype)
    if op == "weights":
        return moe.scaled_dequantize(*moe.scaled_quantize_weights(s["x"]), s["x"].dtype)
    if op == "product":
        return moe.scaled_product(s["codes"], s["scales"], *s["w1"], s["offsets"], _DT[c["dtype"]])
    x = moe.scaled_quantize(s["x"], s["s2f"], s["f2s"], k)
    a = moe.scaled_swiglu(*x, *s["w1"], s["offsets"])
    d = moe.scaled_product(*a, *s["w2"], s["offsets"])
    return moe.merge_rows(d, s["f2s"], s["w"])


def run(state):
    return _library(state) if own else _plain(state)


# ------------------------------------------------------------------ the definitions in 64 bits

def _grid(dev):
    """The magnitudes of e4m3, 0 to 448."""
    sub = torch.arange(8, dtype=torch.float64, device=dev) / 512.0
    binades = [(8.0 + torch.arange(8, dtype=torch.float64, device=dev)) * 2.0 ** (e - 3) for e in range(-6, 9)]
    return torch.cat([sub, *binades])[:-1]


def _stored(x, rows):
    """fp64 [N, K]: every entry replaced by the nearest multiple of its block's scale that 8 bits can hold."""
    N, K = x.shape
    grid = _grid(x.device)
    mid = (grid[1:] + grid[:-1]) / 2
    out = torch.empty_like(x)
    per = max(rows, (1 << 26) // K // rows * rows)
    for i in range(0, N, per):
        for j in range(0, K, 128):
            b = x[i:i + per, j:j + 128]
            top = b.abs().amax(1)
            if rows > 1:
                top = torch.nn.functional.pad(top, (0, -top.numel() % rows)).view(-1, rows).amax(1).repeat_interleave(rows)[:b.shape[0]]
            scale = torch.where(top > 0, (top.float() / 448.0).clamp(min=2.0 ** -126).double(), 1.0)[:, None]
            a = b.abs() / scale
            at = torch.bucketize(a, mid)                              # midpoints below a; at one itself the even code wins
            tie = (at < 126) & (mid[at.clamp(max=125)] == a) & (at % 2 == 1)
            out[i:i + per, j:j + 128] = torch.copysign(grid[at + tie.long()], b) * scale
    return out


def _decoded(w, e):
    codes, scales = w[0][e].double(), w[1][e].double()
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            codes[128 * i:128 * i + 128, 128 * j:128 * j + 128] *= scales[i, j]
    return codes


def _by_expert(x, w, offsets):
    """One expert after the other."""
    out, o = [], offsets.tolist()
    for e in range(len(o) - 1):
        if o[e + 1] > o[e]:
            out.append(x[o[e]:o[e + 1]] @ _decoded(w, e).T)
    return torch.cat(out)


def _exact_choose(s):
    c = s["c"]
    T, E, k, G, dev = c["T"], c["E"], c["k"], c["groups"], s["z"].device
    z = s["z"].double()
    score = torch.sigmoid(z) if c["scores"] == "sigmoid" else torch.softmax(z, 1)
    by = score if s["bias"] is None else score + s["bias"].double()
    by, row = by.clone(), torch.arange(T, device=dev)
    if c["top_groups"] < G:
        b = by.view(T, G, E // G)
        value = torch.topk(b, 2, dim=2).values.sum(2) if E // G > 1 else b[:, :, 0]
        out = torch.ones(T, G, dtype=torch.bool, device=dev)
        for _ in range(c["top_groups"]):
            best = (value == value.amax(1, keepdim=True)).int().argmax(1)
            value[row, best], out[row, best] = -math.inf, False
        by[out.repeat_interleave(E // G, 1)] = -math.inf
    ids = []
    for _ in range(k):
        best = (by == by.amax(1, keepdim=True)).int().argmax(1)       # the first of equals
        ids.append(best)
        by[row, best] = -math.inf
    ids = torch.stack(ids, 1)
    p = score[row[:, None], ids]
    total = p.sum(1, keepdim=True) if c["renormalize"] else torch.ones(T, 1, dtype=torch.float64, device=dev)
    w = c["scale"] * p / total
    res = dict(ids=ids.int(), w=w)
    if c["grad"]:                                                     # through the Jacobian of the chosen scores
        d = s["dw"].double()
        ds = c["scale"] * d / total
        if c["renormalize"]:
            ds = ds - (w * d).sum(1, keepdim=True) / total
        dz = torch.zeros_like(z)
        if c["scores"] == "sigmoid":
            dz[row[:, None], ids] = ds * p * torch.sigmoid(-z[row[:, None], ids])
        else:
            dz[row[:, None], ids] = ds * p
            if not c["renormalize"]:
                dz -= score * (ds * p).sum(1, keepdim=True)
        res["dz"] = dz
    return res


def exact(case, seed):
    c, s = case, prepare(case, seed)
    op, T, k = c["op"], c["T"], c["k"]
    if op == "choose":
        return _exact_choose(s)
    if op == "quantise":
        return _stored(s["x"].double(), 1)
    if op == "weights":
        return torch.stack([_stored(m.double(), 128) for m in s["x"]])
    if op == "product":
        x = s["codes"].double()
        for j in range(s["scales"].shape[1]):
            x[:, 128 * j:128 * j + 128] *= s["scales"][:, j:j + 1].double()
        return _by_expert(x, s["w1"], s["offsets"])
    token = torch.div(s["s2f"].long(), k, rounding_mode="floor")
    h = _by_expert(torch.index_select(_stored(s["x"].double(), 1), 0, token), s["w1"], s["offsets"])
    g, u = h.split(c["I"], dim=1)
    d = _by_expert(_stored(g * torch.sigmoid(g) * u, 1), s["w2"], s["offsets"])
    w = s["w"].double().reshape(-1)[s["s2f"].long()]
    return torch.zeros(T, c["H"], dtype=torch.float64, device=d.device).index_add_(0, token, d * w[:, None])


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
    R, q = T * k, 1.0 + 4.0 / 128                                     # q: bytes of an 8-bit value and its share of a row's scale
    if op == "choose":
        b, f = T * E * el + 8 * R + (4 * E if c["bias"] else 0), 8 * T * E
        if c["grad"]:                                                 # the logits are read once for both directions
            b, f = b + T * E * el + 4 * R, f + 4 * T * E
    elif op == "quantise":
        b, f = 2 * T * H * el + 2 * T * H * q, 4 * T * H
    elif op == "weights":
        n = T * E * H
        b, f = 2 * n * el + 2 * n, 4 * n
    elif op == "product":
        b, f = R * H * q + _active(c) * I * H + R * I * el, 2 * R * H * I
    else:
        rows = T * H * 2 + 2 * R * H * q + 2 * R * I * q + 4 * R * H + T * H * 2
        b, f = rows + _active(c) * 3 * H * I, 6 * R * H * I
    return {"bytes": float(b), "flops": float(f)}
