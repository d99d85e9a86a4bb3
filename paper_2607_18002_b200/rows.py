"""The rows of a routed layer as tensors: sorted by expert and put together again, their gradients, the router's gradient, routers by scores, and the
experts in 4 bits or in e4m3 with block scales (moe_route_grad ... moe_scaled_swiglu of include/moe_apk.h).

Checks of arguments and marshalling only; a call enqueues one kernel on `stream` (the current stream of the tensors' device if
None) and allocates its outputs there.  Nothing is recorded for autograd: gradients are calls of their own.  Wrong types, shapes, strides
or devices and sizes past 32 bits raise ValueError, what the library refuses MoeError.  Inputs may require gradients (experts' outputs of a graph of the caller's own do); results never do.
As with any work on another stream, inputs have to live until `stream` has read them, and `stream` has to be waited for before results are used elsewhere.
A permutation is the pair (sorted_to_flat, flat_to_sorted) of a plan, int32 [T*k] each, the inverses of one another: of moe_plan (a Context's), of moe_plan_static
(up to 32 768 rows and 256 experts, no context) or, for any size and without either, by a stable sort of the expert ids:

    order = torch.argsort(topk_ids.flatten(), stable=True)
    s2f, f2s = order.int(), torch.argsort(order).int()
    offsets = torch.nn.functional.pad(torch.bincount(topk_ids.flatten(), minlength=n_experts).cumsum(0), (1, 0)).int()

    codes, scales = mx_quantize(x, s2f, f2s, k)                          # experts of a layer in 4 bits
    codes, scales = mx_swiglu(codes, scales, w1_codes, w1_scales, offsets)
    rows = mx_product(codes, scales, w2_codes, w2_scales, offsets)
    y = merge_rows(rows, f2s, topk_w)

    codes, scales = scaled_quantize(x, s2f, f2s, k)                      # ... in e4m3, weights from scaled_quantize_weights or a context's
    codes, scales = scaled_swiglu(codes, scales, w1_codes, w1_scales, offsets)
    rows = scaled_product(codes, scales, w2_codes, w2_scales, offsets)   # bf16; dtype=torch.float32 where outputs are not to be rounded before they are merged
    y = merge_rows(rows, f2s, topk_w)
    rows = scaled_product(codes, scales, w_codes, w_scales)              # one matrix [n, K] for all rows: a shared expert, a projection

    ids, topk_w = choose_experts(logits, k, scores="sigmoid", bias=bias, groups=8, top_groups=4, scale=2.5)
    dlogits = choose_experts_grad(logits, ids, dw, scores="sigmoid", scale=2.5)

    xs = sort_rows(x, s2f, f2s, k)                                       # training, with experts of the caller's own
    y = merge_rows(experts(xs), f2s, topk_w)
    drows, dw = merge_rows_grad(dy, rows, s2f, f2s, topk_w)
    dx = sort_rows_grad(dxs, f2s, k)
    dlogits = route_grad(topk_ids, topk_w, dw, n_experts)
"""
from __future__ import annotations

import torch

import paper_2607_18002_b200 as moe

_BF16, _FP32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
_DTYPES = {_BF16: moe.MOE_DTYPE_BF16, torch.float16: moe.MOE_DTYPE_FP16, _FP32: moe.MOE_DTYPE_FP32}
_SORTED_DTYPES = {**_DTYPES, torch.float8_e4m3fn: moe.MOE_DTYPE_FP8_E4M3, _U8: moe.MOE_DTYPE_FP8_E4M3}
_Tensor, _empty = torch.Tensor, torch.empty
# the current device's number and the handle of its current stream: the functions of torch that read them without objects around them, where it has them
_current_device, _stream = (getattr(torch._C, n, None) for n in ("_cuda_getDevice", "_cuda_getCurrentRawStream"))
if _current_device is None or _stream is None:
    _current_device, _stream = torch.cuda.current_device, lambda gpu: torch.cuda.current_stream(gpu).cuda_stream


def _refuse(what):
    raise ValueError(what)


def _past_32_bits(*numbers):
    """Whether one of them is no number of 32 bits with a sign, which the library takes (ctypes would cut it off); each for itself: a negative one hides no others."""
    return any((n + 0x80000000) >> 32 for n in numbers)


def _rows(t, name, dtypes):
    """[n, H] with neighbouring columns -> n, H, elements from a row to the next."""
    if not isinstance(t, _Tensor) or t.dtype not in dtypes or not t.is_cuda or t.dim() != 2:
        _refuse(f"{name} must be a CUDA tensor [rows, columns] of one of {sorted(map(str, dtypes))}")
    n, h = t.shape
    step, one = t.stride()
    if h < 1 or (one != 1 and h > 1) or (n > 1 and step < h):
        _refuse(f"{name}: the columns of a row must be neighbours and rows must not overlap")
    if (n | h) >> 31:
        _refuse(f"{name}: there must be fewer than 2^31 rows and columns")
    return n, h, step if step > h else h


def _plain(t, name, dtype, shape, gpu):
    """A contiguous tensor of this type and shape on GPU number `gpu`."""
    if not isinstance(t, _Tensor) or t.dtype is not dtype or t.shape != shape or t.get_device() != gpu or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous {dtype} tensor {tuple(shape)} on cuda:{gpu}")


def _index(t, name, n, gpu):
    if not isinstance(t, _Tensor) or t.dtype is not _I32 or t.get_device() != gpu or not t.is_contiguous() \
            or t.numel() != n and (n or t.numel() != 1) or n >> 31:     # (a plan without rows has arrays of one entry)
        _refuse(f"{name} must be a contiguous int32 tensor of {n} (fewer than 2^31) on cuda:{gpu}")


def _elsewhere(call, device, stream, *args):
    """The same call with the device current and `stream` its current stream: outputs are allocated there and the kernel is enqueued there."""
    if stream is not None and stream.device != device:
        _refuse(f"the stream is on {stream.device}, the tensors are on {device}")
    with torch.cuda.device(device), torch.cuda.stream(stream):          # (a stream of None changes nothing)
        return call(*args)


def _failed(rc, name):
    raise moe.MoeError(rc, name)


def sort_rows(x, sorted_to_flat, flat_to_sorted, top_k: int, stream=None):
    """x [T, H] -> [T*k, H], the tokens' rows by expert (bf16, fp16, fp32, or one-byte codes)."""
    T, H, step = _rows(x, "x", _SORTED_DTYPES)
    gpu = x.get_device()
    if stream is not None or gpu != _current_device():
        return _elsewhere(sort_rows, x.device, stream, x, sorted_to_flat, flat_to_sorted, top_k)
    _index(sorted_to_flat, "sorted_to_flat", T * top_k, gpu)
    _index(flat_to_sorted, "flat_to_sorted", T * top_k, gpu)
    xs = x.new_empty(T * top_k, H)
    rc = (moe._lib or moe.lib()).moe_sort_rows(x.data_ptr(), step, _SORTED_DTYPES[x.dtype], T, top_k, H, sorted_to_flat.data_ptr(),
                                               flat_to_sorted.data_ptr(), xs.data_ptr(), _stream(gpu))
    if rc:
        _failed(rc, "moe_sort_rows")
    return xs


def sort_rows_grad(dxs, flat_to_sorted, top_k: int, stream=None):
    """dxs [T*k, H], the gradient of sort_rows' result -> that of x [T, H]."""
    R, H, step = _rows(dxs, "dxs", _DTYPES)
    gpu = dxs.get_device()
    if stream is not None or gpu != _current_device():
        return _elsewhere(sort_rows_grad, dxs.device, stream, dxs, flat_to_sorted, top_k)
    if top_k < 1 or R % top_k:
        _refuse("dxs must have top_k rows for every token")
    _index(flat_to_sorted, "flat_to_sorted", R, gpu)
    T = R // top_k
    dx = dxs.new_empty(T, H)
    rc = (moe._lib or moe.lib()).moe_sort_rows_grad(dxs.data_ptr(), step, _DTYPES[dxs.dtype], T, top_k, H, flat_to_sorted.data_ptr(),
                                                    dx.data_ptr(), _stream(gpu))
    if rc:
        _failed(rc, "moe_sort_rows_grad")
    return dx


def _weights(topk_w, R, gpu):
    if not isinstance(topk_w, _Tensor) or topk_w.dtype is not _FP32 or topk_w.dim() != 2 or topk_w.numel() != R or topk_w.get_device() != gpu \
            or not topk_w.is_contiguous():
        _refuse(f"topk_w must be a contiguous fp32 tensor [T, k] on cuda:{gpu}, a weight for each of the {R} rows")
    return topk_w.shape


def merge_rows(rows, flat_to_sorted, topk_w, stream=None):
    """rows [T*k, H] by expert -> y [T, H], the tokens' rows added up with their router weights."""
    R, H, step = _rows(rows, "rows", _DTYPES)
    gpu = rows.get_device()
    if stream is not None or gpu != _current_device():
        return _elsewhere(merge_rows, rows.device, stream, rows, flat_to_sorted, topk_w)
    T, k = _weights(topk_w, R, gpu)
    _index(flat_to_sorted, "flat_to_sorted", R, gpu)
    y = rows.new_empty(T, H)
    rc = (moe._lib or moe.lib()).moe_merge_rows(rows.data_ptr(), step, _DTYPES[rows.dtype], topk_w.data_ptr(), T, k, H,
                                                flat_to_sorted.data_ptr(), y.data_ptr(), _stream(gpu))
    if rc:
        _failed(rc, "moe_merge_rows")
    return y


def merge_rows_grad(dy, rows, sorted_to_flat, flat_to_sorted, topk_w, stream=None):
    """dy [T, H], the gradient of merge_rows' result -> (that of rows [T*k, H], that of topk_w [T, k] fp32)."""
    R, H, step = _rows(rows, "rows", _DTYPES)
    gpu = rows.get_device()
    if stream is not None or gpu != _current_device():
        return _elsewhere(merge_rows_grad, rows.device, stream, dy, rows, sorted_to_flat, flat_to_sorted, topk_w)
    T, k = _weights(topk_w, R, gpu)
    dT, dH, dy_step = _rows(dy, "dy", _DTYPES)
    if dT != T or dH != H or dy.dtype is not rows.dtype or dy.get_device() != gpu:
        _refuse(f"dy must be a {rows.dtype} tensor [{T}, {H}] on cuda:{gpu}")
    _index(sorted_to_flat, "sorted_to_flat", R, gpu)
    _index(flat_to_sorted, "flat_to_sorted", R, gpu)
    drows, dw = rows.new_empty(R, H), topk_w.new_empty(T, k)
    rc = (moe._lib or moe.lib()).moe_merge_rows_grad(dy.data_ptr(), dy_step, rows.data_ptr(), step, _DTYPES[rows.dtype], topk_w.data_ptr(), T, k, H,
                                                     sorted_to_flat.data_ptr(), flat_to_sorted.data_ptr(), drows.data_ptr(), dw.data_ptr(),
                                                     _stream(gpu))
    if rc:
        _failed(rc, "moe_merge_rows_grad")
    return drows, dw


def route_grad(topk_ids, topk_w, d_topk_w, n_experts: int, stream=None):
    """The gradient of route's weights, fp32 [T, k] -> that of the logits, fp32 [T, E]."""
    if not isinstance(topk_ids, _Tensor) or not topk_ids.is_cuda or topk_ids.dim() != 2:
        _refuse("topk_ids must be a CUDA int32 tensor [T, k]")
    shape, gpu = topk_ids.shape, topk_ids.get_device()
    if stream is not None or gpu != _current_device():
        return _elsewhere(route_grad, topk_ids.device, stream, topk_ids, topk_w, d_topk_w, n_experts)
    _plain(topk_ids, "topk_ids", _I32, shape, gpu)
    _plain(topk_w, "topk_w", _FP32, shape, gpu)
    _plain(d_topk_w, "d_topk_w", _FP32, shape, gpu)
    T, k = shape
    if (T | k | n_experts) >> 31 and _past_32_bits(T, k, n_experts):
        _refuse("the tokens, slots and experts must be below 2^31")
    dz = topk_w.new_empty(T, n_experts)
    rc = (moe._lib or moe.lib()).moe_route_grad(topk_ids.data_ptr(), topk_w.data_ptr(), d_topk_w.data_ptr(), T, n_experts, k, dz.data_ptr(),
                                                _stream(gpu))
    if rc:
        _failed(rc, "moe_route_grad")
    return dz


def mx_quantize(x, sorted_to_flat=None, flat_to_sorted=None, top_k: int = 1, stream=None):
    """x [..., K] -> codes uint8 [..., K/2], scales uint8 [..., K/32]; with a permutation x [T, K] -> the T*k rows by expert.  Contiguous, or [T, K] of any row stride."""
    if isinstance(x, _Tensor) and x.dim() not in (0, 2) and x.is_contiguous() and sorted_to_flat is None and flat_to_sorted is None:
        *lead, K = x.shape
        codes, scales = mx_quantize(x.view(x.numel() // K if K else 0, K), None, None, top_k, stream)
        return codes.view(*lead, codes.shape[1]), scales.view(*lead, scales.shape[1])
    T, K, step = _rows(x, "x", _DTYPES)
    gpu = x.get_device()
    if stream is not None or gpu != _current_device():
        return _elsewhere(mx_quantize, x.device, stream, x, sorted_to_flat, flat_to_sorted, top_k)
    if K % 32:
        _refuse("x must have a multiple of 32 columns")
    R = T * top_k
    s2f = f2s = None
    if sorted_to_flat is not None or flat_to_sorted is not None:
        _index(sorted_to_flat, "sorted_to_flat", R, gpu)
        _index(flat_to_sorted, "flat_to_sorted", R, gpu)
        s2f, f2s = sorted_to_flat.data_ptr(), flat_to_sorted.data_ptr()
    elif top_k != 1:
        _refuse("top_k needs a permutation")
    codes = _empty(R, K // 2, dtype=_U8, device=x.device)
    scales = codes.new_empty(R, K // 32)
    rc = (moe._lib or moe.lib()).moe_mx_quantize(x.data_ptr(), step, _DTYPES[x.dtype], T, top_k, K, s2f, f2s, codes.data_ptr(),
                                                 scales.data_ptr(), _stream(gpu))
    if rc:
        _failed(rc, "moe_mx_quantize")
    return codes, scales


def _codes(codes, scales, what, dims):
    """Codes [..., K/2] and scales [..., K/32] of so many dimensions (0: any) -> the shape of the codes and the number of their GPU."""
    if not isinstance(codes, _Tensor) or not isinstance(scales, _Tensor):
        _refuse(f"the codes and scales of {what} must be tensors")
    shape, width, gpu = codes.shape, scales.shape, codes.get_device()
    n = len(shape)
    if codes.dtype is not _U8 or scales.dtype is not _U8 or not codes.is_cuda or gpu != scales.get_device() or not codes.is_contiguous() \
            or not scales.is_contiguous() or (n != dims if dims else not n) or len(width) != n or shape[n - 1] != 16 * width[n - 1] \
            or (shape[0] != width[0] and n > 1) or (n > 2 and shape[1:-1] != width[1:-1]):
        _refuse(f"the codes and scales of {what} must be contiguous uint8 tensors of {dims or 'some'} dimensions on one GPU, a scale for 16 bytes of codes")
    return shape, gpu


def mx_dequantize(codes, scales, dtype=_BF16, stream=None):
    """The values [..., K] that codes [..., K/2] with scales [..., K/32] stand for."""
    if dtype not in _DTYPES:
        _refuse(f"dtype must be one of {sorted(map(str, _DTYPES))}")
    (*lead, half), gpu = _codes(codes, scales, "the rows", 0)
    K = 2 * half
    if stream is not None or gpu != _current_device():
        return _elsewhere(mx_dequantize, codes.device, stream, codes, scales, dtype)
    if K >> 31:
        _refuse("there must be fewer than 2^31 columns")
    out = _empty(*lead, K, dtype=dtype, device=codes.device)
    if K:
        rc = (moe._lib or moe.lib()).moe_mx_dequantize(codes.data_ptr(), scales.data_ptr(), out.numel() // K, K, _DTYPES[dtype], out.data_ptr(),
                                                       _stream(gpu))
        if rc:
            _failed(rc, "moe_mx_dequantize")
    return out


def _operands(codes, scales, w_codes, w_scales, offsets):
    """-> number of the GPU, R, E, n, K"""
    (R, half), gpu = _codes(codes, scales, "the rows", 2)
    (E, n, w_half), w_gpu = _codes(w_codes, w_scales, "the weights", 3)
    if w_half != half or w_gpu != gpu:
        _refuse(f"the weights must have {2 * half} columns and be on cuda:{gpu}, as the rows")
    if (R | E | n | 2 * half) >> 31:
        _refuse("the rows, experts and columns must be below 2^31")
    _index(offsets, "offsets", E + 1, gpu)
    return gpu, R, E, n, 2 * half


def mx_product(codes, scales, w_codes, w_scales, offsets, stream=None):
    """Sorted 4-bit rows [R, K] times the experts' matrices [E, n, K] -> bf16 [R, n]."""
    gpu, R, E, n, K = _operands(codes, scales, w_codes, w_scales, offsets)
    if stream is not None or gpu != _current_device():
        return _elsewhere(mx_product, codes.device, stream, codes, scales, w_codes, w_scales, offsets)
    out = _empty(R, n, dtype=_BF16, device=codes.device)
    rc = (moe._lib or moe.lib()).moe_mx_product(codes.data_ptr(), scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), offsets.data_ptr(), R, E,
                                                n, K, out.data_ptr(), _stream(gpu))
    if rc:
        _failed(rc, "moe_mx_product")
    return out


def mx_swiglu(codes, scales, w_codes, w_scales, offsets, stream=None):
    """Sorted 4-bit rows [R, K] times gate and up matrices [E, 2 I, K], silu(gate) * up -> codes [R, I/2], scales [R, I/32]."""
    gpu, R, E, n, K = _operands(codes, scales, w_codes, w_scales, offsets)
    if n % 64:
        _refuse("the weights must have gate and up rows, a multiple of 32 each")
    if stream is not None or gpu != _current_device():
        return _elsewhere(mx_swiglu, codes.device, stream, codes, scales, w_codes, w_scales, offsets)
    out, out_scales = codes.new_empty(R, n // 4), codes.new_empty(R, n // 64)
    rc = (moe._lib or moe.lib()).moe_mx_swiglu(codes.data_ptr(), scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), offsets.data_ptr(), R, E,
                                               n // 2, K, out.data_ptr(), out_scales.data_ptr(), _stream(gpu))
    if rc:
        _failed(rc, "moe_mx_swiglu")
    return out, out_scales


_SCORES = {"softmax": moe.MOE_SCORES_SOFTMAX, "sigmoid": moe.MOE_SCORES_SIGMOID}
_F8 = torch.float8_e4m3fn


def choose_experts(logits, top_k: int, *, scores: str = "softmax", bias=None, groups: int = 1, top_groups: int = 1, group_sum: int = 2,
                   renormalize: bool = True, scale: float = 1.0, stream=None):
    """logits [T, E] (bf16, fp16, fp32) -> (topk_ids int32 [T, k], topk_w fp32 [T, k]): the k largest scores (softmax or sigmoid) plus bias [E] fp32
    among the top_groups groups of experts, weighted by their scores (moe_choose_experts)."""
    T, E, step = _rows(logits, "logits", _DTYPES)
    gpu = logits.get_device()
    if stream is not None or gpu != _current_device():
        return _elsewhere(lambda: choose_experts(logits, top_k, scores=scores, bias=bias, groups=groups, top_groups=top_groups, group_sum=group_sum,
                                                 renormalize=renormalize, scale=scale), logits.device, stream)
    if scores not in _SCORES:
        _refuse(f"scores must be one of {sorted(_SCORES)}")
    if bias is not None:
        _plain(bias, "bias", _FP32, (E,), gpu)
    if (top_k | groups | top_groups | group_sum) >> 31 and _past_32_bits(top_k, groups, top_groups, group_sum):      # (a negative one, or one past 32 bits)
        _refuse("top_k and the groups must be below 2^31")
    k = top_k if top_k > 0 else 0               # (the library refuses what is not)
    device = logits.device
    ids, w = _empty(T, k, dtype=_I32, device=device), _empty(T, k, dtype=_FP32, device=device)
    rc = (moe._lib or moe.lib()).moe_choose_experts(logits.data_ptr(), step, _DTYPES[logits.dtype], None if bias is None else bias.data_ptr(), T, E, top_k,
                                                    groups, top_groups, group_sum, _SCORES[scores], renormalize, scale, ids.data_ptr(), w.data_ptr(),
                                                    _stream(gpu))
    if rc:
        _failed(rc, "moe_choose_experts")
    return ids, w


def choose_experts_grad(logits, topk_ids, d_topk_w, *, scores: str = "softmax", renormalize: bool = True, scale: float = 1.0, stream=None):
    """The gradient of choose_experts' weights, fp32 [T, k] -> that of the logits [T, E], of their type."""
    T, E, step = _rows(logits, "logits", _DTYPES)
    gpu = logits.get_device()
    if stream is not None or gpu != _current_device():
        return _elsewhere(lambda: choose_experts_grad(logits, topk_ids, d_topk_w, scores=scores, renormalize=renormalize, scale=scale), logits.device,
                          stream)
    if scores not in _SCORES:
        _refuse(f"scores must be one of {sorted(_SCORES)}")
    if not isinstance(topk_ids, _Tensor) or topk_ids.dim() != 2:
        _refuse("topk_ids must be a CUDA int32 tensor [T, k]")
    k = topk_ids.shape[1]
    _plain(topk_ids, "topk_ids", _I32, (T, k), gpu)
    _plain(d_topk_w, "d_topk_w", _FP32, (T, k), gpu)
    if k >> 31:
        _refuse("there must be fewer than 2^31 slots")
    dz = logits.new_empty(T, E)
    rc = (moe._lib or moe.lib()).moe_choose_experts_grad(logits.data_ptr(), step, _DTYPES[logits.dtype], topk_ids.data_ptr(), d_topk_w.data_ptr(), T, E, k,
                                                         _SCORES[scores], renormalize, scale, dz.data_ptr(), _stream(gpu))
    if rc:
        _failed(rc, "moe_choose_experts_grad")
    return dz


def _blocks(n):
    return (n + 127) // 128


def scaled_quantize(x, sorted_to_flat=None, flat_to_sorted=None, top_k: int = 1, stream=None):
    """x [..., K] -> codes float8_e4m3fn [..., K], scales fp32 [..., ceil(K/128)]; with a permutation x [T, K] -> the T*k rows by expert.  Contiguous, or [T, K]
    of any row stride."""
    if isinstance(x, _Tensor) and x.dim() not in (0, 2) and x.is_contiguous() and sorted_to_flat is None and flat_to_sorted is None:
        *lead, K = x.shape
        codes, scales = scaled_quantize(x.view(x.numel() // K if K else 0, K), None, None, top_k, stream)
        return codes.view(*lead, K), scales.view(*lead, scales.shape[1])
    T, K, step = _rows(x, "x", _DTYPES)
    gpu = x.get_device()
    if stream is not None or gpu != _current_device():
        return _elsewhere(scaled_quantize, x.device, stream, x, sorted_to_flat, flat_to_sorted, top_k)
    if K % 16:
        _refuse("x must have a multiple of 16 columns")
    R = T * top_k
    s2f = f2s = None
    if sorted_to_flat is not None or flat_to_sorted is not None:
        _index(sorted_to_flat, "sorted_to_flat", R, gpu)
        _index(flat_to_sorted, "flat_to_sorted", R, gpu)
        s2f, f2s = sorted_to_flat.data_ptr(), flat_to_sorted.data_ptr()
    elif top_k != 1:
        _refuse("top_k needs a permutation")
    codes = _empty(R, K, dtype=_F8, device=x.device)
    scales = _empty(R, _blocks(K), dtype=_FP32, device=x.device)
    rc = (moe._lib or moe.lib()).moe_scaled_quantize(x.data_ptr(), step, _DTYPES[x.dtype], T, top_k, K, s2f, f2s, codes.data_ptr(), scales.data_ptr(),
                                                     _stream(gpu))
    if rc:
        _failed(rc, "moe_scaled_quantize")
    return codes, scales


def scaled_quantize_weights(w, stream=None):
    """w [E, n, K] or [n, K], contiguous -> codes float8_e4m3fn of that shape, scales fp32 [E, ceil(n/128), ceil(K/128)] or without E."""
    if not isinstance(w, _Tensor) or w.dtype not in _DTYPES or not w.is_cuda or w.dim() not in (2, 3) or not w.is_contiguous():
        _refuse(f"w must be a contiguous CUDA tensor [E, n, K] or [n, K] of one of {sorted(map(str, _DTYPES))}")
    gpu = w.get_device()
    if stream is not None or gpu != _current_device():
        return _elsewhere(scaled_quantize_weights, w.device, stream, w)
    *lead, n, K = w.shape
    if K % 16 or not K or not n:
        _refuse("w must have rows, and a multiple of 16 columns")
    if (w.shape[0] | n | K) >> 31:
        _refuse("the experts, rows and columns must be below 2^31")
    codes = _empty(w.shape, dtype=_F8, device=w.device)
    scales = _empty(*lead, _blocks(n), _blocks(K), dtype=_FP32, device=w.device)
    rc = (moe._lib or moe.lib()).moe_scaled_quantize_weights(w.data_ptr(), _DTYPES[w.dtype], lead[0] if lead else 1, n, K, codes.data_ptr(),
                                                             scales.data_ptr(), _stream(gpu))
    if rc:
        _failed(rc, "moe_scaled_quantize_weights")
    return codes, scales


def _scaled(codes, scales, what, per_row):
    """Codes [..., n, K] with a scale for every 128 columns of a row (per_row) or of 128 rows -> their shape and the number of their GPU."""
    if not isinstance(codes, _Tensor) or not isinstance(scales, _Tensor):
        _refuse(f"the codes and scales of {what} must be tensors")
    shape, blocks, gpu, dtype = codes.shape, scales.shape, codes.get_device(), codes.dtype
    n = len(shape)
    if dtype is not _F8 and dtype is not _U8 or scales.dtype is not _FP32 or gpu < 0 or gpu != scales.get_device() \
            or not codes.is_contiguous() or not scales.is_contiguous() or n < 2 or len(blocks) != n or blocks[n - 1] != (shape[n - 1] + 127) // 128 \
            or blocks[n - 2] != (shape[n - 2] if per_row else (shape[n - 2] + 127) // 128) or n > 2 and shape[:n - 2] != blocks[:n - 2]:
        _refuse(f"the codes and scales of {what} must be contiguous e4m3 (or uint8) and fp32 tensors on one GPU, a scale for 128 columns "
                f"of {'a row' if per_row else '128 rows'}")
    return shape, gpu


def scaled_dequantize(codes, scales, dtype=_BF16, stream=None):
    """The values [..., n, K] that codes stand for with the scales of rows [..., n, ceil(K/128)] or of weights [..., ceil(n/128), ceil(K/128)]."""
    if dtype not in _DTYPES:
        _refuse(f"dtype must be one of {sorted(map(str, _DTYPES))}")
    if isinstance(codes, _Tensor) and isinstance(scales, _Tensor) and codes.dim() == 1:
        return scaled_dequantize(codes[None], scales[None], dtype, stream)[0]
    per_row = isinstance(codes, _Tensor) and isinstance(scales, _Tensor) and codes.dim() > 1 and scales.dim() > 1 and scales.shape[-2] == codes.shape[-2]
    shape, gpu = _scaled(codes, scales, "the values", per_row)
    if stream is not None or gpu != _current_device():
        return _elsewhere(scaled_dequantize, codes.device, stream, codes, scales, dtype)
    values, n, K = codes.numel(), shape[-2], shape[-1]
    E = values // (n * K) if values else 0
    if (E | n | K) >> 31:
        _refuse("the matrices, rows and columns must be below 2^31")
    out = _empty(*shape, dtype=dtype, device=codes.device)
    if values:
        rc = (moe._lib or moe.lib()).moe_scaled_dequantize(codes.data_ptr(), scales.data_ptr(), E, n, K, 1 if per_row else 128,
                                                           _DTYPES[dtype], out.data_ptr(), _stream(gpu))
        if rc:
            _failed(rc, "moe_scaled_dequantize")
    return out


def _scaled_operands(codes, scales, w_codes, w_scales, offsets):
    """-> number of the GPU, R, E, n, K, address of the offsets"""
    shape, gpu = _scaled(codes, scales, "the rows", True)
    w_shape, w_gpu = _scaled(w_codes, w_scales, "the weights", False)
    dims = len(w_shape)
    if len(shape) != 2 or dims > 3 or w_shape[dims - 1] != shape[1] or w_gpu != gpu:
        _refuse(f"rows must be [R, K] and weights [E, n, K] or [n, K], all on cuda:{gpu}")
    E, n = w_shape[0] if dims == 3 else 1, w_shape[dims - 2]
    if (shape[0] | shape[1] | E | n) >> 31:
        _refuse("the rows, experts and columns must be below 2^31")
    at = None
    if offsets is not None:
        _index(offsets, "offsets", E + 1, gpu)
        at = offsets.data_ptr()
    elif E != 1:
        _refuse("more than one matrix needs offsets")
    return gpu, shape[0], E, n, shape[1], at


def scaled_product(codes, scales, w_codes, w_scales, offsets=None, dtype=_BF16, stream=None):
    """Sorted e4m3 rows [R, K] times the experts' matrices [E, n, K], or all rows times [n, K] (no offsets) -> [R, n] of dtype."""
    if dtype not in _DTYPES:
        _refuse(f"dtype must be one of {sorted(map(str, _DTYPES))}")
    gpu, R, E, n, K, at = _scaled_operands(codes, scales, w_codes, w_scales, offsets)
    if stream is not None or gpu != _current_device():
        return _elsewhere(scaled_product, codes.device, stream, codes, scales, w_codes, w_scales, offsets, dtype)
    out = _empty(R, n, dtype=dtype, device=codes.device)
    rc = (moe._lib or moe.lib()).moe_scaled_product(codes.data_ptr(), scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), at, R, E, n, K,
                                                    _DTYPES[dtype], out.data_ptr(), _stream(gpu))
    if rc:
        _failed(rc, "moe_scaled_product")
    return out


def scaled_swiglu(codes, scales, w_codes, w_scales, offsets=None, stream=None):
    """Sorted e4m3 rows [R, K] times gate and up matrices [E, 2 I, K] (or [2 I, K]), silu(gate) * up -> codes [R, I], scales [R, I/128]."""
    gpu, R, E, n, K, at = _scaled_operands(codes, scales, w_codes, w_scales, offsets)
    if stream is not None or gpu != _current_device():
        return _elsewhere(scaled_swiglu, codes.device, stream, codes, scales, w_codes, w_scales, offsets)
    if n % 256 or not n:
        _refuse("the weights must have gate and up rows, a multiple of 128 each")
    out = _empty(R, n // 2, dtype=_F8, device=codes.device)
    out_scales = _empty(R, n // 256, dtype=_FP32, device=codes.device)
    rc = (moe._lib or moe.lib()).moe_scaled_swiglu(codes.data_ptr(), scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), at, R, E, n // 2, K,
                                                   out.data_ptr(), out_scales.data_ptr(), _stream(gpu))
    if rc:
        _failed(rc, "moe_scaled_swiglu")
    return out, out_scales
