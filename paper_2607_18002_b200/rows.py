"""The rows of a routed layer as tensors: sorted by expert and put together again, their gradients, the router's gradient, and the
experts in 4 bits (moe_sort_rows ... moe_mx_swiglu of include/moe_apk.h).

Checks of arguments and marshalling only; a call enqueues one kernel on `stream` (the current stream of the tensors' device if
None) and allocates its outputs there.  Nothing is recorded for autograd: gradients are calls of their own.  Wrong types, shapes, strides
or devices raise ValueError, what the library refuses MoeError.  Inputs may require gradients (experts' outputs of a graph of the caller's own do); results never do.
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


def _rows(t, name, dtypes):
    """[n, H] with neighbouring columns -> n, H, elements from a row to the next."""
    if not isinstance(t, _Tensor) or t.dtype not in dtypes or not t.is_cuda or t.dim() != 2:
        _refuse(f"{name} must be a CUDA tensor [rows, columns] of one of {sorted(map(str, dtypes))}")
    n, h = t.shape
    step, one = t.stride()
    if h < 1 or (one != 1 and h > 1) or (n > 1 and step < h):
        _refuse(f"{name}: the columns of a row must be neighbours and rows must not overlap")
    return n, h, step if step > h else h


def _plain(t, name, dtype, shape, gpu):
    """A contiguous tensor of this type and shape on GPU number `gpu`."""
    if not isinstance(t, _Tensor) or t.dtype is not dtype or t.shape != shape or t.get_device() != gpu or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous {dtype} tensor {tuple(shape)} on cuda:{gpu}")


def _index(t, name, n, gpu):
    if not isinstance(t, _Tensor) or t.dtype is not _I32 or t.get_device() != gpu or not t.is_contiguous() \
            or t.numel() != n and (n or t.numel() != 1):                # (a plan without rows has arrays of one entry)
        _refuse(f"{name} must be a contiguous int32 tensor of {n} on cuda:{gpu}")


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
