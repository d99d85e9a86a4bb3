"""The rows of a routed layer as tensors: sorted by expert and put together again, their gradients, the router's gradient, and the
experts in 4 bits (moe_sort_rows ... moe_mx_swiglu of include/moe_apk.h).

Checks of arguments and marshalling only; a call enqueues one kernel on `stream` (the current stream of the tensors' device if
None) and allocates its outputs there.  Wrong types, shapes, strides or devices raise ValueError, what the library refuses MoeError.
A permutation is the pair (sorted_to_flat, flat_to_sorted) of a plan, int32 [T*k] each.

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

import contextlib

import torch

import paper_2607_18002_b200 as moe

_DTYPES = {torch.bfloat16: moe.MOE_DTYPE_BF16, torch.float16: moe.MOE_DTYPE_FP16, torch.float32: moe.MOE_DTYPE_FP32}
_SORTED_DTYPES = {**_DTYPES, torch.float8_e4m3fn: moe.MOE_DTYPE_FP8_E4M3, torch.uint8: moe.MOE_DTYPE_FP8_E4M3}


def _refuse(what):
    raise ValueError(what)


def _rows(t, name, dtypes, device=None, dtype=None):
    """[n, H] with neighbouring columns -> elements from a row to the next."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2 or t.dtype not in dtypes or not t.is_cuda:
        _refuse(f"{name} must be a CUDA tensor [rows, columns] of one of {sorted(map(str, dtypes))}")
    if (device is not None and t.device != device) or (dtype is not None and t.dtype != dtype):
        _refuse(f"{name} must be on {device} with {dtype}, as the other rows")
    n, h = t.shape
    if h < 1 or (t.stride(1) != 1 and h > 1) or (n > 1 and t.stride(0) < h):
        _refuse(f"{name}: the columns of a row must be neighbours and rows must not overlap")
    return max(t.stride(0), h)


def _plain(t, name, dtype, shape, device):
    """A contiguous tensor of this type and shape."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or tuple(t.shape) != shape or t.device != device or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous {dtype} tensor {shape} on {device}")


def _index(t, name, n, device):
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or t.dim() != 1 or t.device != device or not t.is_contiguous() \
            or t.shape[0] != n and (n or t.shape[0] != 1):              # (a plan without rows has arrays of one entry)
        _refuse(f"{name} must be a contiguous int32 tensor [{n}] on {device}")


@contextlib.contextmanager
def _elsewhere(device, stream):
    with torch.cuda.device(device):
        if stream is None:
            yield
        else:
            with torch.cuda.stream(stream):
                yield


_here = contextlib.nullcontext()


def _on(device, stream):
    """The device current and `stream` its current stream: outputs are allocated there and the kernel is enqueued there."""
    if stream is None and device.index == torch.cuda.current_device():
        return _here
    if stream is not None and stream.device != device:
        _refuse(f"the stream is on {stream.device}, the tensors are on {device}")
    return _elsewhere(device, stream)


def _go(name, *args):
    rc = getattr(moe._lib or moe.lib(), name)(*args, moe.Context._stream(None))
    if rc:
        raise moe.MoeError(rc, name)


def sort_rows(x, sorted_to_flat, flat_to_sorted, top_k: int, stream=None):
    """x [T, H] -> [T*k, H], the tokens' rows by expert (bf16, fp16, fp32, or one-byte codes)."""
    stride = _rows(x, "x", _SORTED_DTYPES)
    (T, H), dev = x.shape, x.device
    _index(sorted_to_flat, "sorted_to_flat", T * top_k, dev)
    _index(flat_to_sorted, "flat_to_sorted", T * top_k, dev)
    with _on(dev, stream):
        xs = torch.empty((T * top_k, H), dtype=x.dtype, device=dev)
        _go("moe_sort_rows", x.data_ptr(), stride, _SORTED_DTYPES[x.dtype], T, top_k, H, sorted_to_flat.data_ptr(),
            flat_to_sorted.data_ptr(), xs.data_ptr())
    return xs


def sort_rows_grad(dxs, flat_to_sorted, top_k: int, stream=None):
    """dxs [T*k, H], the gradient of sort_rows' result -> that of x [T, H]."""
    stride = _rows(dxs, "dxs", _DTYPES)
    (R, H), dev = dxs.shape, dxs.device
    if top_k < 1 or R % top_k:
        _refuse("dxs must have top_k rows for every token")
    _index(flat_to_sorted, "flat_to_sorted", R, dev)
    with _on(dev, stream):
        dx = torch.empty((R // top_k, H), dtype=dxs.dtype, device=dev)
        _go("moe_sort_rows_grad", dxs.data_ptr(), stride, _DTYPES[dxs.dtype], R // top_k, top_k, H, flat_to_sorted.data_ptr(), dx.data_ptr())
    return dx


def _weights(topk_w, R, dev):
    if not isinstance(topk_w, torch.Tensor) or topk_w.dim() != 2 or topk_w.numel() != R:
        _refuse("topk_w must be fp32 [T, k], a weight for every row")
    _plain(topk_w, "topk_w", torch.float32, tuple(topk_w.shape), dev)
    return topk_w.shape


def merge_rows(rows, flat_to_sorted, topk_w, stream=None):
    """rows [T*k, H] by expert -> y [T, H], the tokens' rows added up with their router weights."""
    stride = _rows(rows, "rows", _DTYPES)
    (R, H), dev = rows.shape, rows.device
    T, k = _weights(topk_w, R, dev)
    _index(flat_to_sorted, "flat_to_sorted", R, dev)
    with _on(dev, stream):
        y = torch.empty((T, H), dtype=rows.dtype, device=dev)
        _go("moe_merge_rows", rows.data_ptr(), stride, _DTYPES[rows.dtype], topk_w.data_ptr(), T, k, H, flat_to_sorted.data_ptr(), y.data_ptr())
    return y


def merge_rows_grad(dy, rows, sorted_to_flat, flat_to_sorted, topk_w, stream=None):
    """dy [T, H], the gradient of merge_rows' result -> (that of rows [T*k, H], that of topk_w [T, k] fp32)."""
    stride = _rows(rows, "rows", _DTYPES)
    (R, H), dev = rows.shape, rows.device
    dy_stride = _rows(dy, "dy", _DTYPES, dev, rows.dtype)
    T, k = _weights(topk_w, R, dev)
    if tuple(dy.shape) != (T, H):
        _refuse(f"dy must be [{T}, {H}]")
    _index(sorted_to_flat, "sorted_to_flat", R, dev)
    _index(flat_to_sorted, "flat_to_sorted", R, dev)
    with _on(dev, stream):
        drows = torch.empty((R, H), dtype=rows.dtype, device=dev)
        dw = torch.empty((T, k), dtype=torch.float32, device=dev)
        _go("moe_merge_rows_grad", dy.data_ptr(), dy_stride, rows.data_ptr(), stride, _DTYPES[rows.dtype], topk_w.data_ptr(), T, k, H,
            sorted_to_flat.data_ptr(), flat_to_sorted.data_ptr(), drows.data_ptr(), dw.data_ptr())
    return drows, dw


def route_grad(topk_ids, topk_w, d_topk_w, n_experts: int, stream=None):
    """The gradient of route's weights, fp32 [T, k] -> that of the logits, fp32 [T, E]."""
    if not isinstance(topk_ids, torch.Tensor) or not topk_ids.is_cuda or topk_ids.dim() != 2:
        _refuse("topk_ids must be a CUDA int32 tensor [T, k]")
    shape, dev = tuple(topk_ids.shape), topk_ids.device
    _plain(topk_ids, "topk_ids", torch.int32, shape, dev)
    _plain(topk_w, "topk_w", torch.float32, shape, dev)
    _plain(d_topk_w, "d_topk_w", torch.float32, shape, dev)
    with _on(dev, stream):
        dz = torch.empty((shape[0], n_experts), dtype=torch.float32, device=dev)
        _go("moe_route_grad", topk_ids.data_ptr(), topk_w.data_ptr(), d_topk_w.data_ptr(), shape[0], n_experts, shape[1], dz.data_ptr())
    return dz


def mx_quantize(x, sorted_to_flat=None, flat_to_sorted=None, top_k: int = 1, stream=None):
    """x [..., K] -> codes uint8 [..., K/2], scales uint8 [..., K/32]; with a permutation x [T, K] -> the T*k rows by expert."""
    lead = None
    if isinstance(x, torch.Tensor) and x.dim() > 2 and x.is_contiguous() and sorted_to_flat is None and flat_to_sorted is None:
        lead, x = x.shape[:-1], x.view(-1, x.shape[-1])
    stride = _rows(x, "x", _DTYPES)
    (T, K), dev = x.shape, x.device
    if K % 32:
        _refuse("x must have a multiple of 32 columns")
    s2f = f2s = None
    if sorted_to_flat is not None or flat_to_sorted is not None:
        _index(sorted_to_flat, "sorted_to_flat", T * top_k, dev)
        _index(flat_to_sorted, "flat_to_sorted", T * top_k, dev)
        s2f, f2s = sorted_to_flat.data_ptr(), flat_to_sorted.data_ptr()
    elif top_k != 1:
        _refuse("top_k needs a permutation")
    with _on(dev, stream):
        codes = torch.empty((T * top_k, K // 2), dtype=torch.uint8, device=dev)
        scales = torch.empty((T * top_k, K // 32), dtype=torch.uint8, device=dev)
        _go("moe_mx_quantize", x.data_ptr(), stride, _DTYPES[x.dtype], T, top_k, K, s2f, f2s, codes.data_ptr(), scales.data_ptr())
    return (codes, scales) if lead is None else (codes.view(*lead, -1), scales.view(*lead, -1))


def _mx(codes, scales, names, dims, device=None):
    """codes [..., K/2] and scales [..., K/32] -> K."""
    if not isinstance(codes, torch.Tensor) or codes.dtype != torch.uint8 or not codes.is_cuda or not codes.is_contiguous() \
            or (dims and codes.dim() != dims) or codes.dim() < 1 or codes.shape[-1] % 16 or (device is not None and codes.device != device):
        _refuse(f"{names[0]} must be a contiguous CUDA uint8 tensor of {dims or 'some'} dimensions, a multiple of 16 bytes wide")
    _plain(scales, names[1], torch.uint8, (*codes.shape[:-1], codes.shape[-1] // 16), codes.device)
    return codes.shape[-1] * 2


def mx_dequantize(codes, scales, dtype=torch.bfloat16, stream=None):
    """The values [..., K] that codes [..., K/2] with scales [..., K/32] stand for."""
    if dtype not in _DTYPES:
        _refuse(f"dtype must be one of {sorted(map(str, _DTYPES))}")
    K = _mx(codes, scales, ("codes", "scales"), 0)
    with _on(codes.device, stream):
        out = torch.empty((*codes.shape[:-1], K), dtype=dtype, device=codes.device)
        if K:
            _go("moe_mx_dequantize", codes.data_ptr(), scales.data_ptr(), out.numel() // K, K, _DTYPES[dtype], out.data_ptr())
    return out


def _operands(codes, scales, w_codes, w_scales, offsets):
    K = _mx(codes, scales, ("codes", "scales"), 2)
    dev = codes.device
    if _mx(w_codes, w_scales, ("w_codes", "w_scales"), 3, dev) != K:
        _refuse("w_codes must be as wide as codes")
    E, n, _ = w_codes.shape
    _index(offsets, "offsets", E + 1, dev)
    return codes.shape[0], E, n, K


def mx_product(codes, scales, w_codes, w_scales, offsets, stream=None):
    """Sorted 4-bit rows [R, K] times the experts' matrices [E, n, K] -> bf16 [R, n]."""
    R, E, n, K = _operands(codes, scales, w_codes, w_scales, offsets)
    with _on(codes.device, stream):
        out = torch.empty((R, n), dtype=torch.bfloat16, device=codes.device)
        _go("moe_mx_product", codes.data_ptr(), scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), offsets.data_ptr(), R, E, n, K,
            out.data_ptr())
    return out


def mx_swiglu(codes, scales, w_codes, w_scales, offsets, stream=None):
    """Sorted 4-bit rows [R, K] times gate and up matrices [E, 2 I, K], silu(gate) * up -> codes [R, I/2], scales [R, I/32]."""
    R, E, n, K = _operands(codes, scales, w_codes, w_scales, offsets)
    if n % 64:
        _refuse("w_codes must have gate and up rows, a multiple of 32 each")
    with _on(codes.device, stream):
        out = torch.empty((R, n // 4), dtype=torch.uint8, device=codes.device)
        out_scales = torch.empty((R, n // 64), dtype=torch.uint8, device=codes.device)
        _go("moe_mx_swiglu", codes.data_ptr(), scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), offsets.data_ptr(), R, E, n // 2, K,
            out.data_ptr(), out_scales.data_ptr())
    return out, out_scales
