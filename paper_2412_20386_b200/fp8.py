"""Linears in 8-bit floating point (e4m3) with a scale for each block of 128 (the C ABI of ``include/ptq_fp8.h``) on torch tensors.

    w8, ws = fp8_quantize_weight(w)                     # once per layer: codes [N, K], scales [ceil(N/128), ceil(K/128)]
    y = fp8_linear(x, w8, ws, bias)                     # quantizes x [..., K] and multiplies
    a8, sa = fp8_quantize(x)                            # or once for several layers that read x
    q, k = fp8_matmul(a8, sa, wq8, wqs), fp8_matmul(a8, sa, wk8, wks)

Beside the int8 linears of ``PtqLinear`` these need no calibration and no step size per token position: the scales are found from
the data of each call.  x is float16, bfloat16 or float32, its rows any distance apart; codes are ``torch.float8_e4m3fn`` with rows
on 16-byte boundaries (new ones are made so; a tensor from elsewhere whose K is no multiple of 16 needs a wider row pitch).

``stream=None`` is the current stream of the tensors' device.  Outputs that are not passed are allocated by the call, on its stream.
Outputs overlap no input.
"""
from __future__ import annotations

import ctypes

from . import binding
from .block import _call

FP8_BLOCK = 128                   # PTQ_FP8_BLOCK: values of a row that share a scale

_bound = None


def _native():
    global _bound
    if _bound is None:
        L, native = binding.load_library(), binding._load_native()
        L.ptq_fp8_linear_workspace_bytes.restype = ctypes.c_size_t
        native.bind_fp8(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
            L.ptq_fp8_quantize, L.ptq_fp8_quantize_weight, L.ptq_fp8_matmul, L.ptq_fp8_linear_workspace_bytes, L.ptq_fp8_linear)))
        _bound = native
    return _bound


def fp8_quantize(x, codes=None, scales=None, stream=None):
    """``ptq_fp8_quantize``: x ``[..., K]`` -> codes ``[..., K]`` and float32 scales ``[..., ceil(K/128)]``,

        top = max(2^-100, max |x| of 128 neighbouring values);  scale = top / 448;  code = e4m3(x (448 / top))

    Scales that are not passed lie with those of one block next to each other (strides 1 over the rows)."""
    return _call(_native().fp8_quantize, stream, x, x, codes, scales)


def fp8_quantize_weight(w, stream=None):
    """``ptq_fp8_quantize_weight``: w ``[N, K]`` -> codes ``[N, K]`` and scales ``[ceil(N/128), ceil(K/128)]``, one for 128 x 128 values."""
    return _call(_native().fp8_quantize_weight, stream, w, w)


def _code(dtype):
    import torch
    codes = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
    if dtype not in codes:
        raise ValueError("dtype must be float16, bfloat16 or float32")
    return codes[dtype]


def fp8_matmul(a, a_scales, w, w_scales, bias=None, dtype=None, y=None, stream=None):
    """``ptq_fp8_matmul``: y ``[..., N]`` of ``dtype`` (y's, where it is passed; else bfloat16) from codes a ``[..., K]``, w ``[N, K]`` and
    their scales, ``bias`` float32 ``[N]``.  The products of a block are summed in float32 before the scales multiply them."""
    if dtype is None:
        import torch
        dtype = torch.bfloat16 if y is None else y.dtype
    return _call(_native().fp8_matmul, stream, a, a, a_scales, w, w_scales, bias, _code(dtype), y)


def fp8_linear(x, w, w_scales, bias=None, y=None, stream=None):
    """``ptq_fp8_linear``: ``fp8_quantize`` and ``fp8_matmul`` in one call, y ``[..., N]`` of x's type; up to 16 rows in one kernel."""
    return _call(_native().fp8_linear, stream, x, x, w, w_scales, bias, y)


def fp8_device_status():
    """Raises ``PtqError`` if a kernel of these operators gave up a bounded wait on the current device since the last call; waits for
    the device."""
    binding._check(binding.load_library().ptq_fp8_device_status())
