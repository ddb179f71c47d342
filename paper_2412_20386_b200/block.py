"""The operators between the quantized linears of a Mamba block (the C ABI of ``include/ptq_block.h``) on torch tensors.

    x, r = block_norm(out, w, residual=r)               # norm in front of a block, the residual stream carried along
    xz = in_proj.forward(x)                             # PtqLinear
    u = short_conv(xz[..., :D], conv_w, conv_b)
    dbc = x_proj.forward(u)                             # low-rank dt, B, C
    y = gated_scan(u, delta, A, dbc[..., R:R + N], dbc[..., R + N:], D=skip, z=xz[..., D:], delta_bias=dt_bias)
    out = out_proj.forward(y)

Activations are float16, bfloat16 or float32 tensors ``[batch, length, channels]``, all of a call of one type, whose rows may
be any distance apart (slices of a projection's output); parameters and recurrent states are float32.  Gradients are explicit
calls: ``gated_scan_backward``, ``block_norm_backward`` and ``short_conv_backward`` take what the forward call took and return one
gradient per tensor that was given, dense and in its shape (for an expanded tensor one value per token: the caller sums), in a dict
by argument name; ``dy`` and the gradients of further outputs are contiguous.  They do not record anything for ``torch.autograd``.

``stream=None`` is the current stream of the tensors' device.  Outputs that are not passed are allocated by the call, on its stream;
buffers that the caller passes (``scan_history`` among them, allocated on the current stream) must not be in use on another one.
Outputs overlap no input unless a function says so.
``lengths`` (int32 ``[batch]`` on the device) makes a batch padded: rows behind a sequence's end are not read; a passed
output is left as it is there, a new one holds zeros, and gradients are zeros.
"""
from __future__ import annotations

from . import binding

FLAG_SEQ_REVERSE, FLAG_SCAN_SOFTPLUS, FLAG_CONV_SILU, FLAG_NORM_LAYER, FLAG_NORM_GATE_OUT = 2, 1, 1, 1, 2
SCAN_HISTORY = 8                  # PTQ_SCAN_HISTORY: steps between two states that the backward pass starts from


def _native():
    return binding._native_block or binding._load_native_block()


def _call(f, stream, tensor, *args):
    """An extension call on `stream` (None: the current one of the tensors' device); a status code becomes an exception."""
    if stream is None:
        r = f(*args)
    else:
        import torch
        if torch.is_tensor(tensor) and tensor.device != stream.device:
            raise ValueError("the stream belongs to another device than the tensors")
        with torch.cuda.stream(stream):
            r = f(*args)
    if r.__class__ is int:
        binding._check(r)
    return r


def scan_history(u, states: int):
    """The buffer ``[batch, ceil(length / 8), channels, states]`` that ``gated_scan`` fills for ``gated_scan_backward``."""
    import torch
    return torch.empty((u.shape[0], -(-u.shape[1] // SCAN_HISTORY), u.shape[2], states), dtype=torch.float32, device=u.device)


def gated_scan(u, delta, A, B, C, D=None, z=None, delta_bias=None, state=None, lengths=None, softplus: bool = True, reverse: bool = False,
               y=None, final_state=None, history=None, stream=None):
    """``ptq_scan_forward``: the gated linear recurrence of every channel over its sequence,

        dt = softplus(delta + delta_bias);  h <- exp(dt A) h + dt u B;  y = (C . h + D u) silu(z)

    u, delta, z ``[batch, length, channels]``; A ``[channels, states]`` (at most 32 states); B, C ``[batch, length, states]``, or
    ``[batch, length, groups, states]`` shared by channels / groups neighbouring channels each; D, delta_bias ``[channels]``.  ``state``
    ``[batch, channels, states]`` is h in front of the first step; ``final_state`` receives h behind the last one and may be ``state``
    itself.  ``reverse`` goes from the last token to the first.  ``history`` (``scan_history``) is kept for the backward pass."""
    flags = (FLAG_SCAN_SOFTPLUS if softplus else 0) | (FLAG_SEQ_REVERSE if reverse else 0)
    return _call(_native().scan, stream, u, 0, u, delta, A, B, C, D, z, delta_bias, state, lengths, flags, y, final_state, history)


def gated_scan_step(state, u, delta, A, B, C, D=None, z=None, delta_bias=None, softplus: bool = True, new_state=None, y=None, stream=None):
    """``gated_scan`` of one token per sequence: u, delta, z ``[batch, channels]``, B, C ``[batch, states]`` or ``[batch, groups, states]``.
    ``state`` is replaced unless ``new_state`` is given.  Returns y ``[batch, channels]``."""
    return _call(_native().scan, stream, u, 1, u, delta, A, B, C, D, z, delta_bias, state, None, FLAG_SCAN_SOFTPLUS if softplus else 0, y,
                 state if new_state is None else new_state, None)


def gated_scan_backward(dy, u, delta, A, B, C, history, D=None, z=None, delta_bias=None, state=None, lengths=None, softplus: bool = True,
                        reverse: bool = False, dfinal=None, stream=None):
    """``ptq_scan_backward``: gradients of ``gated_scan`` for dy and dfinal (the gradient of ``final_state``), from the ``history`` that the
    forward call filled.  ``state`` is the one that the forward call started from."""
    flags = (FLAG_SCAN_SOFTPLUS if softplus else 0) | (FLAG_SEQ_REVERSE if reverse else 0)
    g = _call(_native().scan_backward, stream, u, u, delta, A, B, C, D, z, delta_bias, state, lengths, flags, dy, history, dfinal)
    return dict(zip(("u", "delta", "A", "B", "C", "D", "z", "delta_bias", "state"), g))


def _norm_flags(kind, gate_at):
    if kind not in ("rms", "layer") or gate_at not in ("in", "out"):
        raise ValueError("kind must be 'rms' or 'layer', gate_at 'in' or 'out'")
    return (FLAG_NORM_LAYER if kind == "layer" else 0) | (FLAG_NORM_GATE_OUT if gate_at == "out" else 0)


def block_norm(x, weight=None, bias=None, residual=None, scale=None, gate=None, kind: str = "rms", gate_at: str = "in", eps: float = 1e-5, y=None,
               residual_out=None, stream=None):
    """``ptq_norm_forward`` over the last dimension (at most 8192):

        v = x silu(gate) (gate_at "in"), or x;  r = residual + scale v;  y = norm(r) weight + bias, times silu(gate) (gate_at "out")

    with the root-mean-square norm or (``kind="layer"``) the layer norm.  The residual may be float32 beside any x, and
    so may a ``residual_out`` without one.  Returns y, or (y, r) where ``residual`` or ``residual_out`` is given; ``residual_out`` may be ``residual``
    itself."""
    out, r = _call(_native().norm, stream, x, x, weight, bias, residual, scale, gate, _norm_flags(kind, gate_at), eps, y, residual_out)
    return out if r is None else (out, r)


def block_norm_backward(dy, x, weight=None, bias=None, residual=None, scale=None, gate=None, kind: str = "rms", gate_at: str = "in", eps: float = 1e-5,
                        dresidual_out=None, stream=None):
    """``ptq_norm_backward``: gradients of ``block_norm`` for dy and dresidual_out (the gradient of r, in r's type)."""
    g = _call(_native().norm_backward, stream, x, x, weight, bias, residual, scale, gate, _norm_flags(kind, gate_at), eps, dy, dresidual_out)
    return dict(zip(("x", "weight", "bias", "residual", "scale", "gate"), g))


def short_conv(x, weight, bias=None, state=None, lengths=None, silu: bool = True, reverse: bool = False, y=None, final_state=None, stream=None):
    """``ptq_conv_forward``: causal depthwise convolution over the tokens, x ``[batch, length, channels]``, weight ``[channels, taps]``
    (2 to 4 taps, the last one for the token itself), followed by silu.  ``state`` ``[batch, taps - 1, channels]`` holds the rows in front of
    the first step; ``final_state`` receives the last rows and may be ``state`` itself: one token of a generating model is a call of
    length 1."""
    flags = (FLAG_CONV_SILU if silu else 0) | (FLAG_SEQ_REVERSE if reverse else 0)
    return _call(_native().conv, stream, x, x, weight, bias, state, lengths, flags, y, final_state)


def short_conv_backward(dy, x, weight, bias=None, state=None, lengths=None, silu: bool = True, reverse: bool = False, dfinal=None, stream=None):
    """``ptq_conv_backward``: gradients of ``short_conv`` for dy and dfinal (the gradient of ``final_state``)."""
    flags = (FLAG_CONV_SILU if silu else 0) | (FLAG_SEQ_REVERSE if reverse else 0)
    g = _call(_native().conv_backward, stream, x, x, weight, bias, state, lengths, flags, dy, dfinal)
    return dict(zip(("x", "weight", "bias", "state"), g))
