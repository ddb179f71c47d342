"""Linear attention with a decay for each head (the C ABI of ``include/ptq_heads.h``) on torch tensors: the recurrence of blocks whose state
is a matrix per head, beside ``gated_scan``, which has one decay per channel and state.

    xbc = short_conv(zx[..., D:], conv_w, conv_b)                          # u, B and C next to each other
    u = xbc[..., :D].unflatten(-1, (H, P))
    y = head_scan(u, delta, A, xbc[..., D:D + N], xbc[..., D + N:], D=skip, delta_bias=dt_bias)
    y = block_norm(y.flatten(-2), w, gate=zx[..., :D])                     # the gate, and the norm in front of out_proj

Activations are float16, bfloat16 or float32, all of a call of one type, the columns of a head (of a group of B and C) next to each other and
everything else any distance apart; parameters and states are float32.  Gradients are explicit calls: ``head_scan_backward`` takes what the
forward call took and returns one gradient per tensor that was given, dense and in its shape, in a dict by argument name.  It does
not record anything for ``torch.autograd``.

``stream=None`` is the current stream of the tensors' device.  Outputs that are not passed are allocated by the call, on its stream; buffers
that the caller passes must not be in use on another one.  Outputs overlap no input unless a function says so.  ``lengths`` as in ``block``:
rows behind a sequence's end are not read, a passed output is left as it is there, a new one holds zeros, and gradients are zeros.
"""
from __future__ import annotations

import ctypes

from . import binding
from .block import FLAG_SEQ_REVERSE, _call

FLAG_HEADS_SOFTPLUS, FLAG_HEADS_UNSCALED = 1, 4
HEADS_HISTORY = 64                # PTQ_HEADS_HISTORY: steps between two states that the backward pass starts from

_bound = None


def _native():
    global _bound
    if _bound is None:
        L, native = binding.load_library(), binding._load_native()
        native.bind_heads(*(ctypes.cast(f, ctypes.c_void_p).value for f in (L.ptq_heads_workspace_bytes, L.ptq_heads_forward, L.ptq_heads_backward)))
        _bound = native
    return _bound


def _flags(softplus, scale_input, reverse=False):
    return (FLAG_HEADS_SOFTPLUS if softplus else 0) | (0 if scale_input else FLAG_HEADS_UNSCALED) | (FLAG_SEQ_REVERSE if reverse else 0)


def head_scan_history(u, states: int):
    """The buffer ``[batch, ceil(length / 64), heads, columns, states]`` that ``head_scan`` fills for ``head_scan_backward``."""
    import torch
    return torch.empty((u.shape[0], -(-u.shape[1] // HEADS_HISTORY), u.shape[2], u.shape[3], states), dtype=torch.float32, device=u.device)


def head_scan(u, delta, A, B, C, D=None, delta_bias=None, state=None, lengths=None, softplus: bool = True, scale_input: bool = True,
              reverse: bool = False, y=None, final_state=None, history=None, stream=None):
    """``ptq_heads_forward``: for every head the recurrence of a matrix S over its sequence,

        dt = softplus(delta + delta_bias);  S <- exp(dt A) S + dt u B^T;  y = S C + D u

    u ``[batch, length, heads, columns]`` (at most 256 columns); delta ``[batch, length, heads]``, or None for a fixed decay (dt = 1);
    A, D, delta_bias ``[heads]``; B, C ``[batch, length, states]`` (at most 128), or ``[batch, length, groups, states]`` shared by heads / groups
    neighbouring heads each.  With ``scale_input=False`` the input is u B^T: linear attention with queries C, keys B, values u and decay
    exp(dt A).  ``state`` ``[batch, heads, columns, states]`` is S in front of the first step; ``final_state`` receives S behind the last
    one and may be ``state`` itself.  ``reverse`` goes from the last token to the first.  ``history`` (``head_scan_history``) is kept for the
    backward pass."""
    return _call(_native().heads, stream, u, 0, u, delta, A, B, C, D, delta_bias, state, lengths, _flags(softplus, scale_input, reverse), y, final_state, history)


def head_scan_step(state, u, delta, A, B, C, D=None, delta_bias=None, softplus: bool = True, scale_input: bool = True, new_state=None, y=None,
                   stream=None):
    """``head_scan`` of one token per sequence, in float32 throughout: u ``[batch, heads, columns]``, delta ``[batch, heads]`` or None, B, C
    ``[batch, states]`` or ``[batch, groups, states]``.  ``state`` is replaced unless ``new_state`` is given.  Returns y like u."""
    return _call(_native().heads, stream, u, 1, u, delta, A, B, C, D, delta_bias, state, None, _flags(softplus, scale_input), y,
                 state if new_state is None else new_state, None)


def head_scan_backward(dy, u, delta, A, B, C, history, D=None, delta_bias=None, state=None, lengths=None, softplus: bool = True, scale_input: bool = True,
                       reverse: bool = False, dfinal=None, stream=None):
    """``ptq_heads_backward``: gradients of ``head_scan`` for dy and dfinal (the gradient of ``final_state``), from the ``history`` that the
    forward call filled.  ``state`` is the one that the forward call started from.  The call takes about 8 bytes of memory for each token, head and state
    (and each 64 columns of a head) while it runs."""
    g = _call(_native().heads_backward, stream, u, u, delta, A, B, C, D, delta_bias, state, lengths, _flags(softplus, scale_input, reverse), dy, history, dfinal)
    return dict(zip(("u", "delta", "A", "B", "C", "D", "delta_bias", "state"), g))
