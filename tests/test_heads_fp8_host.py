"""The C ABIs of include/ptq_heads.h and include/ptq_fp8.h and the binding's checks, as far as they need no GPU."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import __graft_entry__ as entry

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
vp, ci, i64, u32, size_t = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint, ctypes.c_size_t
NULL, SHAPE, VALUE, ALIGN, ARCH, CUDA = 1, 2, 3, 4, 5, 6


class Heads(ctypes.Structure):
    _fields_ = [("dtype", ci), ("batch", ci), ("length", ci), ("heads", ci), ("cols", ci), ("states", ci), ("groups", ci), ("flags", u32), ("u", vp),
                ("delta", vp), ("B", vp), ("C", vp), ("u_pitch", i64 * 3), ("B_pitch", i64 * 3), ("C_pitch", i64 * 3), ("delta_pitch", i64 * 3),
                ("A", vp), ("D", vp), ("delta_bias", vp), ("state", vp), ("lengths", vp)]


class Input(ctypes.Structure):
    _fields_ = [("dtype", ci), ("cols", ci), ("rows", i64), ("x", vp), ("x_pitch", i64)]


class Weight(ctypes.Structure):
    _fields_ = [("cols", ci), ("outputs", ci), ("codes", vp), ("codes_pitch", i64), ("scales", vp), ("bias", vp)]


P = 4096                                                     # a device address that no host code looks at


def filled(s, kw):
    for k, v in kw.items():
        setattr(s, k, (type(getattr(s, k)))(*v) if isinstance(v, tuple) else v)
    return s


def heads(**kw):
    return filled(Heads(dtype=0, batch=2, length=100, heads=4, cols=16, states=8, groups=2, u=P, delta=P, B=P, C=P, A=P), kw)


def inp(**kw):
    return filled(Input(dtype=0, cols=100, rows=3, x=P, x_pitch=100), kw)


def weight(**kw):
    return filled(Weight(cols=100, outputs=50, codes=P, codes_pitch=112, scales=P), kw)


@pytest.fixture(scope="module")
def lib():
    entry.build()
    from paper_2412_20386_b200 import binding
    L = binding.load_library()
    L.ptq_heads_workspace_bytes.restype = L.ptq_fp8_linear_workspace_bytes.restype = size_t
    return L


@pytest.mark.parametrize("header,count", [("ptq_heads.h", 3), ("ptq_fp8.h", 6)])
def test_library_exports_every_declared_symbol(lib, header, count):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ptq_[a-z_0-9]+)\s*\(", text)))
    assert len(names) == count
    for n in names:
        assert hasattr(lib, n), n


def forward(lib, s, y=P, final=None, history=None, ws=P, nbytes=1 << 40):
    return lib.ptq_heads_forward(ctypes.byref(s) if s is not None else None, vp(y), vp(final), vp(history), vp(ws), size_t(nbytes), None)


def backward(lib, s, g=(P,) * 8, history=P, dy=P, ws=P, nbytes=1 << 40):
    return lib.ptq_heads_backward(ctypes.byref(s), vp(history), vp(dy), None, (vp * 8)(*g) if g else None, vp(ws), size_t(nbytes), None)


def test_heads_refusals(lib):
    assert forward(lib, None) == NULL and forward(lib, heads(), y=None) == NULL
    for k in ("u", "B", "C", "A"):
        assert forward(lib, heads(**{k: None})) == NULL, k
    assert forward(lib, heads(delta=None, delta_bias=P)) == NULL
    for kw in (dict(batch=0), dict(length=0), dict(length=(1 << 30) + 1), dict(heads=0), dict(heads=4097), dict(cols=0), dict(cols=257), dict(states=0),
               dict(states=129), dict(groups=0), dict(groups=3), dict(u_pitch=(0, -1, 0)), dict(C_pitch=(0, 0, -1)), dict(delta_pitch=(-1, 0, 0)),
               dict(batch=2 ** 31 - 1, heads=4096)):
        assert forward(lib, heads(**kw)) == SHAPE, kw
    for kw in (dict(dtype=3), dict(flags=8)):
        assert forward(lib, heads(**kw)) == VALUE, kw
    for kw in (dict(u=P + 1), dict(A=P + 2), dict(state=P + 2), dict(lengths=P + 1), dict(delta=P + 1)):
        assert forward(lib, heads(**kw)) == ALIGN, kw
    assert forward(lib, heads(), y=P + 1) == ALIGN and forward(lib, heads(), final=P + 2) == ALIGN and forward(lib, heads(), history=P + 2) == ALIGN
    long = heads(batch=1, length=20000, heads=2)
    need = lib.ptq_heads_workspace_bytes(ctypes.byref(long), 0)
    assert need > 0 and forward(lib, long, ws=None) == NULL and forward(lib, long, nbytes=need - 1) == SHAPE and forward(lib, long, ws=P + 8) == ALIGN
    assert lib.ptq_heads_workspace_bytes(None, 0) == 0 and lib.ptq_heads_workspace_bytes(ctypes.byref(heads(groups=3)), 1) == 0


def test_heads_backward_refusals(lib):
    assert backward(lib, heads(), history=None) == NULL and backward(lib, heads(), dy=None) == NULL and backward(lib, heads(), g=None) == NULL
    for i in (0, 1, 2, 3, 4):                                # du, ddelta (where delta is given), dB, dC, dA
        assert backward(lib, heads(), g=tuple(None if k == i else P for k in range(8))) == NULL, i
    assert backward(lib, heads(delta=None)) == NULL          # ddelta without delta
    assert backward(lib, heads(), g=(P + 1,) + (P,) * 7) == ALIGN and backward(lib, heads(), g=(P,) * 7 + (P + 2,)) == ALIGN
    need = lib.ptq_heads_workspace_bytes(ctypes.byref(heads()), 1)
    assert need > 0 and backward(lib, heads(), nbytes=need - 1) == SHAPE and backward(lib, heads(), ws=None) == NULL


def test_workspaces_grow_with_the_call_and_never_overflow(lib):
    for kw in (dict(), dict(batch=128, length=197, heads=12, cols=64, states=128), dict(batch=1, length=1 << 30, heads=4096, cols=256, states=128),
               dict(batch=2 ** 31 - 1, length=1 << 30, heads=4096, cols=256, states=128, groups=4096)):
        s = heads(**kw)
        fwd, bwd = (lib.ptq_heads_workspace_bytes(ctypes.byref(s), k) for k in (0, 1))
        assert bwd >= fwd and bwd >= min(8 * s.batch * s.length * s.heads * s.states, 1 << 60), kw
    assert lib.ptq_fp8_linear_workspace_bytes(i64(1), 768, 384) == 0
    assert lib.ptq_fp8_linear_workspace_bytes(i64(1 << 30), 65536, 1 << 20) >= 1 << 46
    for bad in ((0, 8, 8), (8, 0, 8), (8, 8, 0), (8, 65537, 8)):
        assert lib.ptq_fp8_linear_workspace_bytes(i64(bad[0]), *bad[1:]) == 0


def test_fp8_refusals(lib):
    sp = (i64 * 2)(1, 3)
    q = lambda x, codes=P, pitch=112, scales=P, s=sp: lib.ptq_fp8_quantize(ctypes.byref(x) if x is not None else None, vp(codes), i64(pitch), vp(scales), s, None)
    assert q(None) == NULL and q(inp(x=None)) == NULL and q(inp(), codes=None) == NULL and q(inp(), scales=None) == NULL and q(inp(), s=None) == NULL
    for kw in (dict(rows=0), dict(rows=(1 << 30) + 1), dict(cols=0), dict(cols=65537), dict(x_pitch=-1)):
        assert q(inp(**kw)) == SHAPE, kw
    assert q(inp(dtype=4)) == VALUE and q(inp(x=P + 1)) == ALIGN and q(inp(), codes=P + 8) == ALIGN and q(inp(), pitch=100) == ALIGN and q(inp(), scales=P + 2) == ALIGN
    assert q(inp(), pitch=96) == SHAPE and q(inp(), s=(i64 * 2)(-1, 0)) == SHAPE and q(inp(), pitch=1 << 41) == SHAPE
    w = lambda x, codes=P, pitch=112, scales=P: lib.ptq_fp8_quantize_weight(ctypes.byref(x), vp(codes), i64(pitch), vp(scales), None)
    assert w(inp(rows=(1 << 20) + 1)) == SHAPE and w(inp(), scales=None) == NULL and w(inp(), pitch=104) == ALIGN

    def mm(d=weight(), rows=3, a=P, a_pitch=112, sa=P, s=sp, y=P, y_dtype=1, y_pitch=50):
        return lib.ptq_fp8_matmul(ctypes.byref(d) if d is not None else None, i64(rows), vp(a), i64(a_pitch), vp(sa), s, vp(y), y_dtype, i64(y_pitch), None)
    assert mm(d=None) == NULL and mm(d=weight(codes=None)) == NULL and mm(d=weight(scales=None)) == NULL and mm(a=None) == NULL and mm(sa=None) == NULL
    assert mm(y=None) == NULL and mm(s=None) == NULL
    assert mm(rows=0) == SHAPE and mm(y_pitch=49) == SHAPE and mm(d=weight(outputs=0)) == SHAPE and mm(d=weight(outputs=(1 << 20) + 1)) == SHAPE
    assert mm(d=weight(cols=65537)) == SHAPE and mm(a_pitch=96) == SHAPE
    assert mm(y_dtype=5) == VALUE and mm(d=weight(codes=P + 8)) == ALIGN and mm(d=weight(codes_pitch=104)) == ALIGN and mm(y=P + 1) == ALIGN
    assert mm(d=weight(bias=P + 2)) == ALIGN and mm(a=P + 4) == ALIGN and mm(sa=P + 1) == ALIGN

    def linear(d=weight(), x=inp(rows=100), y=P, pitch=50, ws=P, n=1 << 40):
        return lib.ptq_fp8_linear(ctypes.byref(d), ctypes.byref(x), vp(y), i64(pitch), vp(ws), size_t(n), None)
    need = lib.ptq_fp8_linear_workspace_bytes(i64(100), 100, 50)
    assert need >= 100 * 112 + 400 and linear(n=need - 1) == SHAPE and linear(ws=None) == NULL and linear(ws=P + 8) == ALIGN
    assert linear(x=inp(cols=96, rows=100)) == SHAPE and linear(y=None) == NULL and linear(pitch=1) == SHAPE


def test_fp8_scales_that_are_written_do_not_overlap(lib):
    q = lambda x, pitches: lib.ptq_fp8_quantize(ctypes.byref(x), vp(P), i64(x.cols + 15 & ~15), vp(P), (i64 * 2)(*pitches), None)
    assert q(inp(rows=3, cols=100), (0, 1)) == SHAPE and q(inp(rows=1, cols=300), (1, 0)) == SHAPE
    if not torch.cuda.is_available():                        # a single row, a single block: any pitch will do
        assert q(inp(rows=1, cols=300), (0, 1)) in (ARCH, CUDA) and q(inp(rows=3, cols=100), (1, 0)) in (ARCH, CUDA)


def test_without_a_device_a_good_call_fails_with_an_error_code(lib):
    if torch.cuda.is_available():
        pytest.skip("a CUDA device is present")
    sp = (i64 * 2)(1, 3)
    assert forward(lib, heads()) in (ARCH, CUDA) and forward(lib, heads(delta=None)) in (ARCH, CUDA) and backward(lib, heads()) in (ARCH, CUDA)
    assert lib.ptq_fp8_quantize(ctypes.byref(inp()), vp(P), i64(112), vp(P), sp, None) in (ARCH, CUDA)
    assert lib.ptq_fp8_matmul(ctypes.byref(weight()), i64(3), vp(P), i64(112), vp(P), sp, vp(P), 1, i64(50), None) in (ARCH, CUDA)
    assert lib.ptq_fp8_linear(ctypes.byref(weight()), ctypes.byref(inp()), vp(P), i64(50), None, size_t(0), None) in (ARCH, CUDA)
    assert lib.ptq_fp8_device_status() in (ARCH, CUDA)


@pytest.mark.parametrize("module,name,n", [("heads", "heads", 14), ("heads", "heads_backward", 13), ("fp8", "fp8_quantize", 3), ("fp8", "fp8_quantize_weight", 1),
                                           ("fp8", "fp8_matmul", 7), ("fp8", "fp8_linear", 5)])
def test_the_binding_refuses_wrong_objects_before_the_library_is_called(module, name, n):
    entry.build()
    import importlib
    f = getattr(importlib.import_module("paper_2412_20386_b200." + module)._native(), name)
    first = [0] if name == "heads" else []
    rest = [None] * (n - 1 - len(first))
    with pytest.raises(TypeError):
        f(*[None] * (n + 1))
    with pytest.raises(TypeError):
        f(*first, None, *rest)
    with pytest.raises(TypeError):
        f(*first, np.zeros((1, 1, 1, 1), np.float16), *rest)
    with pytest.raises(ValueError):
        f(*first, torch.zeros(1, 1, 1, 1), *rest)


def test_constants_agree_with_the_headers():
    from paper_2412_20386_b200 import block, fp8, heads as h
    value = lambda header, name: int(re.search(r"#define %s\s+(\d+)u?" % name, open(os.path.join(ROOT, "include", header)).read()).group(1))
    assert (value("ptq_heads.h", "PTQ_HEADS_SOFTPLUS"), value("ptq_heads.h", "PTQ_HEADS_UNSCALED"), value("ptq_heads.h", "PTQ_HEADS_HISTORY"),
            value("ptq_block.h", "PTQ_SEQ_REVERSE")) == (h.FLAG_HEADS_SOFTPLUS, h.FLAG_HEADS_UNSCALED, h.HEADS_HISTORY, block.FLAG_SEQ_REVERSE)
    assert value("ptq_fp8.h", "PTQ_FP8_BLOCK") == fp8.FP8_BLOCK
    with pytest.raises(ValueError):
        fp8._code(torch.float64)
