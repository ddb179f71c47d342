"""The C ABI of include/ptq_block.h and the binding's checks, as far as they need no GPU."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import __graft_entry__ as entry

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
vp, ci, i64, u32, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint, ctypes.c_float
OK, NULL, SHAPE, VALUE, ALIGN, ARCH, CUDA = 0, 1, 2, 3, 4, 5, 6


class Scan(ctypes.Structure):
    _fields_ = [("dtype", ci), ("batch", ci), ("length", ci), ("channels", ci), ("states", ci), ("groups", ci), ("flags", u32), ("u", vp), ("delta", vp),
                ("z", vp), ("B", vp), ("C", vp), ("u_pitch", i64 * 2), ("delta_pitch", i64 * 2), ("z_pitch", i64 * 2), ("B_pitch", i64 * 3),
                ("C_pitch", i64 * 3), ("A", vp), ("D", vp), ("delta_bias", vp), ("state", vp), ("lengths", vp)]


class Norm(ctypes.Structure):
    _fields_ = [("dtype", ci), ("residual_dtype", ci), ("rows", i64), ("cols", ci), ("flags", u32), ("eps", f32), ("x", vp), ("residual", vp), ("gate", vp),
                ("x_pitch", i64), ("residual_pitch", i64), ("gate_pitch", i64), ("weight", vp), ("bias", vp), ("scale", vp)]


class Conv(ctypes.Structure):
    _fields_ = [("dtype", ci), ("batch", ci), ("length", ci), ("channels", ci), ("taps", ci), ("flags", u32), ("x", vp), ("x_pitch", i64 * 2), ("weight", vp),
                ("bias", vp), ("state", vp), ("lengths", vp)]


P = 4096                                                     # a device address that no host code looks at


def scan(**kw):
    s = Scan(dtype=0, batch=2, length=8, channels=16, states=4, groups=1, u=P, delta=P, B=P, C=P, A=P)
    for k, v in kw.items():
        setattr(s, k, (type(getattr(s, k)))(*v) if isinstance(v, tuple) else v)
    return s


def norm(**kw):
    n = Norm(dtype=0, residual_dtype=0, rows=3, cols=8, eps=1e-5, x=P)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


def conv(**kw):
    c = Conv(dtype=0, batch=2, length=8, channels=16, taps=4, x=P, weight=P)
    for k, v in kw.items():
        setattr(c, k, (type(getattr(c, k)))(*v) if isinstance(v, tuple) else v)
    return c


@pytest.fixture(scope="module")
def lib():
    entry.build()
    from paper_2412_20386_b200 import binding
    L = binding.load_library()
    for name in ("ptq_scan_workspace_bytes", "ptq_norm_workspace_bytes", "ptq_conv_workspace_bytes"):
        getattr(L, name).restype = ctypes.c_size_t
    return L


@pytest.fixture(scope="module")
def native():
    entry.build()
    from paper_2412_20386_b200 import binding
    return binding._load_native_block()


def test_library_exports_every_declared_symbol(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ptq_block.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ptq_[a-z_0-9]+)\s*\(", text)))
    assert len(names) == 9
    for n in names:
        assert hasattr(lib, n), n


def forward(lib, s, y=P, final=None, history=None, ws=P, nbytes=1 << 40):
    return lib.ptq_scan_forward(ctypes.byref(s) if s is not None else None, vp(y), vp(final), vp(history), vp(ws), ctypes.c_size_t(nbytes), None)


def test_scan_refusals(lib):
    assert forward(lib, None) == NULL
    for k in ("u", "delta", "B", "C", "A"):
        assert forward(lib, scan(**{k: None})) == NULL, k
    assert forward(lib, scan(), y=None) == NULL
    for kw in (dict(batch=0), dict(length=0), dict(length=(1 << 30) + 1), dict(channels=0), dict(channels=65537), dict(states=0), dict(states=33),
               dict(groups=0), dict(groups=3), dict(u_pitch=(1, -1)), dict(B_pitch=(0, 0, -4)), dict(batch=2 ** 31 - 1, channels=65536)):
        assert forward(lib, scan(**kw)) == SHAPE, kw
    for kw in (dict(dtype=3), dict(dtype=-1), dict(flags=4)):
        assert forward(lib, scan(**kw)) == VALUE, kw
    for kw in (dict(u=P + 1), dict(A=P + 2), dict(state=P + 2), dict(lengths=P + 1), dict(z=P + 1)):
        assert forward(lib, scan(**kw)) == ALIGN, kw
    assert forward(lib, scan(), y=P + 1) == ALIGN and forward(lib, scan(), final=P + 2) == ALIGN
    if not torch.cuda.is_available():                        # the pitches of what is not given do not count: as far as the device
        assert forward(lib, scan(z_pitch=(-1, -1))) in (ARCH, CUDA)
        assert lib.ptq_norm_forward(ctypes.byref(norm(gate_pitch=-1, residual_pitch=-1)), vp(P), None, None) in (ARCH, CUDA)
    need = lib.ptq_scan_workspace_bytes(ctypes.byref(scan(length=4000)), 0)
    assert need > 0
    assert forward(lib, scan(length=4000), ws=None) == NULL
    assert forward(lib, scan(length=4000), nbytes=need - 1) == SHAPE
    assert forward(lib, scan(length=4000), ws=P + 8) == ALIGN
    assert b"bytes" in lib.ptq_last_error() or b"aligned" in lib.ptq_last_error()
    assert lib.ptq_scan_workspace_bytes(None, 0) == 0 and lib.ptq_scan_workspace_bytes(ctypes.byref(scan(groups=3)), 1) == 0


def test_scan_backward_refusals(lib):
    def back(s, history=P, dy=P, grads=None, **kw):
        g = dict(du=P, ddelta=P, dz=None, dB=P, dC=P, dA=P, dD=None, ddelta_bias=None, dstate=None, **{})
        g.update(kw)
        arr = (vp * 9)(*[g[k] for k in ("du", "ddelta", "dz", "dB", "dC", "dA", "dD", "ddelta_bias", "dstate")])
        return lib.ptq_scan_backward(ctypes.byref(s), vp(history), vp(dy), None, arr if grads is None else None, vp(P), ctypes.c_size_t(1 << 40), None)
    assert back(scan(), history=None) == NULL and back(scan(), dy=None) == NULL and back(scan(), grads=False) == NULL
    for k in ("du", "ddelta", "dB", "dC", "dA"):
        assert back(scan(), **{k: None}) == NULL, k
    assert back(scan(z=P)) == NULL and back(scan(), dz=P) == NULL           # z and dz go together
    assert back(scan(), du=P + 1) == ALIGN and back(scan(), dstate=P + 2) == ALIGN
    s = scan()
    arr = (vp * 9)(P, P, None, P, P, P, None, None, None)
    need = lib.ptq_scan_workspace_bytes(ctypes.byref(s), 1)
    assert lib.ptq_scan_backward(ctypes.byref(s), vp(P), vp(P), None, arr, vp(P), ctypes.c_size_t(need - 1), None) == SHAPE


def test_norm_refusals(lib):
    f = lambda n, y=P, r=None: lib.ptq_norm_forward(ctypes.byref(n) if n is not None else None, vp(y), vp(r), None)
    assert f(None) == NULL and f(norm(x=None)) == NULL and f(norm(), y=None) == NULL
    for kw in (dict(rows=0), dict(cols=0), dict(cols=8193), dict(x_pitch=-1), dict(rows=(1 << 40) + 1)):
        assert f(norm(**kw)) == SHAPE, kw
    for kw in (dict(dtype=7), dict(residual_dtype=1), dict(flags=8), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert f(norm(**kw)) == VALUE, kw
    assert f(norm(weight=P + 2)) == ALIGN and f(norm(residual=P + 1)) == ALIGN and f(norm(), r=P + 1) == ALIGN
    b = lambda n, g, ws=P, nbytes=1 << 40: lib.ptq_norm_backward(ctypes.byref(n), vp(P), None, g, vp(ws), ctypes.c_size_t(nbytes), None)
    assert b(norm(), None) == NULL and b(norm(), (vp * 6)()) == NULL
    assert b(norm(gate=P), (vp * 6)(P)) == NULL and b(norm(), (vp * 6)(P, P)) == NULL       # gate and dgate go together
    need = lib.ptq_norm_workspace_bytes(ctypes.byref(norm()))
    assert need > 0 and b(norm(), (vp * 6)(P), nbytes=need - 1) == SHAPE and b(norm(), (vp * 6)(P), ws=None) == NULL


def test_conv_refusals(lib):
    f = lambda c, y=P, s=None: lib.ptq_conv_forward(ctypes.byref(c) if c is not None else None, vp(y), vp(s), None)
    assert f(None) == NULL and f(conv(x=None)) == NULL and f(conv(weight=None)) == NULL and f(conv(), y=None) == NULL
    for kw in (dict(batch=0), dict(length=0), dict(channels=0), dict(channels=65537), dict(taps=1), dict(taps=5), dict(x_pitch=(-1, 0)),
               dict(batch=2 ** 31 - 1, length=1 << 30, channels=65536)):
        assert f(conv(**kw)) == SHAPE, kw
    assert f(conv(dtype=9)) == VALUE and f(conv(flags=16)) == VALUE
    assert f(conv(x=P + 1)) == ALIGN and f(conv(bias=P + 1)) == ALIGN and f(conv(), s=P + 1) == ALIGN
    b = lambda c, g, nbytes=1 << 40: lib.ptq_conv_backward(ctypes.byref(c), vp(P), None, g, vp(P), ctypes.c_size_t(nbytes), None)
    assert b(conv(), None) == NULL and b(conv(), (vp * 4)(P)) == NULL
    need = lib.ptq_conv_workspace_bytes(ctypes.byref(conv()))
    assert need > 0 and b(conv(), (vp * 4)(P, None, P, None), nbytes=need - 1) == SHAPE


def test_without_a_device_a_good_call_fails_with_an_error_code(lib):
    if torch.cuda.is_available():
        pytest.skip("a CUDA device is present")
    assert forward(lib, scan()) in (ARCH, CUDA)
    assert lib.ptq_norm_forward(ctypes.byref(norm()), vp(P), None, None) in (ARCH, CUDA)
    assert lib.ptq_conv_forward(ctypes.byref(conv()), vp(P), None, None) in (ARCH, CUDA)


def test_workspaces_grow_with_the_call_and_never_overflow(lib):
    for kw in (dict(), dict(batch=128, length=197, channels=768, states=16), dict(batch=1, length=1 << 30, channels=65536, states=32),
               dict(batch=4096, length=1 << 20, channels=65536, states=32, groups=65536)):
        s = scan(**kw)
        fwd, bwd = lib.ptq_scan_workspace_bytes(ctypes.byref(s), 0), lib.ptq_scan_workspace_bytes(ctypes.byref(s), 1)
        assert bwd >= fwd + 4 * s.batch * s.channels * s.states, kw


@pytest.mark.parametrize("name,n", [("scan", 15), ("scan_backward", 14), ("norm", 10), ("norm_backward", 10), ("conv", 8), ("conv_backward", 8)])
def test_the_binding_refuses_wrong_objects_before_the_library_is_called(native, name, n):
    f = getattr(native, name)
    with pytest.raises(TypeError):
        f(*[None] * (n - 1))
    with pytest.raises(TypeError):
        f(*([0] if name == "scan" else []), *[None] * (n - (name == "scan")))
    with pytest.raises(TypeError):
        f(*([0] if name == "scan" else []), np.zeros((1, 1, 1), np.float16), *[None] * (n - 1 - (name == "scan")))
    with pytest.raises(ValueError):
        f(*([0] if name == "scan" else []), torch.zeros(1, 1, 1), *[None] * (n - 1 - (name == "scan")))


def test_names_of_kinds_are_checked():
    from paper_2412_20386_b200 import block
    for kw in (dict(kind="batch"), dict(gate_at="middle")):
        with pytest.raises(ValueError):
            block.block_norm(torch.zeros(1, 8), **kw)
        with pytest.raises(ValueError):
            block.block_norm_backward(torch.zeros(1, 8), torch.zeros(1, 8), **kw)


def test_constants_agree_with_the_header():
    from paper_2412_20386_b200 import block
    text = open(os.path.join(ROOT, "include", "ptq_block.h")).read()
    value = lambda name: int(re.search(r"#define %s\s+(\d+)u?" % name, text).group(1))
    assert (value("PTQ_SEQ_REVERSE"), value("PTQ_SCAN_SOFTPLUS"), value("PTQ_CONV_SILU"), value("PTQ_NORM_LAYER"), value("PTQ_NORM_GATE_OUT"),
            value("PTQ_SCAN_HISTORY")) == (block.FLAG_SEQ_REVERSE, block.FLAG_SCAN_SOFTPLUS, block.FLAG_CONV_SILU, block.FLAG_NORM_LAYER,
                                           block.FLAG_NORM_GATE_OUT, block.SCAN_HISTORY)
