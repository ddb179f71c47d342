"""block_norm and block_norm_backward where a residual stream begins: r is handed on without a residual coming in, so that the backward pass has
a gradient of r to add and no residual to read.  Against the formulas in 64 bits.

Tolerances as in block_ref: half a step of the result's type, and 2^-18 of the expression by magnitude, in which n stands with the error of r relative to
its rms and mean, and the gradient of r twice (its terms, and the factor 1 / rms that they share)."""
import itertools

import pytest
import torch

import block_ref as ref
from test_gpu_block_norm import make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ptq():
    import __graft_entry__ as entry
    entry.build()
    import paper_2412_20386_b200 as p
    torch.cuda.set_device(0)
    return p


def magnitudes(t, kind, gate_at, eps, dy, dr):
    """Per gradient the expression by magnitude."""
    x = {k: None if v is None else v.detach().double().cpu() for k, v in t.items()}
    silu = torch.ones(1, dtype=torch.float64) if t["gate"] is None else x["gate"] * torch.sigmoid(x["gate"])
    front, behind = (silu if gate_at == "in" else 1.0), (silu.abs() if gate_at == "out" else 1.0)
    v = x["x"] * front
    s = 1.0 if t["scale"] is None else x["scale"]
    w = 1.0 if t["weight"] is None else x["weight"].abs()
    r, r_abs = s * v, (s * v).abs()
    d = r - (r.mean(-1, keepdim=True) if kind == "layer" else 0.0)
    rms = torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    n = (d / rms).abs() + (r_abs + r_abs.mean(-1, keepdim=True)) / rms + (d / rms).abs() * (r_abs * d.abs()).mean(-1, keepdim=True) / rms ** 2
    dt = dy.double().cpu().abs() * behind
    dn = dt * w
    g = 2 * (dn + n * (dn * n).mean(-1, keepdim=True) + dn.mean(-1, keepdim=True)) / rms + (0.0 if dr is None else dr.double().cpu().abs())
    s = abs(s)
    gate = 1.2 * g * s * x["x"].abs() if gate_at == "in" else 1.2 * dy.double().cpu().abs() * (n * w + (0.0 if t["bias"] is None else x["bias"].abs()))
    return {"x": g * s * (silu.abs() if gate_at == "in" else 1.0), "weight": (dt * n).sum(0), "bias": dt.sum(0), "scale": (g * v.abs()).sum(0), "gate": gate}


def check(ptq, t, kind, gate_at, dr_type, eps=1e-5, seed=3):
    args = {k: t[k] for k in ("weight", "bias", "scale", "gate")}
    kw = dict(kind=kind, gate_at=gate_at, eps=eps)
    gen = torch.Generator().manual_seed(seed)
    dy = torch.randn(t["x"].shape, generator=gen).to(t["x"].dtype).cuda()
    dr = None if dr_type is None else torch.randn(t["x"].shape, generator=gen).to(dr_type).cuda()
    x64 = ref.leaves(t)
    y64, r64 = ref.norm(x64["x"], **{k: x64.get(k) for k in args}, **kw)
    want = ref.gradients((y64, r64), (dy, dr), x64)
    got = ptq.block_norm_backward(dy, t["x"], **args, **kw, dresidual_out=dr)
    bound = magnitudes(t, kind, gate_at, eps, dy, dr)
    for k in ("x", "weight", "bias", "scale", "gate"):
        if t[k] is None:
            assert got[k] is None
            continue
        assert got[k].dtype == t[k].dtype
        ref.close(got[k], want[k], bound[k], 2.0 ** -18, "gradient of " + k)
    assert got["residual"] is None
    return got


@pytest.mark.parametrize("kind,gate_at", list(itertools.product(["rms", "layer"], ["in", "out"])))
@pytest.mark.parametrize("dtype", [ref.F32, ref.F16, ref.BF16], ids=["f32", "f16", "bf16"])
def test_a_gradient_of_r_without_a_residual(ptq, kind, gate_at, dtype):
    """One row and two rows at a time, aligned rows and general ones, every other optional input."""
    for i, (scale, gate, bias) in enumerate(itertools.product([False, True], repeat=3)):
        check(ptq, make(i, dtype, 5, 72, None, scale, gate, bias=bias), kind, gate_at, dtype)
        check(ptq, make(i, dtype, 5, 35, None, scale, gate, bias=bias), kind, gate_at, dtype)
    check(ptq, make(20, dtype, 1187, 72, None, True, True), kind, gate_at, dtype)
    check(ptq, make(21, dtype, 1200, 35, None, True, True), kind, gate_at, dtype)


@pytest.mark.parametrize("D", [8, 256, 384, 768, 2040, 2048, 2049, 2056, 4096, 8191, 8192])
def test_widths_with_a_gradient_of_r_alone(ptq, D):
    """One warp to 32; two sets of rows in shared memory, and the one that the widest rows leave room for."""
    for dtype, gate in ((ref.F32, True), (ref.BF16, False)):
        check(ptq, make(D, dtype, 3, D, None, True, gate), "layer", "in", dtype)
    if D <= 768:
        check(ptq, make(D, ref.F16, 2400, D, None, gate=True), "rms", "out", ref.F16)


def test_the_gradient_of_r_is_added_as_beside_a_residual_of_zeros(ptq):
    """The same numbers as a call whose residual is zeros: dx and dgate to the bit."""
    t = make(4, ref.BF16, 1300, 768, None, True, True)
    dy, dr = (torch.randn(1300, 768, device="cuda").to(torch.bfloat16) for _ in range(2))
    args = {k: t[k] for k in ("weight", "bias", "scale", "gate")}
    a = ptq.block_norm_backward(dy, t["x"], **args, dresidual_out=dr)
    b = ptq.block_norm_backward(dy, t["x"], **args, dresidual_out=dr, residual=torch.zeros_like(t["x"]))
    assert torch.equal(a["x"], b["x"]) and torch.equal(a["gate"], b["gate"])
    assert not torch.equal(a["x"], ptq.block_norm_backward(dy, t["x"], **args)["x"])
