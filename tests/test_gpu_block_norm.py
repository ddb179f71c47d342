"""block_norm and block_norm_backward against the formulas in 64 bits."""
import itertools

import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ptq():
    import __graft_entry__ as entry
    entry.build()
    import paper_2412_20386_b200 as p
    torch.cuda.set_device(0)
    return p


def make(seed, dtype, M, D, residual=None, scale=False, gate=False, weight=True, bias=True, pad=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    rows = lambda t, dt: torch.cat([t, torch.full((M, pad), float("nan"))], 1).to(dt).cuda()[:, :D] if pad else t.to(dt).cuda()
    return {"x": rows(r(M, D), dtype), "weight": (1 + 0.2 * r(D)).cuda() if weight else None, "bias": r(D).cuda() if bias else None,
            "residual": rows(2 * r(M, D), residual) if residual else None, "scale": (r(D)).cuda() if scale else None,
            "gate": rows(r(M, D), dtype) if gate else None}


def check(ptq, t, kind, gate_at, eps=1e-5, cotangent=True, seed=3):
    kw = dict(kind=kind, gate_at=gate_at, eps=eps)
    args = {k: t[k] for k in ("weight", "bias", "residual", "scale", "gate")}
    out = ptq.block_norm(t["x"], **args, **kw)
    y, r = out if t["residual"] is not None else (out, None)
    x64 = ref.leaves(t)
    pick = {k: x64.get(k) for k in args}
    y64, r64 = ref.norm(x64["x"], **pick, **kw)
    # scales: n is at most sqrt(D) and carries the error of r relative to its rms and mean
    n, _ = ref.norm(x64["x"], residual=pick["residual"], scale=pick["scale"], gate=pick["gate"], kind=kind, gate_at=gate_at if gate_at == "in" else "in", eps=eps) \
        if gate_at == "in" or pick["gate"] is None else ref.norm(x64["x"], residual=pick["residual"], scale=pick["scale"], kind=kind, eps=eps)
    big = lambda v: 0.0 if v is None else v.detach().abs()
    gate = torch.ones(1, dtype=torch.float64) if t["gate"] is None else (x64["gate"] * torch.sigmoid(x64["gate"])).detach().abs()
    v_abs = x64["x"].detach().abs() * (gate if gate_at == "in" and t["gate"] is not None else 1.0)
    r_abs = v_abs * (big(pick["scale"]) if pick["scale"] is not None else 1.0) + big(pick["residual"])
    d = r64.detach() - (r64.detach().mean(-1, keepdim=True) if kind == "layer" else 0.0)
    rms = torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    w = 1.0 if pick["weight"] is None else big(pick["weight"])
    n_scale = n.detach().abs() + (r_abs + r_abs.mean(-1, keepdim=True)) / rms + n.detach().abs() * (r_abs * d.abs()).mean(-1, keepdim=True) / rms ** 2
    out_gate = gate if gate_at == "out" and t["gate"] is not None else 1.0
    f = 2.0 ** -19
    ref.close(y, y64, (n_scale * w + big(pick["bias"])) * out_gate, f, "y")
    if r is not None:
        ref.close(r, r64, r_abs, f, "r")
    gen = torch.Generator().manual_seed(seed)
    dy = torch.randn(t["x"].shape, generator=gen).to(t["x"].dtype).cuda()
    dr = torch.randn(t["x"].shape, generator=gen).to(t["residual"].dtype).cuda() if t["residual"] is not None and cotangent else None
    g64 = ref.gradients((y64, r64), (dy, dr), x64)
    got = ptq.block_norm_backward(dy, t["x"], **args, **kw, dresidual_out=dr)
    dt_abs = dy.double().cpu().abs() * out_gate
    dn = dt_abs * w
    na = n_scale
    dr_scale = (dn + na * (dn * na).mean(-1, keepdim=True) + dn.mean(-1, keepdim=True)) / rms * (1 + na.max(-1, keepdim=True).values * 0 + 1) + (
        0.0 if dr is None else dr.double().cpu().abs())
    s = 1.0 if pick["scale"] is None else big(pick["scale"])
    bound = {"weight": (dt_abs * na).sum(0), "bias": dt_abs.sum(0), "residual": dr_scale, "scale": (dr_scale * v_abs).sum(0)}
    if t["gate"] is not None and gate_at == "in":
        bound["x"], bound["gate"] = dr_scale * s * gate, 1.2 * dr_scale * s * x64["x"].detach().abs()
    else:
        bound["x"] = dr_scale * s
        bound["gate"] = 1.2 * dy.double().cpu().abs() * (na * w + big(pick["bias"]))
    for k in t:
        if t[k] is None:
            assert got[k] is None
            continue
        assert got[k].dtype == t[k].dtype
        ref.close(got[k], g64[k], bound[k], 2 * f, "gradient of " + k)


@pytest.mark.parametrize("kind,gate_at", list(itertools.product(["rms", "layer"], ["in", "out"])))
@pytest.mark.parametrize("dtype,residual", [(ref.F32, ref.F32), (ref.BF16, ref.F32), (ref.BF16, ref.BF16), (ref.F16, ref.F16), (ref.F16, ref.F32), (ref.F16, None)])
def test_forms_and_types(ptq, kind, gate_at, dtype, residual):
    for i, (scale, gate, weight, bias) in enumerate(itertools.product([False, True], repeat=4)):
        check(ptq, make(i, dtype, 5, 72, residual, scale, gate, weight, bias), kind, gate_at, cotangent=i % 3 > 0)


@pytest.mark.parametrize("D", [1, 2, 7, 8, 9, 31, 250, 256, 257, 768, 1000, 1024, 2040, 2048, 2049, 2056, 4100, 8191, 8192])
def test_widths(ptq, D):
    """One thread, one warp, several, and the wide form; ends inside a thread's eight columns."""
    check(ptq, make(D, ref.BF16, 3, D, ref.F32, True, True), "layer" if D > 1 else "rms", "in")
    check(ptq, make(D, ref.F32, 2, D, ref.F32, gate=True), "rms", "out")


@pytest.mark.parametrize("M", [1, 2, 1183, 1185, 1187, 4801])
def test_row_counts(ptq, M):
    """Sets of rows with an incomplete last one; grids that go over the rows more than once."""
    check(ptq, make(M, ref.F16, M, 40, ref.F16, True), "layer", "in")
    check(ptq, make(M, ref.BF16, M, 264, None, gate=True), "rms", "in")


@pytest.mark.parametrize("pad", [1, 2, 8])
def test_rows_at_any_pitch(ptq, pad):
    """Slices of wider rows, the rest NaN: not read."""
    check(ptq, make(pad, ref.F16, 9, 96, ref.F32, True, True, pad=pad), "layer", "out")
    check(ptq, make(pad, ref.F32, 9, 33, ref.F32, pad=pad), "rms", "in")


def test_leading_dimensions_and_outputs_of_the_caller(ptq):
    t = make(1, ref.F16, 6 * 11, 40, ref.F16)
    y, r = ptq.block_norm(t["x"], t["weight"], t["bias"], residual=t["residual"])
    y3, r3 = ptq.block_norm(t["x"].reshape(6, 11, 40), t["weight"], t["bias"], residual=t["residual"].reshape(6, 11, 40))
    assert torch.equal(y3.reshape(66, 40), y) and torch.equal(r3.reshape(66, 40), r)
    sliced = torch.randn(6, 11, 80, device="cuda", dtype=torch.float16)[..., 40:]
    assert torch.equal(ptq.block_norm(sliced, t["weight"]), ptq.block_norm(sliced.contiguous(), t["weight"]))
    assert torch.equal(ptq.block_norm(sliced[:, :1], t["weight"]), ptq.block_norm(sliced[:, :1].contiguous(), t["weight"]))
    one = t["x"][0]
    assert torch.equal(ptq.block_norm(one, t["weight"], t["bias"], residual=t["residual"][0])[0], y[0])
    out, stream = torch.empty_like(t["x"]), t["residual"].clone()
    got = ptq.block_norm(t["x"], t["weight"], t["bias"], residual=stream, y=out, residual_out=stream)      # the stream is replaced
    assert got[0] is not None and torch.equal(out, y) and torch.equal(stream, r)
    y_only = ptq.block_norm(t["x"], t["weight"], residual_out=(copy := torch.empty_like(t["x"])))
    assert torch.equal(copy, t["x"]) and torch.equal(y_only[0], ptq.block_norm(t["x"], t["weight"]))


def test_rows_of_zeros_constants_and_large_values(ptq):
    """A row without variance gives its bias; values near the type's end do not overflow before they are squared in binary32."""
    x = torch.zeros(4, 64, dtype=torch.float16, device="cuda")
    x[1] = 3.0
    x[2] = 60000.0
    x[3, 0] = 60000.0
    w, b = torch.ones(64, device="cuda"), torch.full((64,), 0.25, device="cuda")
    y = ptq.block_norm(x, w, b, kind="layer")
    assert torch.equal(y[:3], torch.full_like(y[:3], 0.25))
    y64, _ = ref.norm(x.double().cpu(), w.double().cpu(), b.double().cpu(), kind="layer")
    ref.close(y, y64, y64.abs(), 2.0 ** -18, "y")
    rms = ptq.block_norm(x, w, eps=0.0)
    assert torch.isnan(rms[0]).all() and torch.allclose(rms[2].float(), torch.ones(64, device="cuda"), atol=1e-3)
    x[1, 5] = float("nan")
    y = ptq.block_norm(x, w, b)
    assert torch.isnan(y[1]).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[2:]).all()


def test_gradients_against_differences(ptq):
    t = make(5, ref.F32, 6, 24, ref.F32, True, True)
    gen = torch.Generator().manual_seed(2)
    dy, dr = (torch.randn(6, 24, generator=gen).cuda() for _ in range(2))
    for kind, gate_at in itertools.product(["rms", "layer"], ["in", "out"]):
        g = ptq.block_norm_backward(dy, **t, kind=kind, gate_at=gate_at, dresidual_out=dr)
        x = {k: v.double().cpu() for k, v in t.items()}
        for k in t:
            v = torch.randn(x[k].shape, generator=gen, dtype=torch.float64)

            def loss(s):
                y, r = ref.norm(**{**x, k: x[k] + s * v}, kind=kind, gate_at=gate_at)
                return float((y * dy.double().cpu()).sum() + (r * dr.double().cpu()).sum())
            got = g[k].double().cpu() * v
            assert abs(float(got.sum()) - (loss(1e-5) - loss(-1e-5)) / 2e-5) <= 2.0 ** -15 * float(got.abs().sum()), (kind, gate_at, k)


def test_same_bits_every_time(ptq):
    t = make(8, ref.BF16, 3000, 384, ref.F32, True, True)
    dy = torch.randn(3000, 384, device="cuda", dtype=torch.bfloat16)
    first = ptq.block_norm_backward(dy, **t)
    for _ in range(3):
        again = ptq.block_norm_backward(dy, **t)
        assert all(torch.equal(first[k], again[k]) for k in first)
