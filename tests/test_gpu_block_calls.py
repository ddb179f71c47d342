"""How the operators between a block's linears are called: streams, captured graphs, refused arguments, far offsets, and all of them together as
a block uses them."""
import numpy as np
import pytest
import torch

import block_ref as ref
import oracle
from paper_2412_20386_b200 import workloads as wl
from parity_util import assert_y_close
from test_gpu_block_conv import make as make_conv
from test_gpu_block_norm import make as make_norm
from test_gpu_block_scan import call as call_scan, make as make_scan

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ptq():
    import __graft_entry__ as entry
    entry.build()
    import paper_2412_20386_b200 as p
    torch.cuda.set_device(0)
    return p


def everything(ptq, s, n, c, stream=None):
    """One call of each operator, forward and backward, with all that allocates."""
    with torch.cuda.stream(stream):                         # a buffer of the caller belongs to the stream that uses it
        history = ptq.scan_history(s["u"], s["A"].shape[1])
    kw = dict(D=s["D"], z=s["z"], delta_bias=s["delta_bias"], state=s["state"], stream=stream)
    args = (s["u"], s["delta"], s["A"], s["B"], s["C"])
    y = ptq.gated_scan(*args, **kw, history=history)
    out = [y, *ptq.gated_scan_backward(y, *args, history, **kw).values()]
    out += [*ptq.block_norm(**n, stream=stream), *ptq.block_norm_backward(n["x"].contiguous(), **n, stream=stream).values()]
    yc = ptq.short_conv(**c, stream=stream)
    return out + [yc, *ptq.short_conv_backward(yc, **c, stream=stream).values()]


def inputs(seed, L=300):
    return (make_scan(seed, ref.F16, 2, L, 48, 16, state=True), make_norm(seed, ref.BF16, 700, 264, ref.F32, True, True),
            make_conv(seed, ref.F16, 2, L, 72, 4, state=True)[0])


def same(a, b):
    return all((x is None and y is None) or torch.equal(x, y) for x, y in zip(a, b))


def test_calls_on_other_streams_while_freed_memory_is_still_written(ptq):
    sets = [inputs(i) for i in range(3)]
    want = [everything(ptq, *x) for x in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    a = torch.randn(4096, 4096, device="cuda")
    for _ in range(4):
        block = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
        a @ a
        block.fill_(255)
        del block
        got = [everything(ptq, *x, stream=st) for x, st in zip(sets, streams)]         # at the same time
        torch.cuda.synchronize()
        assert all(same(g, w) for g, w in zip(got, want))
    with torch.cuda.stream(streams[0]):                     # the current stream is the one that is used
        got = everything(ptq, *sets[1])
    streams[0].synchronize()
    assert same(got, want[1])


def test_graphs_are_captured_and_replayed_with_new_inputs(ptq):
    """Two graphs with memory of their own, replayed in turn and at the same time on two streams, on inputs that changed."""
    sets = [inputs(i + 10) for i in range(2)]
    later = [inputs(i + 20) for i in range(2)]
    want = [everything(ptq, *x) for x in later]
    graphs, outs = [], []
    for x in sets:
        everything(ptq, *x)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(everything(ptq, *x))
        graphs.append(g)
    for x, new in zip(sets, later):
        for a, b in zip(x, new):
            for k in a:
                if torch.is_tensor(a[k]):
                    a[k].copy_(b[k])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        assert all(same(o, w) for o, w in zip(outs, want))


FIRST_CALL = r"""
import torch, sys
import paper_2412_20386_b200 as ptq
x = torch.randn(3, 300, 2312, device="cuda").half()
A, w, B = -torch.rand(2312, 16, device="cuda"), torch.rand(2312, 4, device="cuda"), torch.randn(3, 300, 16, device="cuda").half()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
def run():
    h = ptq.scan_history(x, 16)
    y = ptq.gated_scan(x, x, A, B, B, history=h)
    return [y, *ptq.gated_scan_backward(y, x, x, A, B, B, h).values(), ptq.block_norm(x), *ptq.block_norm_backward(y, x).values(),
            *ptq.short_conv_backward(ptq.short_conv(x, w), x, w).values()]
with torch.cuda.graph(g):
    got = run()
g.replay()
torch.cuda.synchronize()
print(all(a is None or torch.equal(a, b) for a, b in zip(got, run())))
"""


def test_the_first_call_of_a_process_may_be_captured():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL], cwd=root, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "True", r.stderr[-2000:]


def test_a_token_step_in_a_graph_goes_on_from_its_own_state(ptq):
    t = make_scan(3, ref.BF16, 5, 6, 40, 16, state=True)
    final = torch.empty_like(t["state"])
    whole = call_scan(ptq, t, final_state=final)
    state, cols = t["state"].clone(), {k: t[k][:, 0].clone() for k in ("u", "delta", "z", "B", "C")}
    step = lambda y=None: ptq.gated_scan_step(state, cols["u"], cols["delta"], t["A"], cols["B"], cols["C"], D=t["D"], z=cols["z"],
                                              delta_bias=t["delta_bias"], y=y)
    step()
    state.copy_(t["state"])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = step()
    state.copy_(t["state"])
    for i in range(6):
        for k in cols:
            cols[k].copy_(t[k][:, i])
        g.replay()
        assert torch.allclose(y.float(), whole[:, i].float(), rtol=2.0 ** -7, atol=2.0 ** -7)
    assert torch.allclose(state, final, rtol=1e-5, atol=1e-5)


def test_refused_arguments(ptq):
    s, n, c = inputs(1, 20)
    args = (s["u"], s["delta"], s["A"], s["B"], s["C"])
    bad = [dict(delta=s["delta"].float()), dict(delta=s["delta"][:, :5]), dict(A=s["A"].half()), dict(A=s["A"].t()), dict(A=s["A"][:5]), dict(B=s["B"][..., :3]),
           dict(C=s["C"][:, :3]), dict(u=s["u"].transpose(1, 2)), dict(u=s["u"][0]), dict(u=s["u"].double())]
    names = ("u", "delta", "A", "B", "C")
    for kw in bad:
        with pytest.raises(ValueError):
            ptq.gated_scan(*[kw.get(k, v) for k, v in zip(names, args)])
    for kw in (dict(D=s["D"][:3]), dict(D=s["D"].half()), dict(z=s["z"].float()), dict(state=s["state"][:1]), dict(state=s["state"].half()),
               dict(lengths=torch.ones(2, device="cuda")), dict(lengths=torch.ones(3, dtype=torch.int32, device="cuda")), dict(y=torch.empty(1, device="cuda")),
               dict(final_state=torch.empty(1, device="cuda")), dict(history=torch.empty(2, 1, 48, 16, device="cuda")), dict(z=s["z"].cpu())):
        with pytest.raises(ValueError):
            ptq.gated_scan(*args, **kw)
    with pytest.raises(ValueError):                         # a column stride of two
        ptq.gated_scan(torch.zeros(2, 20, 96, dtype=torch.float16, device="cuda")[..., ::2], *args[1:])
    with pytest.raises(TypeError):
        ptq.gated_scan_step(s["state"], None, *args[1:])
    with pytest.raises(TypeError):
        ptq.gated_scan_backward(None, *args, ptq.scan_history(s["u"], 16))
    with pytest.raises(ptq.PtqError) as e:                  # more states than the kernels hold
        big = torch.zeros(2, 20, 33, dtype=torch.float16, device="cuda")
        ptq.gated_scan(s["u"], s["delta"], torch.zeros(48, 33, device="cuda"), big, big)
    assert e.value.status == 2
    for kw in (dict(B=torch.zeros(2, 20, 5, 16, dtype=torch.float16, device="cuda")),):
        with pytest.raises((ptq.PtqError, ValueError)):     # 48 channels do not make five groups
            ptq.gated_scan(s["u"], s["delta"], s["A"], kw["B"], kw["B"])
    with pytest.raises(ptq.PtqError):                       # nothing to do is refused, as the linears do
        ptq.gated_scan(*[v[:0] if v.dim() > 2 else v for v in args])
    for kw in (dict(weight=n["weight"][:3]), dict(weight=n["weight"].half()), dict(residual=n["residual"].half()), dict(gate=n["gate"].float()),
               dict(scale=n["scale"][None]), dict(residual_out=torch.empty(700, 264, device="cuda", dtype=torch.float16)), dict(y=n["residual"])):
        with pytest.raises((ValueError, ptq.PtqError)):
            ptq.block_norm(**{**n, **kw})
    with pytest.raises(ptq.PtqError):
        ptq.block_norm(torch.zeros(2, 8193, device="cuda"))
    with pytest.raises(ptq.PtqError):
        ptq.block_norm(n["x"], eps=-1.0)
    with pytest.raises(ValueError):                         # rows that are not one distance apart
        ptq.block_norm(torch.zeros(4, 6, 8, device="cuda")[:, :3])
    for kw in (dict(weight=torch.zeros(72, 5, device="cuda")), dict(weight=torch.zeros(72, 1, device="cuda"))):
        with pytest.raises(ptq.PtqError):
            ptq.short_conv(c["x"], kw["weight"])
    for kw in (dict(weight=c["weight"].half()), dict(bias=c["bias"][:3]), dict(state=c["state"].float()), dict(x=c["x"][0])):
        with pytest.raises(ValueError):
            ptq.short_conv(**{**c, **kw})


def test_far_offsets(ptq):
    """Rows whose offsets pass 2^31 elements (and 2^32 bytes): tokens, sequences, and dense outputs."""
    pitch = (1 << 26) + 8
    base = torch.empty(39 * pitch + 64, dtype=torch.bfloat16, device="cuda")           # 5 GB, only a few rows of it are used
    gen = torch.Generator().manual_seed(1)
    vals = torch.randn(1, 40, 64, generator=gen).to(torch.bfloat16).cuda()
    far = base.as_strided((1, 40, 16), (0, pitch, 1))
    for name, lo in (("u", 0), ("delta", 16), ("B", 32), ("C", 48)):
        base.as_strided((1, 40, 16), (0, pitch, 1), lo).copy_(vals[..., lo:lo + 16])
    strided = {n: base.as_strided((1, 40, 16), (0, pitch, 1), lo) for n, lo in (("u", 0), ("delta", 16), ("B", 32), ("C", 48))}
    dense = {n: v.contiguous() for n, v in strided.items()}
    A = -torch.rand(16, 16, device="cuda")
    outs = []
    for t in (strided, dense):
        h = ptq.scan_history(t["u"], 16)
        y = ptq.gated_scan(t["u"], t["delta"], A, t["B"], t["C"], z=t["u"], history=h, reverse=True)
        g = ptq.gated_scan_backward(y, t["u"], t["delta"], A, t["B"], t["C"], h, z=t["u"], reverse=True)
        b = [v.transpose(0, 1) for v in (t["u"], t["delta"], t["B"], t["C"])]           # one token of each of 40 sequences
        state = torch.ones(40, 16, 16, device="cuda")
        ys = ptq.gated_scan_step(state, *[v[:, 0] for v in b[:2]], A, *[v[:, 0] for v in b[2:]])
        w = torch.linspace(-1, 1, 64, device="cuda").reshape(16, 4)
        yc = ptq.short_conv(t["u"], w)
        yn = ptq.block_norm(t["u"], gate=t["delta"])
        outs.append([y, *g.values(), ys, state, yc, *ptq.short_conv_backward(yc, t["u"], w).values(), yn,
                     *ptq.block_norm_backward(yn, t["u"], gate=t["delta"]).values()])
    assert same(*outs)
    assert far.data_ptr() == base.data_ptr()
    del base, far, strided, dense, outs
    # a dense output of more than 2^31 elements: its last rows
    L, D = (1 << 21) + 77, 1024
    x = torch.zeros(1, L, D, dtype=torch.bfloat16, device="cuda")
    x[0, -64:] = torch.randn(64, D, generator=gen).to(torch.bfloat16).cuda()
    w = torch.randn(D, 4, generator=gen).cuda()
    tail = ptq.short_conv(x[:, -64:].contiguous(), w)
    y = ptq.short_conv(x, w)
    assert torch.equal(y[:, -64:], tail)
    g = ptq.short_conv_backward(y, x, w)["x"]
    assert torch.equal(g[0, -64:], ptq.short_conv_backward(tail, x[:, -64:].contiguous(), w)["x"][0])
    del g
    assert torch.equal(ptq.block_norm(x)[0, -64:], ptq.block_norm(x[0, -64:].contiguous()))


def test_expanded_inputs_get_one_gradient_per_token(ptq):
    """B and C shared by all sequences through a pitch of zero: their gradients are dense, and their sum is the shared tensor's."""
    t = make_scan(4, ref.F32, 3, 20, 16, 8)
    for k in ("B", "C"):
        t[k] = t[k][:1].contiguous().expand(3, 20, 1, 8)
    full = {**t, **{k: t[k].contiguous() for k in ("B", "C")}}
    dy = torch.randn(3, 20, 16, device="cuda")
    got = []
    for x in (t, full):
        h = ptq.scan_history(x["u"], 8)
        call_scan(ptq, x, history=h)
        got.append(ptq.gated_scan_backward(dy, x["u"], x["delta"], x["A"], x["B"], x["C"], h, D=x["D"], z=x["z"], delta_bias=x["delta_bias"]))
    assert got[0]["B"].shape == (3, 20, 1, 8) and all(torch.equal(got[0][k], got[1][k]) for k in ("u", "A", "B", "C"))


def quantized(ptq, x, w, bias=None):
    """A W8A8 layer for the weights w, calibrated on x [B,T,K], and its oracle as a function of the input."""
    dw = np.abs(w).max(1).astype(np.float32) / 127
    wq = np.clip(np.rint(w / dw[:, None]), -127, 127).astype(np.int8)
    s, dx = ptq.calibrate(x, wq, dw)
    wq = np.clip(np.rint(w * s / (np.abs(w * s).max(1, keepdims=True) / 127)), -127, 127).astype(np.int8)
    dw = (np.abs(w * s).max(1) / 127).astype(np.float32)
    layer = ptq.PtqLinear(wq, dw, s, dx, bias)
    return layer, lambda v: oracle.linear_forward(v.reshape(-1, v.shape[-1]), v.shape[1], wq, dw, s, dx, bias)


def test_a_block_in_both_directions(ptq):
    """norm, in_proj, then per direction convolution, x_proj, dt_proj and scan, the gated norm, out_proj, residual and the next norm: the
    quantized linears against their oracle and every operator against 64 bits, each on what the one before it gave."""
    rng = np.random.default_rng(11)
    B, T, C, D, N, R = 3, 49, 64, 128, 16, 8
    stream = torch.from_numpy(rng.standard_normal((B, T, C)).astype(np.float32)).cuda()
    out = torch.from_numpy(rng.standard_normal((B, T, C)).astype(np.float16)).cuda()
    vec = lambda n, lo=0.5, hi=1.5: torch.from_numpy(rng.uniform(lo, hi, n).astype(np.float32)).cuda()
    mat = lambda n, k: (rng.standard_normal((n, k)) / np.sqrt(k)).astype(np.float32)
    f64 = lambda t: t.double().cpu()
    f = 2.0 ** -10                                           # of |value| + 1: every operator's own tests hold the tight bounds

    def agrees(got, want, what):
        ref.close(got, want, want.abs() + 1.0, f, what)
    w_norm, scale = vec(C), vec(C, 0.1, 1.0)
    x, stream2 = ptq.block_norm(out, w_norm, residual=stream, scale=scale)
    y64, r64 = ref.norm(f64(out), f64(w_norm), residual=f64(stream), scale=f64(scale))
    agrees(x, y64, "norm"), agrees(stream2, r64, "residual stream")
    layer, want = quantized(ptq, x, mat(2 * D, C))
    xz = layer.forward(x)
    assert_y_close(xz.cpu().numpy().reshape(-1, 2 * D), want(x.cpu().numpy()), "in_proj")
    total = None
    for reverse in (False, True):
        cw, cb = torch.from_numpy(mat(D, 4)).cuda(), vec(D, -0.2, 0.2)
        u = ptq.short_conv(xz[..., :D], cw, cb, reverse=reverse)
        agrees(u, ref.conv(f64(xz[..., :D]), f64(cw), f64(cb), reverse=reverse)[0], "convolution")
        x_proj, want = quantized(ptq, u, mat(R + 2 * N, D))
        dbc = x_proj.forward(u)
        assert_y_close(dbc.cpu().numpy().reshape(-1, R + 2 * N), want(u.cpu().numpy()), "x_proj")
        low = dbc[..., :R].contiguous()
        dt_proj, want = quantized(ptq, low, mat(D, R))
        delta = dt_proj.forward(low)
        A, skip, db = -torch.arange(1.0, N + 1, device="cuda").repeat(D, 1), vec(D), vec(D, -5, -2)
        Bm, Cm = dbc[..., R:R + N], dbc[..., R + N:]
        y = ptq.gated_scan(u, delta, A, Bm, Cm, D=skip, z=xz[..., D:], delta_bias=db, reverse=reverse)
        agrees(y, ref.scan(f64(u), f64(delta), f64(A), f64(Bm), f64(Cm), f64(skip), f64(xz[..., D:]), f64(db), reverse=reverse)[0], "scan")
        total = y if total is None else total + y
    w2 = vec(D)
    normed = ptq.block_norm(total, w2, gate=xz[..., D:], kind="layer", gate_at="out")
    agrees(normed, ref.norm(f64(total), f64(w2), gate=f64(xz[..., D:]), kind="layer", gate_at="out")[0], "gated norm")
    out_proj, want = quantized(ptq, normed, mat(C, D))
    out2 = out_proj.forward(normed)
    assert_y_close(out2.cpu().numpy().reshape(-1, C), want(normed.cpu().numpy()), "out_proj")
    for l in (layer, x_proj, dt_proj, out_proj):
        l.device_status()
    y, stream3 = ptq.block_norm(out2, w_norm, residual=stream2, scale=scale)
    agrees(stream3, f64(stream2) + f64(scale) * f64(out2), "residual stream behind the block")


def test_serving_token_by_token_follows_the_whole_sequence(ptq):
    """conv and scan with their states, as a generating program keeps them, against one call over the sequence."""
    B, T, D, N = 4, 12, 64, 16
    gen = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=gen).cuda()
    xz, cw, cb = r(B, T, 2 * D).to(torch.bfloat16), r(D, 4), r(D)
    A, skip, db = -torch.rand(D, N, generator=gen).cuda() * 4, r(D), r(D) - 3
    dbc, delta = r(B, T, 2 * N).to(torch.bfloat16), r(B, T, D).to(torch.bfloat16)
    u = ptq.short_conv(xz[..., :D], cw, cb)
    y = ptq.gated_scan(u, delta, A, dbc[..., :N], dbc[..., N:], D=skip, z=xz[..., D:], delta_bias=db)
    taps, state = torch.zeros(B, 3, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, D, N, device="cuda")
    for i in range(T):
        ui = ptq.short_conv(xz[:, i:i + 1, :D], cw, cb, state=taps, final_state=taps)
        assert torch.equal(ui, u[:, i:i + 1])
        yi = ptq.gated_scan_step(state, ui[:, 0], delta[:, i], A, dbc[:, i, :N], dbc[:, i, N:], D=skip, z=xz[:, i, D:], delta_bias=db)
        assert torch.allclose(yi.float(), y[:, i].float(), rtol=2.0 ** -7, atol=2.0 ** -6)
