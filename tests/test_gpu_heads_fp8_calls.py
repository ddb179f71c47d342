"""How linear attention with decays and the fp8 linears are called: streams, captured graphs, refused arguments, far offsets, and together with
the operators that stand beside them in a block."""
import pytest
import torch

import block_ref as ref
import heads_ref
from block_ref import BF16, F16, F32, close
from test_gpu_heads import back, call, make

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ptq():
    import __graft_entry__ as entry
    entry.build()
    import paper_2412_20386_b200 as p
    torch.cuda.set_device(0)
    yield p
    p.fp8_device_status()


def inputs(ptq, seed, L=1000):
    """A scan that is cut into segments, rows for every form of the product."""
    t = make(seed, F16, 2, L, 3, 48, 24, state=True)
    gen = torch.Generator().manual_seed(seed)
    w, ws = ptq.fp8_quantize_weight(torch.randn(200, 400, generator=gen).cuda())
    t.update(w=w, ws=ws, b=torch.randn(200, generator=gen).cuda(), x=torch.randn(900, 400, generator=gen).to(BF16).cuda())
    return t


def everything(ptq, t, stream=None):
    with torch.cuda.stream(stream):                         # a buffer of the caller belongs to the stream that uses it
        history = ptq.head_scan_history(t["u"], t["B"].shape[-1])
    y = call(ptq, t, history=history, stream=stream)
    out = [y, *back(ptq, t, y, history, stream=stream).values()]
    for rows in (900, 100, 40, 3):
        x = t["x"][:rows]
        a, sa = ptq.fp8_quantize(x, stream=stream)
        out += [a.view(torch.uint8), sa, ptq.fp8_matmul(a, sa, t["w"], t["ws"], t["b"], dtype=F32, stream=stream), ptq.fp8_linear(x, t["w"], t["ws"], stream=stream)]
    return out


def same(a, b):
    return all((x is None and y is None) or torch.equal(x, y) for x, y in zip(a, b))


def test_calls_on_other_streams_while_freed_memory_is_still_written(ptq):
    sets = [inputs(ptq, i) for i in range(3)]
    want = [everything(ptq, x) for x in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    a = torch.randn(4096, 4096, device="cuda")
    for _ in range(4):
        block = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
        a @ a
        block.fill_(255)
        del block
        got = [everything(ptq, x, stream=st) for x, st in zip(sets, streams)]           # at the same time
        torch.cuda.synchronize()
        assert all(same(g, w) for g, w in zip(got, want))
    with torch.cuda.stream(streams[0]):                     # the current stream is the one that is used
        got = everything(ptq, sets[1])
    streams[0].synchronize()
    assert same(got, want[1])


def test_graphs_are_captured_and_replayed_with_new_inputs(ptq):
    """Two graphs with memory of their own, replayed in turn and at the same time on two streams, on inputs that changed."""
    sets, later = ([inputs(ptq, i + k) for i in range(2)] for k in (10, 20))
    want = [everything(ptq, x) for x in later]
    graphs, outs = [], []
    for x in sets:
        everything(ptq, x)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(everything(ptq, x))
        graphs.append(g)
    for x, new in zip(sets, later):
        for k in x:
            if torch.is_tensor(x[k]):
                (x[k].view(torch.uint8) if x[k].dtype == E4M3 else x[k]).copy_(new[k].view(torch.uint8) if new[k].dtype == E4M3 else new[k])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        assert all(same(o, w) for o, w in zip(outs, want))


FIRST_CALL = r"""
import torch
import paper_2412_20386_b200 as ptq
u = torch.randn(2, 700, 3, 64, device="cuda").half()
d, A, B = torch.randn(2, 700, 3, device="cuda").half(), -torch.rand(3, device="cuda"), torch.randn(2, 700, 32, device="cuda").half()
x, w, ws = torch.randn(300, 256, device="cuda").half(), torch.zeros(96, 256, device="cuda").to(torch.float8_e4m3fn), torch.rand(1, 2, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
def run():
    h = ptq.head_scan_history(u, 32)
    y = ptq.head_scan(u, d, A, B, B, history=h)
    a, s = ptq.fp8_quantize(x)
    state = torch.zeros(2, 3, 64, 32, device="cuda")
    return [y, *ptq.head_scan_backward(y, u, d, A, B, B, h).values(), ptq.head_scan_step(state, u[:, 0], d[:, 0], A, B[:, 0], B[:, 0]), state,
            ptq.fp8_matmul(a, s, w, ws), ptq.fp8_linear(x, w, ws), ptq.fp8_linear(x[:2], w, ws), *[v.view(torch.uint8) for v in ptq.fp8_quantize_weight(x)]]
with torch.cuda.graph(g):
    got = run()
g.replay()
torch.cuda.synchronize()
ptq.fp8_device_status()
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
    t = make(3, BF16, 5, 6, 4, 64, 32, state=True)
    value, scale, F = heads_ref.solve(t)
    state, cols = t["state"].clone(), {k: t[k][:, 0].clone() for k in ("u", "delta", "B", "C")}
    step = lambda: ptq.head_scan_step(state, cols["u"], cols["delta"], t["A"], cols["B"], cols["C"], D=t["D"], delta_bias=t["delta_bias"])
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = step()
    state.copy_(t["state"])
    for i in range(6):
        for k in cols:
            cols[k].copy_(t[k][:, i])
        g.replay()
        close(y, value["y"][:, i], scale["y"][:, i], F, "token")
    close(state, value["final"], scale["final"], F, "state")


def test_refused_arguments_of_the_scan(ptq):
    t = make(1, F16, 2, 20, 3, 16, 8, state=True)
    args = {k: t[k] for k in ("u", "delta", "A", "B", "C")}
    z = lambda *s, dtype=F16: torch.zeros(*s, dtype=dtype, device="cuda")
    for kw in (dict(delta=t["delta"].float()), dict(delta=t["delta"][:, :5]), dict(A=t["A"].half()), dict(A=t["A"][:2]), dict(A=z(6, dtype=F32)[::2]),
               dict(B=t["B"][..., :3]), dict(C=t["C"][:, :3]), dict(u=t["u"][0]), dict(u=t["u"].double()), dict(u=t["u"].transpose(2, 3)), dict(B=z(2, 20, 1, 1, 8)),
               dict(D=t["D"][:2]), dict(D=t["D"].half()), dict(delta_bias=t["delta_bias"][:1]), dict(state=t["state"][:1]), dict(state=t["state"].half()),
               dict(state=t["state"].transpose(2, 3)), dict(lengths=torch.ones(2, device="cuda")), dict(lengths=torch.ones(3, dtype=torch.int32, device="cuda")),
               dict(y=z(1)), dict(final_state=z(1, dtype=F32)), dict(history=z(2, 2, 3, 16, 8, dtype=F32)), dict(A=t["A"].cpu())):
        with pytest.raises(ValueError):
            ptq.head_scan(**{**args, **kw})
    for kw in (dict(u=None), dict(B=None), dict(A=3.0)):
        with pytest.raises(TypeError):
            ptq.head_scan(**{**args, **kw})
    for u, B, A in ((z(1, 2, 3, 257), z(1, 2, 8), z(3, dtype=F32)), (z(1, 2, 3, 8), z(1, 2, 129), z(3, dtype=F32)), (z(1, 2, 3, 8), z(1, 2, 2, 8), z(3, dtype=F32)),
                    (z(0, 2, 3, 8), z(0, 2, 8), z(3, dtype=F32)), (z(1, 0, 3, 8), z(1, 0, 8), z(3, dtype=F32)), (z(1, 1, 4097, 1), z(1, 1, 1), z(4097, dtype=F32))):
        with pytest.raises(ptq.PtqError) as e:               # too wide, too many states, groups that do not divide, nothing to do, too many heads
            ptq.head_scan(u, None, A, B, B)
        assert e.value.status == (2 if u.numel() else 1)     # a tensor without elements has no address
    with pytest.raises(ptq.PtqError):                       # a bias of what is not given
        ptq.head_scan(t["u"], None, t["A"], t["B"], t["C"], delta_bias=t["delta_bias"])
    h = ptq.head_scan_history(t["u"], 8)
    y = call(ptq, t, history=h)
    for kw in (dict(dy=y.float()), dict(dy=y[:, :3]), dict(history=h[:1]), dict(dfinal=t["state"][:1]), dict(dy=y.transpose(0, 1))):
        with pytest.raises(ValueError):
            ptq.head_scan_backward(**{**args, "dy": y, "history": h, **kw})
    with pytest.raises(TypeError):
        ptq.head_scan_step(t["state"], None, t["delta"][:, 0], t["A"], t["B"][:, 0], t["C"][:, 0])
    with pytest.raises(ValueError):
        ptq.head_scan(**args, stream=torch.cuda.Stream(device=0)) if torch.cuda.device_count() > 1 else ptq.head_scan_step(t["state"], t["u"], t["delta"], t["A"], t["B"], t["C"])


def test_refused_arguments_of_the_fp8_linears(ptq):
    x = torch.randn(5, 100, device="cuda", dtype=BF16)
    a, sa = ptq.fp8_quantize(x)
    w, ws = ptq.fp8_quantize_weight(torch.randn(30, 100, device="cuda"))
    raw = torch.zeros(30, 100, dtype=torch.uint8, device="cuda").view(E4M3)
    for f in (lambda: ptq.fp8_quantize(x.double()), lambda: ptq.fp8_quantize(x.t()), lambda: ptq.fp8_quantize(x, scales=sa[:2]),
              lambda: ptq.fp8_quantize(x, codes=torch.empty(5, 100, device="cuda")), lambda: ptq.fp8_quantize(torch.zeros(4, 6, 8, device="cuda")[:, :3]),
              lambda: ptq.fp8_quantize_weight(x[0]), lambda: ptq.fp8_matmul(a, sa, w, ws, dtype=torch.float64), lambda: ptq.fp8_matmul(x, sa, w, ws),
              lambda: ptq.fp8_matmul(a, sa[:, :0], w, ws), lambda: ptq.fp8_matmul(a, sa, w[:, :64], ws), lambda: ptq.fp8_matmul(a, sa, w, ws[:, :0]),
              lambda: ptq.fp8_matmul(a, sa, w, ws, bias=x[0]), lambda: ptq.fp8_matmul(a, sa, w, ws, y=torch.empty(5, 31, device="cuda")),
              lambda: ptq.fp8_matmul(a, sa, w, ws, dtype=F16, y=torch.empty(5, 30, device="cuda")), lambda: ptq.fp8_linear(x[:, :64], w, ws),
              lambda: ptq.fp8_linear(x, w.cpu(), ws), lambda: ptq.fp8_linear(x, w, ws.double()), lambda: ptq.fp8_linear(x, w, ws, y=torch.empty(5, 30, device="cuda"))):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ptq.fp8_linear(x, raw, ws), lambda: ptq.fp8_matmul(raw[:, :100], sa[:1].expand(30, 1), w, ws), lambda: ptq.fp8_linear(x[:0], w, ws),
              lambda: ptq.fp8_quantize(x[:, :0]), lambda: ptq.fp8_quantize(torch.zeros(2, 65537, device="cuda"))):
        with pytest.raises(ptq.PtqError):                   # rows that do not begin on 16 bytes, nothing to do, too wide
            f()
    with pytest.raises(TypeError):
        ptq.fp8_linear(None, w, ws)


def test_far_offsets(ptq):
    """Rows whose offsets pass 2^31 elements (and 2^32 bytes)."""
    pitch = (1 << 26) + 64
    base = torch.empty(80 * pitch + 256, dtype=torch.uint8, device="cuda").view(BF16)   # 5 GB, only a few rows of it are used
    pitch //= 2
    gen = torch.Generator().manual_seed(1)
    cut = {"u": (0, 64), "B": (64, 16), "C": (80, 16), "delta": (96, 2)}
    vals = torch.randn(1, 79, 98, generator=gen).to(BF16).cuda()
    far = {k: base.as_strided((1, 79, n), (0, pitch, 1), lo) for k, (lo, n) in cut.items()}
    for k, (lo, n) in cut.items():
        far[k].copy_(vals[..., lo:lo + n])
    near = {k: v.contiguous() for k, v in far.items()}
    A = torch.tensor([-0.5, -2.0], device="cuda")
    w, ws = ptq.fp8_quantize_weight(torch.randn(40, 64, device="cuda"))
    outs = []
    for t in (far, near):
        u = t["u"].unflatten(-1, (2, 32))
        h = ptq.head_scan_history(u, 16)
        y = ptq.head_scan(u, t["delta"], A, t["B"], t["C"], history=h, reverse=True)
        g = ptq.head_scan_backward(y, u, t["delta"], A, t["B"], t["C"], h, reverse=True)
        state = torch.ones(79, 2, 32, 16, device="cuda")     # one token of each of 79 sequences
        ys = ptq.head_scan_step(state, u[0], t["delta"][0], A, t["B"][0], t["C"][0])
        a, sa = ptq.fp8_quantize(t["u"][0])
        outs.append([y, *g.values(), ys, state, a.view(torch.uint8), sa, ptq.fp8_linear(t["u"][0], w, ws), ptq.fp8_linear(t["u"][0, :9], w, ws)])
    assert same(*outs)
    # results as far apart: written where they belong
    wide = torch.as_strided(base, (79, 40), (pitch, 1), 128)
    ptq.fp8_linear(near["u"][0], w, ws, y=wide)
    assert torch.equal(wide, outs[1][-2])
    del base, far, wide, outs
    # a dense output and a history of more than 2^31 elements: their last rows
    L = (1 << 15) + 64
    u = torch.zeros(1, L, 256, 256, dtype=BF16, device="cuda")
    u[0, -64:] = torch.randn(64, 256, 256, generator=gen).to(BF16).cuda()
    B = torch.randn(1, L, 8, generator=gen).to(BF16).cuda()
    A = -torch.ones(256, device="cuda")
    y = ptq.head_scan(u, None, A, B, B)
    tail = ptq.head_scan(u[:, -64:].contiguous(), None, A, B[:, -64:].contiguous(), B[:, -64:].contiguous())
    assert torch.equal(y[:, -64:], tail) and (y[0, :-64:4096] == 0).all()


def test_expanded_inputs_get_one_gradient_per_token(ptq):
    """B and C shared by all sequences through a pitch of zero: their gradients are dense, and their sum is the shared tensor's."""
    t = make(4, F32, 3, 20, 2, 16, 8)
    for k in ("B", "C"):
        t[k] = t[k][:1].contiguous().expand(3, 20, 1, 8)
    full = {**t, **{k: t[k].contiguous() for k in ("B", "C")}}
    dy = torch.randn(3, 20, 2, 16, device="cuda")
    got = []
    for x in (t, full):
        h = ptq.head_scan_history(x["u"], 8)
        call(ptq, x, history=h)
        got.append(back(ptq, x, dy, h))
    assert got[0]["B"].shape == (3, 20, 1, 8) and all(torch.equal(got[0][k], got[1][k]) for k in ("u", "A", "B", "C", "delta"))


def test_a_block_with_heads_in_both_directions(ptq):
    """norm, in_proj, then per direction convolution and scan, the gated norm, out_proj, residual and the next norm; the gradients through norm and
    scan: every operator against 64 bits on what the one before it gave."""
    gen = torch.Generator().manual_seed(11)
    r = lambda *s: torch.randn(*s, generator=gen)
    B, T, C, H, P, N = 3, 197, 96, 4, 32, 16
    D = H * P
    f64 = lambda t: t.double().cpu()
    f = 2.0 ** -10                                           # of |value| + 1: every operator's own tests hold the tight bounds

    def agrees(got, want, what, more=0.0):
        close(got, want, want.abs() + 1.0, f + more, what)

    def linear(x, n, k, what):
        w, ws = ptq.fp8_quantize_weight((r(n, k) / k ** 0.5).cuda())
        y = ptq.fp8_linear(x, w, ws)
        a, sa = ptq.fp8_quantize(x)
        dequantized = (f64(a.float()) * f64(sa).repeat_interleave(128, -1)[..., :k])
        weights = f64(w.float()) * f64(ws).repeat_interleave(128, 1)[:, :k].repeat_interleave(128, 0)[:n]
        agrees(y, dequantized @ weights.t(), what)
        # and against what was not quantized: a value is off by 2^-4 of itself, or 2^-10 of the largest of its block (the least step of a code)
        full = f64(x) @ weights.t()
        lim = (2.0 ** -4 * f64(x).abs() + 2.0 ** -10 * torch.nn.functional.pad(f64(x).abs(), (0, -k % 128)).unflatten(-1, (-1, 128)).amax(-1).repeat_interleave(
            128, -1)[..., :k]) @ weights.abs().t()
        assert ((f64(y) - full).abs() <= lim + 2.0 ** -10 * (full.abs() + 1)).all(), what
        return y
    stream, out, scale, w_norm = r(B, T, C).cuda(), r(B, T, C).half().cuda(), r(C).abs().cuda(), r(C).abs().cuda()
    x, stream2 = ptq.block_norm(out, w_norm, residual=stream, scale=scale)
    y64, _ = ref.norm(f64(out), f64(w_norm), residual=f64(stream), scale=f64(scale))
    agrees(x, y64, "norm")
    zxd = linear(x, 2 * D + 2 * N + H, C, "in_proj")
    z, xbc, delta = zxd[..., :D], zxd[..., D:2 * D + 2 * N], zxd[..., 2 * D + 2 * N:]
    total, kept = None, []
    for reverse in (False, True):
        cw, cb = (r(D + 2 * N, 4) / 2).cuda(), (r(D + 2 * N) / 5).cuda()
        u = ptq.short_conv(xbc, cw, cb, reverse=reverse)
        agrees(u, ref.conv(f64(xbc), f64(cw), f64(cb), reverse=reverse)[0], "convolution")
        t = {"u": u[..., :D].unflatten(-1, (H, P)), "delta": delta, "A": -(r(H).abs() + 0.5).cuda(), "B": u[..., D:D + N], "C": u[..., D + N:], "D": r(H).cuda(),
             "delta_bias": (r(H) - 3).cuda(), "state": None, "lengths": None}
        history = ptq.head_scan_history(t["u"], N)
        y = call(ptq, t, history=history, reverse=reverse)
        kept.append((t, history, reverse))
        value, sc, F = heads_ref.solve(t, reverse=reverse)
        close(y, value["y"], sc["y"], heads_ref.factor("y", F16, F), "scan")
        total = y if total is None else total + y
    flat, w2 = total.flatten(-2), r(D).abs().cuda()
    normed = ptq.block_norm(flat, w2, gate=z)
    agrees(normed, ref.norm(f64(flat), f64(w2), gate=f64(z))[0], "gated norm")
    out2 = linear(normed, C, D, "out_proj")
    _, stream3 = ptq.block_norm(out2, w_norm, residual=stream2, scale=scale)
    agrees(stream3, f64(stream2) + f64(scale) * f64(out2), "residual stream behind the block")
    dnormed = r(B, T, D).half().cuda()
    g = ptq.block_norm_backward(dnormed, flat, w2, gate=z)
    dy = g["x"].unflatten(-1, (H, P)).contiguous()
    for t, history, reverse in kept:
        value, sc, F = heads_ref.solve(t, dy=dy, reverse=reverse)
        for k, v in back(ptq, t, dy, history, reverse=reverse).items():
            if v is not None:
                close(v, value[k], sc[k], heads_ref.factor(k, v.dtype, F), "d" + k)


def test_serving_token_by_token_follows_the_whole_sequence(ptq):
    """in_proj, convolution, scan with their states, as a generating program keeps them, against one call over the sequence."""
    gen = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=gen).cuda()
    B, T, C, H, P, N = 4, 12, 64, 2, 32, 16
    D = H * P
    w, ws = ptq.fp8_quantize_weight(r(D + 2 * N + H, C) / 8)
    x, cw, cb, A, skip, db = r(B, T, C).to(BF16), r(D + 2 * N, 4), r(D + 2 * N), -r(H).abs(), r(H), r(H) - 3
    xd = ptq.fp8_linear(x, w, ws)
    u = ptq.short_conv(xd[..., :D + 2 * N], cw, cb)
    cols = lambda u: (u[..., :D].unflatten(-1, (H, P)), u[..., D:D + N], u[..., D + N:])
    uu, Bm, Cm = cols(u)
    y = ptq.head_scan(uu, xd[..., D + 2 * N:], A, Bm, Cm, D=skip, delta_bias=db)
    taps, state = torch.zeros(B, 3, D + 2 * N, dtype=BF16, device="cuda"), torch.zeros(B, H, P, N, device="cuda")
    for i in range(T):
        xi = ptq.fp8_linear(x[:, i], w, ws)
        assert torch.allclose(xi.float(), xd[:, i].float(), rtol=2.0 ** -7, atol=2.0 ** -10)          # few rows are cut otherwise
        ui = ptq.short_conv(xd[:, i:i + 1, :D + 2 * N], cw, cb, state=taps, final_state=taps)
        assert torch.equal(ui, u[:, i:i + 1])
        ut, Bt, Ct = cols(ui[:, 0])
        yi = ptq.head_scan_step(state, ut, xd[:, i, D + 2 * N:], A, Bt, Ct, D=skip, delta_bias=db)
        assert torch.allclose(yi.float(), y[:, i].float(), rtol=2.0 ** -6, atol=2.0 ** -5)
