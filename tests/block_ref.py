"""The operators between a block's linears in 64 bits, from their definitions, on the CPU: references of the GPU tests.  Gradients come from
torch.autograd on these forward passes, in 64 bits.

Tolerances.  A result of type t may be off by half a step, eps(t) / 2 relative, and by what binary32 arithmetic does on the way.  The latter is
bounded by `scale`, the same expression evaluated on absolute values, times
  - norm and conv: 2^-19; the longest chain of roundings is a sum of up to 8192 terms, in pairs of lanes and warps (fewer than 64 additions in a
    row, 2^-18 at worst, if all errors had one sign; 2^-24 each), and a sigmoid (|z| 2^-23 relative, |z| < 16 here);
  - scan: 2^-20 (8 + 4 m) (1 + max |dt A|), m the longest memory, the maximum over the steps of m <- a m + 1.  A step's decay is off by
    2^-22 (power of two) + |dt A| 2^-21 (its argument: dt by 2^-22, rate and product by 2^-24 each), its input by 2^-21; a state sums m of
    these, a gradient multiplies two such states and a sigmoid.
"""
import torch

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def close(got, want, scale, factor, what=""):
    """|got - want| <= eps/2 |want| + factor * scale, element by element; NaN and infinities where the reference has them."""
    g, w = got.detach().double().cpu(), want.detach().double().cpu()
    assert g.shape == w.shape, (what, g.shape, w.shape)
    tiny = torch.finfo(got.dtype).tiny if got.dtype != F16 else 2.0 ** -24
    lim = half_step(got.dtype) * w.abs() + factor * torch.as_tensor(scale, dtype=torch.float64).expand_as(w) + tiny
    bad = ~((g - w).abs() <= lim)
    assert not bad.any(), "%s: %d of %d out of tolerance, worst excess %g at %g (got %g)" % (
        what, int(bad.sum()), bad.numel(), float(((g - w).abs() - lim)[bad].max()), float(w[bad][0]), float(g[bad][0]))


def positions(B, L, lengths, reverse):
    """Per sequence the tokens in the order of processing."""
    n = [L] * B if lengths is None else [min(max(int(v), 0), L) for v in lengths]
    return [list(range(k - 1, -1, -1)) if reverse else list(range(k)) for k in n]


def scan(u, delta, A, B, C, D=None, z=None, delta_bias=None, state=None, lengths=None, softplus=True, reverse=False):
    """y (zeros behind the ends), final state; all arguments 64-bit."""
    Bt, L, Dc = u.shape
    if B.dim() == 3:
        B, C = B[:, :, None], C[:, :, None]
    heads = torch.arange(Dc) // (Dc // B.shape[2])
    rows, finals = [], []
    for b, order in enumerate(positions(Bt, L, lengths, reverse)):
        h = torch.zeros(Dc, A.shape[1], dtype=torch.float64) if state is None else state[b]
        out = {}
        for p in order:
            e = delta[b, p] if delta_bias is None else delta[b, p] + delta_bias
            dt = torch.nn.functional.softplus(e, threshold=1e9) if softplus else e
            h = torch.exp(dt[:, None] * A) * h + (dt * u[b, p])[:, None] * B[b, p][heads]
            o = (h * C[b, p][heads]).sum(-1)
            if D is not None:
                o = o + D * u[b, p]
            out[p] = o if z is None else o * z[b, p] * torch.sigmoid(z[b, p])
        rows.append(torch.stack([out.get(p, torch.zeros(Dc, dtype=torch.float64)) for p in range(L)]))
        finals.append(h)
    return torch.stack(rows), torch.stack(finals)


def scan_factor(u, delta, A, delta_bias, softplus, lengths, reverse):
    """The scan's factor on `scale` (see above)."""
    Bt, L, _ = u.shape
    m_max = x_max = 0.0
    for b, order in enumerate(positions(Bt, L, lengths, reverse)):
        m = torch.zeros(A.shape, dtype=torch.float64)
        for p in order:
            e = delta[b, p] if delta_bias is None else delta[b, p] + delta_bias
            dt = torch.nn.functional.softplus(e, threshold=1e9) if softplus else e
            x = dt[:, None] * A
            m = torch.exp(x) * m + 1.0
            m_max, x_max = max(m_max, float(m.max())), max(x_max, float(x.abs().max()))
    return 2.0 ** -20 * (8 + 4 * m_max) * (1 + x_max)


def norm(x, weight=None, bias=None, residual=None, scale=None, gate=None, kind="rms", gate_at="in", eps=1e-5):
    silu = None if gate is None else gate * torch.sigmoid(gate)
    v = x * silu if gate is not None and gate_at == "in" else x
    r = v if scale is None else v * scale
    if residual is not None:
        r = r + residual
    d = r - r.mean(-1, keepdim=True) if kind == "layer" else r
    n = d / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    y = n if weight is None else n * weight
    if bias is not None:
        y = y + bias
    return (y * silu if gate is not None and gate_at == "out" else y), r


def conv(x, weight, bias=None, state=None, lengths=None, silu=True, reverse=False):
    """y (zeros behind the ends), final state."""
    B, L, Dc = x.shape
    W = weight.shape[1]
    rows, finals = [], []
    for b, order in enumerate(positions(B, L, lengths, reverse)):
        window = [torch.zeros(Dc, dtype=torch.float64)] * (W - 1) if state is None else list(state[b])
        out = {}
        for p in order:
            taps = window + [x[b, p]]
            pre = sum(t * weight[:, j] for j, t in enumerate(taps))
            if bias is not None:
                pre = pre + bias
            out[p] = pre * torch.sigmoid(pre) if silu else pre
            window = taps[1:]
        rows.append(torch.stack([out.get(p, torch.zeros(Dc, dtype=torch.float64)) for p in range(L)]))
        finals.append(torch.stack(window))
    return torch.stack(rows), torch.stack(finals)


def leaves(args):
    """64-bit CPU copies of the tensors of a dict that gradients are taken for; what is masked may be anything and becomes 0."""
    return {k: torch.nan_to_num(v.detach().double().cpu(), 0.0, 0.0, 0.0).requires_grad_() for k, v in args.items() if v is not None}


def gradients(outputs, cotangents, inputs):
    """d(sum of outputs times cotangents) / d inputs, zeros where nothing depends on an input."""
    total = sum((o * c.detach().double().cpu()).sum() for o, c in zip(outputs, cotangents) if c is not None)
    total = total + sum(0.0 * v.sum() for v in inputs.values())      # a result that depends on no input has a gradient too: zeros
    names = list(inputs)
    got = torch.autograd.grad(total, [inputs[n] for n in names], allow_unused=True)
    return {n: torch.zeros_like(inputs[n]) if g is None else g for n, g in zip(names, got)}
