"""Linear attention with a decay for each head in 64 bits, from its definition, on the CPU: the reference of its GPU tests.  Gradients come
from torch.autograd on the recurrence, in 64 bits.

Tolerances.  A result of type t may be off by half a step, eps(t) / 2 relative, and by what the arithmetic does on the way, which is bounded by
`scale`, the same sums over absolute values, times
  - F for binary32 results and for ddelta: in a chunk of 64 steps a product sums up to 8 x 3 partial sums on the tensor cores, cut off at
    2^-23 each (2^-18.4); operands have 22 bits at least, factors are off by 2^-21 and by their argument, at most 64 x 1.45 max |dt A| in binary32
    (2^-17.5 max |dt A|); m / 64 + 1 chunks follow one another, m the longest memory (the maximum over the steps of m <- a m + 1); a gradient multiplies two
    such results, and sums of pairs multiply three:  F = 2^-16 (1 + m / 64) (1 + max |dt A|);
  - half a step and F for y, du, dB and dC: each of their terms holds one operand that was rounded to the type.
"""
import torch

from block_ref import half_step, positions

F64 = torch.float64


def recurrence(u, dt, w, log_decay, B, C, D, state, lengths, reverse):
    """y (zeros behind the ends), final state; u [b,l,h,p], dt, w, log_decay [b,l,h], B, C [b,l,g,n]."""
    Bt, L, H, P = u.shape
    group = torch.arange(H) // (H // B.shape[2])
    rows, finals = [], []
    for b, order in enumerate(positions(Bt, L, lengths, reverse)):
        S = torch.zeros(H, P, B.shape[3], dtype=F64) if state is None else state[b]
        out = {}
        for t in order:
            S = torch.exp(log_decay[b, t])[:, None, None] * S + (w[b, t][:, None] * u[b, t])[:, :, None] * B[b, t][group][:, None]
            y = (S * C[b, t][group][:, None]).sum(-1)
            out[t] = y if D is None else y + D[:, None] * u[b, t]
        rows.append(torch.stack([out.get(t, torch.zeros(H, P, dtype=F64)) for t in range(L)]))
        finals.append(S)
    return torch.stack(rows), torch.stack(finals)


NAMES = ("u", "delta", "A", "B", "C", "D", "delta_bias", "state")


def grouped(v):
    return v[:, :, None] if v.dim() == 3 else v


def solve(t, reverse=False, softplus=True, scale_input=True, dy=None, dfinal=None):
    """Values, gradients and scales of the inputs t (a dict by argument name): three dicts with y, final and the gradients by argument name, and F."""
    x = {k: None if t.get(k) is None else torch.nan_to_num(t[k].detach().double().cpu(), 0.0, 0.0, 0.0).requires_grad_() for k in NAMES}
    lengths = None if t.get("lengths") is None else t["lengths"].tolist()
    u = x["u"]
    if x["delta"] is None:
        e, dt = None, torch.ones(u.shape[:3], dtype=F64)
    else:
        e = x["delta"] if x["delta_bias"] is None else x["delta"] + x["delta_bias"]
        dt = torch.nn.functional.softplus(e, threshold=1e9) if softplus else e
    w = dt if scale_input else torch.ones_like(dt)
    y, final = recurrence(u, dt, w, dt * x["A"], grouped(x["B"]), grouped(x["C"]), x["D"], x["state"], lengths, reverse)
    value = {"y": y.detach(), "final": final.detach()}
    # the same with magnitudes; log decays and input factors as leaves of their own
    a = {k: None if x[k] is None else x[k].detach().abs().requires_grad_() for k in ("u", "B", "C", "D", "state")}
    ld, wa = (dt * x["A"]).detach().requires_grad_(), w.detach().abs().requires_grad_()
    ya, fa = recurrence(a["u"], None, wa, ld, grouped(a["B"]), grouped(a["C"]), a["D"], a["state"], lengths, reverse)
    scale = {"y": ya.detach(), "final": fa.detach()}
    m_max = 0.0
    for b, order in enumerate(positions(u.shape[0], u.shape[1], lengths, reverse)):
        m = torch.zeros(u.shape[2], dtype=F64)
        for p in order:
            m = torch.exp(ld[b, p].detach()) * m + 1.0
            m_max = max(m_max, float(m.max()))
    F = 2.0 ** -16 * (1 + m_max / 64) * (1 + float(ld.detach().clamp(min=-100.0).abs().max()))
    if dy is None:
        return value, scale, F

    def pull(outs, cots, wanted):
        total = sum((o * c).sum() for o, c in zip(outs, cots) if c is not None) + sum(0.0 * v.sum() for v in wanted.values())
        got = torch.autograd.grad(total, list(wanted.values()), allow_unused=True)
        return {k: torch.zeros_like(v) if g is None else g for (k, v), g in zip(wanted.items(), got)}
    cots = [None if c is None else c.detach().double().cpu() for c in (dy, dfinal)]
    if lengths is not None:
        live = torch.tensor([[i < n for i in range(u.shape[1])] for n in lengths])
        cots[0] = torch.where(live[..., None, None], cots[0], 0.0)
    value.update(pull((y, final), cots, {k: v for k, v in x.items() if v is not None}))
    s = pull((ya, fa), [None if c is None else c.abs() for c in cots], {**{k: v for k, v in a.items() if v is not None}, "ld": ld, "w": wa})
    dts, A = dt.detach().abs(), x["A"].detach().abs()
    s["A"] = (dts * s["ld"]).sum((0, 1))
    s["delta"] = torch.where(s["ld"] == 0, 0.0, A * s["ld"]) + (s["w"] if scale_input else 0.0)
    s["delta_bias"] = s["delta"].sum((0, 1))
    scale.update({k: s[k] for k in value if k in s})
    return value, scale, F


def factor(name, dtype, F):
    """What multiplies `scale` for the result `name` of type dtype."""
    return F + (half_step(dtype) if name in ("y", "u", "B", "C") and dtype != torch.float32 else 0.0)
