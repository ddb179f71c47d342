"""What a Mamba block computes between its quantized linears: the cases these operators are timed on.

``family`` "scan"   the gated linear recurrence between dt_proj and out_proj: ``gated_scan`` over a batch of token
                    sequences, ``gated_scan_backward`` (training), ``gated_scan_step`` (one token per sequence)
           "norm"   ``block_norm`` before in_proj (residual and scale) or behind the scan (gate), and its backward pass
           "conv"   ``short_conv``, the causal depthwise convolution behind in_proj, and its backward pass
``mode``   "infer" (forward pass), "train" (forward and backward pass), "step" (scan only: one token per sequence)

Where ``own`` is false, ``run`` computes the same in plain torch operations.
"""
import math

import torch

own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"fp16": 2, "bf16": 2, "fp32": 4}


def _scan(mode, dtype, B, L, D, N, G=1, gate=True, skip=True, state=False, ragged=False, reverse=False):
    return {"family": "scan", "mode": mode, "dtype": dtype, "B": B, "L": L, "D": D, "N": N, "G": G, "gate": gate, "skip": skip,
            "state": state, "ragged": ragged, "reverse": reverse}


def _norm(mode, dtype, M, D, kind="rms", residual="", scale=False, gate="", bias=False):
    return {"family": "norm", "mode": mode, "dtype": dtype, "M": M, "D": D, "kind": kind, "residual": residual, "scale": scale,
            "gate": gate, "bias": bias}


def _conv(mode, dtype, B, L, D, W=4, state=False, ragged=False, reverse=False):
    return {"family": "conv", "mode": mode, "dtype": dtype, "B": B, "L": L, "D": D, "W": W, "state": state, "ragged": ragged,
            "reverse": reverse}


def listed():
    return [
        # one image through one block of the smallest backbone: latency
        dict(_scan("infer", "fp16", 1, 197, 384, 16), name="scan, 1 image"),
        # a batch through one block of the middle backbone, the direction that runs from the last token to the first
        dict(_scan("infer", "fp16", 128, 197, 768, 16, reverse=True), name="scan, batch 128"),
        # few long sequences, read in pieces: states come in and go out, nothing is a multiple of anything
        dict(_scan("infer", "bf16", 2, 20011, 1024, 16, state=True), name="scan, 2 long sequences"),
        # fine-tuning one block of the smallest backbone
        dict(_scan("train", "fp16", 64, 197, 384, 16), name="scan training, batch 64"),
        # fine-tuning on sequences of different lengths padded to one, two groups of channels, no gate
        dict(_scan("train", "bf16", 6, 2050, 1000, 8, G=2, gate=False, state=True, ragged=True), name="scan training, ragged"),
        # a hierarchical backbone's second stage in binary32, one state per channel, without gate
        dict(_scan("train", "fp32", 32, 784, 384, 1, gate=False), name="scan training, 1 state fp32"),
        # one token of one sequence: latency
        dict(_scan("step", "fp16", 1, 1, 1536, 16, state=True), name="scan step, 1 sequence"),
        # one token of each of many sequences served together
        dict(_scan("step", "bf16", 1024, 1, 1536, 16, state=True), name="scan step, 1024 sequences"),
        # the norm of a gated scan output in front of out_proj, one image: latency
        dict(_norm("infer", "fp16", 197, 384, gate="in"), name="gated norm, 1 image"),
        # residual, layer scale and norm in front of in_proj, fine-tuning at batch 256; the residual stream is binary32
        dict(_norm("train", "bf16", 256 * 197, 768, kind="layer", residual="fp32", scale=True, bias=True), name="norm training, batch 256"),
        # fine-tuning, the convolution of the middle backbone
        dict(_conv("train", "fp16", 64, 197, 768), name="conv training, batch 64"),
        # one token of each of the served sequences
        dict(_conv("infer", "bf16", 256, 1, 1536, state=True), name="conv step, 256 sequences"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, direction and type, sizes over the whole range, odd ones among them."""
    while True:
        dtype = rng.choice(["fp16", "bf16", "bf16", "fp32"])
        family = rng.choices(["scan", "norm", "conv"], [4, 2, 2])[0]
        D = rng.choice([192, 384, 768, 8 * _log(rng, 2, 256), _log(rng, 3, 2000)])
        if family == "scan":
            mode = rng.choices(["infer", "train", "step"], [2, 2, 1])[0]
            L = 1 if mode == "step" else rng.choice([49, 196, 197, 784, _log(rng, 1, 16384)])
            N = rng.choice([16, 16, 16, 1, 8, rng.randint(1, 32)])
            G = rng.choice([g for g in (1, 1, 1, 2, 4) if D % g == 0])
            c = _scan(mode, dtype, _log(rng, 1, 128), L, D, N, G, gate=rng.random() < 0.6, skip=rng.random() < 0.8,
                      state=mode == "step" or rng.random() < 0.3, ragged=mode != "step" and rng.random() < 0.3,
                      reverse=mode != "step" and rng.random() < 0.4)
            if c["B"] * c["L"] * D * N > 1.2e8:
                continue
        elif family == "norm":
            kind, residual = rng.choice(["rms", "layer"]), rng.choice(["", dtype, "fp32"])
            c = _norm(rng.choice(["infer", "train"]), dtype, _log(rng, 1, 50000), D, kind, residual, scale=residual != "" and rng.random() < 0.5,
                      gate=rng.choice(["", "in", "out"]), bias=rng.random() < 0.5)
            if c["M"] * D > 3.8e7:
                continue
        else:
            L = rng.choice([1, 49, 196, 197, 784, _log(rng, 1, 16384)])
            c = _conv(rng.choice(["infer", "train"]), dtype, _log(rng, 1, 256), L, D, rng.randint(2, 4), state=rng.random() < 0.4,
                      ragged=rng.random() < 0.3, reverse=rng.random() < 0.4)
            if c["B"] * L * D > 3.8e7:
                continue
        return c


# ---------------------------------------------------------------------------------------------------------- inputs
def _normal(gen, shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _uniform(gen, shape, lo, hi):
    return torch.rand(shape, generator=gen, device="cuda") * (hi - lo) + lo


def _lengths(gen, c):
    """Ragged batches hold one full sequence, one of a single token and, from three on, an empty one."""
    B, L = c["B"], c["L"]
    n = torch.randint(1, L + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    n[0] = L
    if B > 1:
        n[1] = 1
    if B > 2:
        n[2] = 0
    return n


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    T = TYPES[case["dtype"]]
    s = {"case": case}
    if case["family"] == "scan":
        B, L, D, N, G = (case[k] for k in "BLDNG")
        # u and the gate as the halves of in_proj's output, B and C as the columns of x_proj's behind the low-rank dt
        xz = _normal(gen, (B, L, 2 * D), T)
        r = (D + 31) // 32
        dbc = _normal(gen, (B, L, r + 2 * G * N), T)
        s["u"], s["delta"] = xz[..., :D], _normal(gen, (B, L, D), T, 0.5)
        s["z"] = xz[..., D:] if case["gate"] else None
        s["B"] = dbc[..., r:r + G * N].unflatten(-1, (G, N))
        s["C"] = dbc[..., r + G * N:].unflatten(-1, (G, N))
        # decays from slow to fast, dt around 0.001 .. 0.1, as such blocks are initialised and stay
        s["A"] = -torch.arange(1, N + 1, device="cuda", dtype=torch.float32) * torch.exp(_normal(gen, (D, N), scale=0.3))
        dt = torch.exp(_uniform(gen, (D,), math.log(1e-3), math.log(0.1)))
        s["delta_bias"] = dt + torch.log(-torch.expm1(-dt))
        s["D"] = _normal(gen, (D,)) if case["skip"] else None
        s["state"] = _normal(gen, (B, D, N)) if case["state"] else None
        s["final"] = torch.empty(B, D, N, device="cuda") if case["state"] else None
        s["lengths"] = _lengths(gen, case) if case["ragged"] else None
        if case["mode"] == "train":
            s["dy"] = _normal(gen, (B, L, D), T)
            s["dfinal"] = _normal(gen, (B, D, N)) if case["state"] else None
        if case["mode"] == "step":
            for k in ("u", "delta", "z", "B", "C"):
                s[k] = None if s[k] is None else s[k][:, 0]
    elif case["family"] == "norm":
        M, D = case["M"], case["D"]
        s["x"] = _normal(gen, (M, D), T)
        s["weight"] = 1.0 + _normal(gen, (D,), scale=0.2)
        s["bias"] = _normal(gen, (D,), scale=0.2) if case["bias"] else None
        s["scale"] = _uniform(gen, (D,), 0.05, 1.0) if case["scale"] else None
        s["residual"] = _normal(gen, (M, D), TYPES[case["residual"]], 2.0) if case["residual"] else None
        s["gate"] = _normal(gen, (M, 2 * D), T)[:, D:] if case["gate"] else None     # the second half of in_proj's output
        if case["mode"] == "train":
            s["dy"] = _normal(gen, (M, D), T)
            s["dr"] = _normal(gen, (M, D), TYPES[case["residual"]]) if case["residual"] else None
    else:
        B, L, D, W = (case[k] for k in "BLDW")
        s["x"] = _normal(gen, (B, L, 2 * D), T)[..., :D]                             # the first half of in_proj's output
        s["weight"] = _uniform(gen, (D, W), -1.0, 1.0) / math.sqrt(W)
        s["bias"] = _normal(gen, (D,), scale=0.2)
        s["state"] = _normal(gen, (B, W - 1, D), T) if case["state"] else None
        s["final"] = torch.empty(B, W - 1, D, device="cuda", dtype=T) if case["state"] else None
        s["lengths"] = _lengths(gen, case) if case["ragged"] else None
        if case["mode"] == "train":
            s["dy"] = _normal(gen, (B, L, D), T)
            s["dfinal"] = _normal(gen, (B, W - 1, D), T) if case["state"] else None
    return s


# ---------------------------------------------------------------------------------------------------------- one pass
def run(state):
    f = {"scan": (_plain_scan, _own_scan), "norm": (_plain_norm, _own_norm), "conv": (_plain_conv, _own_conv)}[state["case"]["family"]]
    return f[1 if own else 0](state)


def _own_scan(s):
    import paper_2412_20386_b200 as ptq
    c = s["case"]
    if c["mode"] == "step":
        y = ptq.gated_scan_step(s["state"], s["u"], s["delta"], s["A"], s["B"], s["C"], D=s["D"], z=s["z"], delta_bias=s["delta_bias"],
                                new_state=s["final"])
        return {"y": y, "final": s["final"]}
    args = (s["u"], s["delta"], s["A"], s["B"], s["C"])
    kw = dict(D=s["D"], z=s["z"], delta_bias=s["delta_bias"], state=s["state"], lengths=s["lengths"], reverse=c["reverse"])
    if c["mode"] == "infer":
        y = ptq.gated_scan(*args, **kw, final_state=s["final"])
        return {"y": y, "final": s["final"]}
    history = ptq.scan_history(s["u"], c["N"])
    y = ptq.gated_scan(*args, **kw, final_state=s["final"], history=history)
    g = ptq.gated_scan_backward(s["dy"], *args, history, **kw, dfinal=s["dfinal"])
    return {"y": y, "final": s["final"], **{"d" + k: v for k, v in g.items()}}


def _own_norm(s):
    import paper_2412_20386_b200 as ptq
    c = s["case"]
    kw = dict(residual=s["residual"], scale=s["scale"], gate=s["gate"], kind=c["kind"], gate_at=c["gate"] or "in", eps=1e-5)
    out = ptq.block_norm(s["x"], s["weight"], s["bias"], **kw)
    y, r = out if s["residual"] is not None else (out, None)
    if c["mode"] == "infer":
        return {"y": y, "r": r}
    g = ptq.block_norm_backward(s["dy"], s["x"], s["weight"], s["bias"], dresidual_out=s["dr"], **kw)
    return {"y": y, "r": r, **{"d" + k: v for k, v in g.items()}}


def _own_conv(s):
    import paper_2412_20386_b200 as ptq
    c = s["case"]
    kw = dict(state=s["state"], lengths=s["lengths"], reverse=c["reverse"])
    y = ptq.short_conv(s["x"], s["weight"], s["bias"], **kw, final_state=s["final"])
    if c["mode"] == "infer":
        return {"y": y, "final": s["final"]}
    g = ptq.short_conv_backward(s["dy"], s["x"], s["weight"], s["bias"], **kw, dfinal=s["dfinal"])
    return {"y": y, "final": s["final"], **{"d" + k: v for k, v in g.items()}}


# ---------------------------------------------------------------------------------------------------------- plain forms
def _order(s, B, L):
    """(positions in the order of processing [B,L], which of them hold a token [B,L])"""
    i = torch.arange(L, device="cuda").expand(B, L)
    n = torch.full((B, 1), L, device="cuda") if s["lengths"] is None else s["lengths"].long()[:, None]
    valid = i < n
    return (torch.where(valid, n - 1 - i, i) if s["case"]["reverse"] else i), valid


def _rows(t, pos, valid):
    """Rows of t [B,L,...] in the order of processing, in 32 bits, zeros where there is no token."""
    idx = pos.reshape(pos.shape + (1,) * (t.dim() - 2)).expand(t.shape)
    keep = valid.reshape(valid.shape + (1,) * (t.dim() - 2))
    return torch.where(keep, t.gather(1, idx).float(), 0.0)


def _back(t, pos, valid, dtype):
    """The inverse of _rows, rounded."""
    keep = valid.reshape(valid.shape + (1,) * (t.dim() - 2))
    idx = pos.reshape(pos.shape + (1,) * (t.dim() - 2)).expand(t.shape)
    return torch.zeros(t.shape, dtype=dtype, device="cuda").scatter_(1, idx, torch.where(keep, t, 0.0).to(dtype))


def _states(a, x, h0):
    """h_i = a_i h_{i-1} + x_i for all i of dimension 1: within about sqrt(L) blocks side by side, then from block to block."""
    B, L = x.shape[:2]
    n = max(1, math.isqrt(L))
    c = -(-L // n)
    n = -(-L // c)
    if n * c > L:
        fill = (B, n * c - L) + x.shape[2:]
        a, x = torch.cat([a, a.new_ones(fill)], 1), torch.cat([x, x.new_zeros(fill)], 1)
    a, x = (t.reshape((B, n, c) + t.shape[2:]).clone() for t in (a, x))
    for i in range(1, c):
        x[:, :, i] += a[:, :, i] * x[:, :, i - 1]
        a[:, :, i] *= a[:, :, i - 1]
    carry = [h0]
    for j in range(n - 1):
        carry.append(x[:, j, -1] + a[:, j, -1] * carry[-1])
    a *= torch.stack(carry, 1)[:, :, None]
    return (x + a).reshape((B, n * c) + x.shape[3:])[:, :L]


def _plain_scan(s):
    c = s["case"]
    T = TYPES[c["dtype"]]
    step = c["mode"] == "step"
    tok = {k: None if s[k] is None else (s[k][:, None] if step else s[k]) for k in ("u", "delta", "z", "B", "C")}
    B, L, D = tok["u"].shape
    N, G = c["N"], c["G"]
    pos, valid = _order(s, B, L)
    u, Bm, Cm = (_rows(tok[k], pos, valid) for k in ("u", "B", "C"))
    z = None if tok["z"] is None else _rows(tok["z"], pos, valid)
    e = _rows(tok["delta"], pos, valid) + s["delta_bias"]
    dt = torch.where(valid[..., None], torch.where(e > 20, e, torch.log1p(torch.exp(e))), 0.0)
    per = lambda t: t.repeat_interleave(D // G, 2)                                   # [B,L,G,N] -> [B,L,D,N]
    A = s["A"]
    h0 = torch.zeros(B, D, N, device="cuda") if s["state"] is None else s["state"]
    a = torch.exp(dt[..., None] * A)
    h = _states(a, (dt * u)[..., None] * per(Bm), h0)
    o = (h * per(Cm)).sum(-1)
    if s["D"] is not None:
        o = o + s["D"] * u
    gate = None if z is None else torch.sigmoid(z)
    y = o if z is None else o * z * gate
    out = {"y": _back(y, pos, valid, T), "final": None if s["final"] is None else h[:, -1].clone()}
    if step:
        out["y"] = out["y"][:, 0]
    if c["mode"] != "train":
        return out
    dy = _rows(s["dy"], pos, valid)
    do = dy if z is None else dy * z * gate
    last = torch.zeros(B, D, N, device="cuda") if s["dfinal"] is None else s["dfinal"]
    after = torch.cat([a[:, 1:], a.new_ones(B, 1, D, N)], 1)
    g = _states(after.flip(1), (do[..., None] * per(Cm)).flip(1), last).flip(1)
    q = g * a * torch.cat([h0[:, None], h[:, :-1]], 1)
    gB = (g * per(Bm)).sum(-1)
    ddelta = (u * gB + (q * A).sum(-1)) * torch.sigmoid(e)
    ddelta = torch.where(valid[..., None], ddelta, 0.0)
    du = dt * gB
    if s["D"] is not None:
        du = du + s["D"] * do
    split = lambda t: t.reshape(B, L, G, D // G, N).sum(3)
    out["du"], out["ddelta"] = _back(du, pos, valid, T), _back(ddelta, pos, valid, T)
    out["dA"] = (q * dt[..., None]).sum((0, 1))
    out["dB"] = _back(split(g * (dt * u)[..., None]), pos, valid, T)
    out["dC"] = _back(split(h * do[..., None]), pos, valid, T)
    out["dD"] = None if s["D"] is None else (u * do).sum((0, 1))
    out["dz"] = None if z is None else _back(dy * o * gate * (1 + z * (1 - gate)), pos, valid, T)
    out["ddelta_bias"] = ddelta.sum((0, 1))
    out["dstate"] = None if s["state"] is None else a[:, 0] * g[:, 0]
    return out


def _plain_norm(s):
    c = s["case"]
    T, eps = TYPES[c["dtype"]], 1e-5
    x = s["x"].float()
    gate = None if s["gate"] is None else s["gate"].float()
    sig = None if gate is None else torch.sigmoid(gate)
    v = x * gate * sig if c["gate"] == "in" else x
    r = v if s["scale"] is None else v * s["scale"]
    if s["residual"] is not None:
        r = r + s["residual"].float()
    d = r - r.mean(-1, keepdim=True) if c["kind"] == "layer" else r
    rstd = torch.rsqrt((d * d).mean(-1, keepdim=True) + eps)
    n = d * rstd
    t = n * s["weight"]
    if s["bias"] is not None:
        t = t + s["bias"]
    y = t * gate * sig if c["gate"] == "out" else t
    out = {"y": y.to(T), "r": None if s["residual"] is None else r.to(s["residual"].dtype)}
    if c["mode"] != "train":
        return out
    dy = s["dy"].float()
    dgate = None
    slope = None if gate is None else sig * (1 + gate * (1 - sig))
    if c["gate"] == "out":
        dgate, dy = dy * t * slope, dy * gate * sig
    dn = dy * s["weight"]
    dr = dn - n * (dn * n).mean(-1, keepdim=True)
    if c["kind"] == "layer":
        dr = dr - dn.mean(-1, keepdim=True)
    dr = dr * rstd
    if s["dr"] is not None:
        dr = dr + s["dr"].float()
    dv = dr if s["scale"] is None else dr * s["scale"]
    if c["gate"] == "in":
        dgate, dx = dv * x * slope, dv * gate * sig
    else:
        dx = dv
    out["dx"], out["dweight"] = dx.to(T), (dy * n).sum(0)
    out["dbias"] = None if s["bias"] is None else dy.sum(0)
    out["dresidual"] = None if s["residual"] is None else dr.to(s["residual"].dtype)
    out["dscale"] = None if s["scale"] is None else (dr * v).sum(0)
    out["dgate"] = None if gate is None else dgate.to(T)
    return out


def _plain_conv(s):
    c = s["case"]
    T, W = TYPES[c["dtype"]], c["W"]
    B, L, D = s["x"].shape
    pos, valid = _order(s, B, L)
    x = _rows(s["x"], pos, valid)
    before = torch.zeros(B, W - 1, D, device="cuda") if s["state"] is None else s["state"].float()
    full = torch.cat([before, x], 1)                                                 # row i + W - 1: token i
    pre = s["bias"] + sum(full[:, j:j + L] * s["weight"][:, j] for j in range(W))
    sig = torch.sigmoid(pre)
    out = {"y": _back(pre * sig, pos, valid, T), "final": None}
    n = torch.full((B,), L, device="cuda") if s["lengths"] is None else s["lengths"].long()
    tail = (n[:, None] + torch.arange(W - 1, device="cuda"))[..., None].expand(B, W - 1, D)
    if s["final"] is not None:
        out["final"] = full.gather(1, tail).to(T)
    if c["mode"] != "train":
        return out
    dpre = _rows(s["dy"], pos, valid) * sig * (1 + pre * (1 - sig))
    dfull = torch.zeros_like(full)
    for j in range(W):
        dfull[:, j:j + L] += dpre * s["weight"][:, j]
    if s["dfinal"] is not None:
        dfull.scatter_add_(1, tail, s["dfinal"].float())
    out["dx"] = _back(dfull[:, W - 1:], pos, valid, T)
    out["dweight"] = torch.stack([(dpre * full[:, j:j + L]).sum((0, 1)) for j in range(W)], 1)
    out["dbias"] = dpre.sum((0, 1))
    out["dstate"] = None if s["state"] is None else dfull[:, :W - 1].to(T)
    return out


# ---------------------------------------------------------------------------------------------------------- exact values
def exact(case, seed):
    """The definitions in 64 bits, token by token."""
    s = prepare(case, seed)
    d = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    return {"scan": _exact_scan, "norm": _exact_norm, "conv": _exact_conv}[case["family"]](case, d)


def _put(rows):
    """put(t, p, on, v): t[b, p[b]] = v[b] in the rows that have a token."""
    return lambda t, p, on, v: t.index_put_((rows, p), torch.where(on.reshape((-1,) + (1,) * (v.dim() - 1)), v, t[rows, p]))


def _tokens(case, s):
    """For every step of processing: the rows' positions and which rows have one [B]."""
    B, L = case["B"], case["L"]
    n = torch.full((B,), L, device="cuda") if s["lengths"] is None else s["lengths"].long()
    for i in range(L):
        on = i < n
        yield torch.where(on, n - 1 - i, 0) if case["reverse"] else torch.full_like(n, i), on


def _exact_scan(case, s):
    B, L, D, N, G, step = case["B"], case["L"], case["D"], case["N"], case["G"], case["mode"] == "step"
    if step:
        s = {**s, **{k: None if s[k] is None else s[k][:, None] for k in ("u", "delta", "z", "B", "C")}}
    rows, heads = torch.arange(B, device="cuda"), torch.arange(D, device="cuda") // (D // G)
    train, put = case["mode"] == "train", _put(rows)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    h = torch.zeros(B, D, N, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"]
    y = torch.zeros(B, L, D, dtype=torch.float64, device="cuda")
    kept, steps = [], list(_tokens(case, s))
    take = lambda name, p: s[name][rows, p]
    soft = lambda e: torch.clamp(e, min=0.0) + torch.log1p(torch.exp(-e.abs()))
    for p, on in steps:
        e = take("delta", p) + s["delta_bias"]
        dt, u = soft(e), take("u", p)
        new = torch.exp(dt[..., None] * s["A"]) * h + (dt * u)[..., None] * take("B", p)[:, heads]
        if train:
            kept.append(h)
        h = torch.where(on[:, None, None], new, h)
        o = (h * take("C", p)[:, heads]).sum(-1)
        if s["D"] is not None:
            o = o + s["D"] * u
        if s["z"] is not None:
            z = take("z", p)
            o = o * z / (1 + torch.exp(-z))
        put(y, p, on, o)
    out = {"y": y[:, 0] if step else y, "final": None if s["final"] is None else h}
    if not train:
        return out
    du, dd, dz = (torch.zeros(B, L, D, dtype=torch.float64, device="cuda") for _ in range(3))
    dB, dC = (torch.zeros(B, L, G, N, dtype=torch.float64, device="cuda") for _ in range(2))
    dA, dD, db = torch.zeros_like(s["A"]), torch.zeros(D, dtype=torch.float64, device="cuda"), torch.zeros(D, dtype=torch.float64, device="cuda")
    gh = torch.zeros_like(h) if s["dfinal"] is None else s["dfinal"].clone()
    for (p, on), before in zip(reversed(steps), reversed(kept)):
        e, u, dy = take("delta", p) + s["delta_bias"], take("u", p), take("dy", p)
        dt, Bt, Ct = soft(e), take("B", p)[:, heads], take("C", p)[:, heads]
        a = torch.exp(dt[..., None] * s["A"])
        now = a * before + (dt * u)[..., None] * Bt
        o = (now * Ct).sum(-1) + (s["D"] * u if s["D"] is not None else 0.0)
        do = dy
        if s["z"] is not None:
            z = take("z", p)
            sg = 1 / (1 + torch.exp(-z))
            do = dy * z * sg
            put(dz, p, on, dy * o * sg * (1 + z * (1 - sg)))
        do = torch.where(on[:, None], do, zero)
        k = on[:, None, None]
        g = gh + do[..., None] * Ct
        q = torch.where(k, g * a * before, zero)
        gb = (g * Bt).sum(-1)
        de = torch.where(on[:, None], (u * gb + (q * s["A"]).sum(-1)) / (1 + torch.exp(-e)), zero)
        put(dd, p, on, de)
        put(du, p, on, dt * gb + (s["D"] * do if s["D"] is not None else 0.0))
        put(dB, p, on, (g * (dt * u)[..., None]).reshape(B, G, -1, N).sum(2))
        put(dC, p, on, (now * do[..., None]).reshape(B, G, -1, N).sum(2))
        dA += (q * dt[..., None]).sum(0)
        dD += torch.where(on[:, None], u * do, zero).sum(0)
        db += de.sum(0)
        gh = torch.where(k, g * a, gh)
    out.update(du=du, ddelta=dd, dA=dA, dB=dB, dC=dC, dD=None if s["D"] is None else dD, dz=None if s["z"] is None else dz, ddelta_bias=db,
               dstate=None if s["state"] is None else gh)
    return out


def _exact_norm(case, s):
    """Gradients from those of the sum over dy*y + dr*r, term by term."""
    D = case["D"]
    g = s["gate"]
    silu = None if g is None else g / (1 + torch.exp(-g))
    turn = None if g is None else 1 / (1 + torch.exp(-g)) + g * torch.exp(-g) / (1 + torch.exp(-g)) ** 2
    alpha = 1.0 if s["scale"] is None else s["scale"]
    v = s["x"] * silu if case["gate"] == "in" else s["x"]
    r = alpha * v + (0.0 if s["residual"] is None else s["residual"])
    mu = r.sum(-1, keepdim=True) / D if case["kind"] == "layer" else torch.zeros_like(r[:, :1])
    sd = torch.sqrt(((r - mu) ** 2).sum(-1, keepdim=True) / D + 1e-5)
    n = (r - mu) / sd
    t = n * s["weight"] + (0.0 if s["bias"] is None else s["bias"])
    out = {"y": t * silu if case["gate"] == "out" else t, "r": None if s["residual"] is None else r}
    if case["mode"] != "train":
        return out
    dt = s["dy"] * silu if case["gate"] == "out" else s["dy"]
    dn = dt * s["weight"]
    back = dn - (n * dn).sum(-1, keepdim=True) / D * n
    if case["kind"] == "layer":
        back = back - dn.sum(-1, keepdim=True) / D
    dr = back / sd + (0.0 if s["dr"] is None else s["dr"])
    inner = case["gate"] == "in"
    out["dx"] = alpha * dr * silu if inner else alpha * dr
    out["dweight"] = (dt * n).sum(0)
    out["dbias"] = None if s["bias"] is None else dt.sum(0)
    out["dresidual"] = None if s["residual"] is None else dr
    out["dscale"] = None if s["scale"] is None else (dr * v).sum(0)
    out["dgate"] = None if g is None else (alpha * dr * s["x"] * turn if inner else s["dy"] * t * turn)
    return out


def _exact_conv(case, s):
    B, L, D, W = (case[k] for k in "BLDW")
    rows, w = torch.arange(B, device="cuda"), s["weight"]
    put = _put(rows)
    window = [torch.zeros(B, D, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"][:, j] for j in range(W - 1)]
    first = list(window)
    y = torch.zeros(B, L, D, dtype=torch.float64, device="cuda")
    kept, steps = [], list(_tokens(case, s))
    for p, on in steps:
        x = s["x"][rows, p]
        taps = window + [x]
        pre = s["bias"] + sum(t * w[:, j] for j, t in enumerate(taps))
        put(y, p, on, pre / (1 + torch.exp(-pre)))
        kept.append((taps, pre) if case["mode"] == "train" else None)
        window = [torch.where(on[:, None], b, a) for a, b in zip(window, taps[1:])]
    out = {"y": y, "final": None if s["final"] is None else torch.stack(window, 1)}
    if case["mode"] != "train":
        return out
    dx, dw, db = torch.zeros_like(y), torch.zeros_like(w), torch.zeros(D, dtype=torch.float64, device="cuda")
    # gradients of the window behind the last token, handed back from step to step
    dwin = [torch.zeros_like(first[0]) if s["dfinal"] is None else s["dfinal"][:, j] for j in range(W - 1)]
    for (p, on), (taps, pre) in zip(reversed(steps), reversed(kept)):
        k = on[:, None]
        sg = 1 / (1 + torch.exp(-pre))
        dp = torch.where(k, s["dy"][rows, p] * sg * (1 + pre * (1 - sg)), 0.0)
        db += dp.sum(0)
        dw += torch.stack([(dp * torch.where(k, t, 0.0)).sum(0) for t in taps], 1)
        dtaps = [dp * w[:, j] + (dwin[j - 1] if j > 0 else 0.0) for j in range(W)]
        put(dx, p, on, dtaps[-1])
        dwin = [torch.where(k, a, b) for a, b in zip(dtaps[:-1], dwin)]
    out.update(dx=dx, dweight=dw, dbias=db, dstate=None if s["state"] is None else torch.stack(dwin, 1))
    return out


# ---------------------------------------------------------------------------------------------------------- work
def work(case):
    e = BYTES[case["dtype"]]
    train = case["mode"] == "train"
    if case["family"] == "scan":
        B, L, D, N, G = (case[k] for k in "BLDNG")
        el, bc, st, par = B * L * D, 2 * B * L * G * N, B * D * N, D * (N + 2)
        gate, state = int(case["gate"]), int(case["state"])
        bytes_ = e * ((3 + gate) * el + bc) + 4 * (2 * state * st + par)
        flops = el * N * 7 + el * 8                        # exponent, decay, input, output; softplus and gate
        if train:                                          # the backward pass reads the same again, and dy
            bytes_ += e * ((3 + gate) * el + bc) + e * ((2 + gate) * el + bc) + 4 * (3 * state * st + 2 * par)
            flops += el * N * 18 + el * 16
        return {"bytes": bytes_, "flops": flops}
    if case["family"] == "norm":
        el, D = case["M"] * case["D"], case["D"]
        res, gate = BYTES.get(case["residual"], 0), e * int(case["gate"] != "")
        bytes_ = el * (2 * e + 2 * res + gate) + 4 * D * 3
        if train:
            bytes_ += el * (3 * e + 3 * res + 2 * gate) + 4 * D * 6
        return {"bytes": bytes_, "flops": el * (10 + (25 if train else 0))}
    B, L, D, W = (case[k] for k in "BLDW")
    el, st = B * L * D, B * D * (W - 1) * int(case["state"])
    bytes_ = e * (2 * el + 2 * st) + 4 * D * (W + 1)
    if train:
        bytes_ += e * (3 * el + 3 * st) + 8 * D * (W + 1)
    return {"bytes": bytes_, "flops": el * (2 * W + 4) + (el * (6 * W + 8) if train else 0)}
