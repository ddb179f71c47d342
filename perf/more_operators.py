"""Operators of blocks whose recurrence has heads, and of linears in 8-bit floating point: the cases that they are timed on.

``family`` "heads"  linear attention with a decay for each head, the token mixer between in_proj and out_proj of blocks with heads:
                    ``head_scan`` over a batch of token sequences (prompts), ``head_scan_backward`` (training), ``head_scan_step``
                    (one token per sequence).  ``mode`` "infer", "train" (forward and backward pass), "step"
           "fp8"    the linears around it in e4m3 with a scale for each block of 128: ``fp8_quantize`` of activations (1 x 128),
                    ``fp8_matmul`` of two quantized matrices (weights: 128 x 128), ``fp8_linear``, which does both.
                    ``mode`` "quantize", "product", "linear"

Where ``own`` is false, ``run`` computes the same in plain torch operations.
"""
import math

import torch

own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"fp16": 2, "bf16": 2, "fp32": 4}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
BLOCK = 128                            # values that share a scale
LEAST = 2.0 ** -100                    # a block's largest magnitude counts as this at least


def _heads(mode, dtype, B, L, H, P, N, G=1, skip=True, state=False, ragged=False, reverse=False, fixed=False):
    return {"family": "heads", "mode": mode, "dtype": dtype, "B": B, "L": L, "H": H, "P": P, "N": N, "G": G, "skip": skip, "state": state,
            "ragged": ragged, "reverse": reverse, "fixed": fixed}


def _fp8(mode, dtype, M, K, N=0, bias=False):
    return {"family": "fp8", "mode": mode, "dtype": dtype, "M": M, "K": K, "N": N, "bias": bias}


def listed():
    return [
        # one image through one block of the smallest backbone: latency
        dict(_heads("infer", "fp16", 1, 197, 6, 64, 64), name="heads, 1 image"),
        # a batch through one block of the middle backbone, the direction that runs from the last token to the first
        dict(_heads("infer", "fp16", 128, 197, 12, 64, 128, reverse=True), name="heads, batch 128"),
        # few long sequences, read in pieces: states come in and go out
        dict(_heads("infer", "bf16", 2, 20011, 16, 64, 128, state=True), name="heads, 2 long sequences"),
        # fine-tuning one block of the middle backbone
        dict(_heads("train", "fp16", 64, 197, 12, 64, 64), name="heads training, batch 64"),
        # fine-tuning on sequences of different lengths padded to one, two groups of heads, nothing a multiple of anything
        dict(_heads("train", "bf16", 6, 2050, 10, 50, 24, G=2, state=True, ragged=True), name="heads training, ragged"),
        # a hierarchical backbone's second stage in binary32
        dict(_heads("train", "fp32", 8, 784, 6, 64, 16), name="heads training, fp32"),
        # one token of one sequence: latency
        dict(_heads("step", "fp16", 1, 1, 24, 64, 128, state=True), name="heads step, 1 sequence"),
        # one token of each of many sequences served together
        dict(_heads("step", "bf16", 256, 1, 24, 64, 128, state=True), name="heads step, 256 sequences"),
        # out_proj of the middle backbone for one token of one sequence: latency
        dict(_fp8("linear", "fp16", 1, 768, 384), name="fp8 linear, 1 token"),
        # a ragged layer for one image's tokens
        dict(_fp8("linear", "bf16", 197, 1000, 1111, bias=True), name="fp8 linear, 1 image"),
        # activations of the largest backbone at batch 256, quantized once for the linears that read them
        dict(_fp8("quantize", "bf16", 256 * 197, 768), name="fp8 quantize, batch 256"),
        # a large layer, its activations quantized already
        dict(_fp8("product", "bf16", 8192, 4096, 8192), name="fp8 product, 8192 rows"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, direction and type, sizes over the whole range, odd ones among them."""
    while True:
        dtype = rng.choice(["fp16", "bf16", "bf16", "fp32"])
        if rng.random() < 0.6:
            mode = rng.choices(["infer", "train", "step"], [2, 2, 1])[0]
            L = 1 if mode == "step" else rng.choice([49, 196, 197, 784, _log(rng, 1, 16384)])
            H = rng.choice([6, 12, 24, _log(rng, 1, 48)])
            P, N = rng.choice([64, 64, 32, 128, rng.randint(1, 128)]), rng.choice([64, 128, 16, rng.randint(1, 128)])
            G = rng.choice([g for g in (1, 1, 1, 2, 4, H) if H % g == 0])
            fixed = mode != "step" and rng.random() < 0.2
            c = _heads(mode, dtype, _log(rng, 1, 256), L, H, P, N, G, skip=rng.random() < 0.8, state=mode == "step" or rng.random() < 0.4,
                       ragged=mode != "step" and rng.random() < 0.3, reverse=mode != "step" and rng.random() < 0.4, fixed=fixed)
            if c["B"] * max(L, 64) * H * P * N > {"infer": 2.5e9, "train": 6e8, "step": 1.3e9 * 64}[mode] or c["B"] * H * P * N > 1e8:
                continue
        else:
            mode = rng.choice(["quantize", "product", "linear"])
            M, K = _log(rng, 1, 50432), rng.choice([192, 384, 768, 1536, _log(rng, 1, 8192)])
            N = 0 if mode == "quantize" else rng.choice([192, 384, 768, 1536, _log(rng, 1, 8192)])
            if mode == "linear" and dtype == "fp32":
                dtype = "bf16"
            c = _fp8(mode, dtype, M, K, N, bias=mode != "quantize" and rng.random() < 0.4)
            if M * K > 8e7 or M * N > 7e7 or M * K * N > 2.8e11:
                continue
        return c


# ---------------------------------------------------------------------------------------------------------- inputs
def _normal(gen, shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _uniform(gen, shape, lo, hi):
    return torch.rand(shape, generator=gen, device="cuda") * (hi - lo) + lo


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    T = TYPES[case["dtype"]]
    s = {"case": case}
    if case["family"] == "heads":
        B, L, H, P, N, G = (case[k] for k in "BLHPNG")
        # the convolved columns of in_proj's output: u, B and C next to each other; delta in columns of its own
        xbc = _normal(gen, (B, L, H * P + 2 * G * N), T)
        s["u"] = xbc[..., :H * P].unflatten(-1, (H, P))
        s["B"] = xbc[..., H * P:H * P + G * N].unflatten(-1, (G, N))
        s["C"] = xbc[..., H * P + G * N:].unflatten(-1, (G, N))
        # decays from slow to fast, dt around 0.001 .. 0.1, as such blocks are initialised and stay; or one fixed decay per head
        dt = torch.exp(_uniform(gen, (H,), math.log(1e-3), math.log(0.1)))
        s["delta"] = None if case["fixed"] else _normal(gen, (B, L, H), T, 0.5)
        s["delta_bias"] = None if case["fixed"] else dt + torch.log(-torch.expm1(-dt))
        s["A"] = -dt if case["fixed"] else -_uniform(gen, (H,), 1.0, 16.0)
        s["D"] = _normal(gen, (H,)) if case["skip"] else None
        s["state"] = _normal(gen, (B, H, P, N)) if case["state"] else None
        s["final"] = torch.empty(B, H, P, N, device="cuda") if case["state"] else None
        s["lengths"] = None
        if case["ragged"]:                             # one full sequence, one of a single token and, from three on, an empty one
            n = torch.randint(1, L + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
            n[:3] = torch.tensor([L, 1, 0], device="cuda")[:B]
            s["lengths"] = n
        if case["mode"] == "train":
            s["dy"] = _normal(gen, (B, L, H, P), T)
            s["dfinal"] = _normal(gen, (B, H, P, N)) if case["state"] else None
        if case["mode"] == "step":
            for k in ("u", "delta", "B", "C"):
                s[k] = s[k][:, 0]
    else:
        M, K, N = case["M"], case["K"], case["N"]
        # channels of different size, as activations have
        s["x"] = (torch.randn(M, K, generator=gen, device="cuda") * torch.exp(_normal(gen, (K,)))).to(T)
        if case["mode"] == "product":
            s["a"], s["a_scales"] = _plain_quantize(s.pop("x"))
        if N:
            s["w"], s["w_scales"] = _weights(_normal(gen, (N, K), scale=1.0 / math.sqrt(K)))
        s["bias"] = _normal(gen, (N,)) if case["bias"] else None
    return s


def _weights(w):
    """A layer's weights as its checkpoint holds them: e4m3 codes [N,K], a scale for each 128 x 128 block."""
    N, K = w.shape
    pad = torch.nn.functional.pad(w, (0, -K % BLOCK, 0, -N % BLOCK))
    tiles = pad.unflatten(1, (-1, BLOCK)).unflatten(0, (-1, BLOCK))
    scales = tiles.abs().amax((1, 3)).clamp(min=LEAST) / E4M3_MAX
    codes = (tiles / scales[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).flatten(2).flatten(0, 1)[:N, :K].to(E4M3)
    rows = torch.zeros(N, K + (-K % 16), device=w.device, dtype=torch.uint8).view(E4M3)
    rows.view(torch.uint8)[:, :K] = codes.view(torch.uint8)
    return rows[:, :K], scales


# ---------------------------------------------------------------------------------------------------------- one pass
def run(state):
    if state["case"]["family"] == "heads":
        return _own_heads(state) if own else _plain_heads(state)
    return _own_fp8(state) if own else _plain_fp8(state)


def _own_heads(s):
    import paper_2412_20386_b200 as ptq
    c = s["case"]
    args = (s["u"], s["delta"], s["A"], s["B"], s["C"])
    if c["mode"] == "step":
        y = ptq.head_scan_step(s["state"], *args, D=s["D"], delta_bias=s["delta_bias"], new_state=s["final"])
        return {"y": y, "final": s["final"]}
    kw = dict(D=s["D"], delta_bias=s["delta_bias"], state=s["state"], lengths=s["lengths"], reverse=c["reverse"])
    if c["mode"] == "infer":
        y = ptq.head_scan(*args, **kw, final_state=s["final"])
        return {"y": y, "final": s["final"]}
    history = ptq.head_scan_history(s["u"], c["N"])
    y = ptq.head_scan(*args, **kw, final_state=s["final"], history=history)
    g = ptq.head_scan_backward(s["dy"], *args, history, **kw, dfinal=s["dfinal"])
    return {"y": y, "final": s["final"], **{"d" + k: v for k, v in g.items()}}


def _own_fp8(s):
    import paper_2412_20386_b200 as ptq
    c = s["case"]
    if c["mode"] == "quantize":
        codes, scales = ptq.fp8_quantize(s["x"])
        return {"codes": codes, "scales": scales}
    if c["mode"] == "product":
        return {"y": ptq.fp8_matmul(s["a"], s["a_scales"], s["w"], s["w_scales"], s["bias"], dtype=TYPES[c["dtype"]])}
    return {"y": ptq.fp8_linear(s["x"], s["w"], s["w_scales"], s["bias"])}


# ---------------------------------------------------------------------------------------------------------- plain forms
def _order(s, B, L):
    """(positions in the order of processing [B,L], which of them hold a token [B,L])"""
    i = torch.arange(L, device="cuda").expand(B, L)
    n = torch.full((B, 1), L, device="cuda") if s["lengths"] is None else s["lengths"].long()[:, None]
    valid = i < n
    return (torch.where(valid, n - 1 - i, i) if s["case"]["reverse"] else i), valid


def _take(t, pos, valid):
    """Rows of t [B,L,...] in the order of processing, in 32 bits, zeros where there is no token."""
    more = (1,) * (t.dim() - 2)
    return torch.where(valid.reshape(valid.shape + more), t.gather(1, pos.reshape(pos.shape + more).expand(t.shape)).float(), 0.0)


def _put_back(t, pos, valid, dtype):
    """The inverse of _take, rounded."""
    more = (1,) * (t.dim() - 2)
    t = torch.where(valid.reshape(valid.shape + more), t, 0.0).to(dtype)
    return torch.zeros(t.shape, dtype=dtype, device="cuda").scatter_(1, pos.reshape(pos.shape + more).expand(t.shape), t)


def _pieces(t, Q):
    """[B,L,H,...] -> [B,H,pieces,Q,...], zeros behind the end."""
    t = torch.nn.functional.pad(t, (0, 0) * (t.dim() - 2) + (0, -t.shape[1] % Q))
    return t.unflatten(1, (-1, Q)).movedim(3, 1)


def _whole(t, L):
    """The inverse of _pieces."""
    return t.movedim(1, 3).flatten(1, 2)[:, :L]


def _between(c):
    """exp(c_i - c_j) for j <= i, else 0, along the last dimension of running sums c in 64 bits."""
    n = c.shape[-1]
    keep = torch.ones(n, n, dtype=torch.bool, device=c.device).tril()
    return torch.exp(torch.where(keep, c[..., :, None] - c[..., None, :], -math.inf)).float()


def _plain_heads(s):
    """In pieces of Q steps: within a piece all pairs of steps, from piece to piece the states."""
    c = s["case"]
    T = TYPES[c["dtype"]]
    step = c["mode"] == "step"
    tok = {k: None if s[k] is None else (s[k][:, None] if step else s[k]) for k in ("u", "delta", "B", "C")}
    B, L, H, P = tok["u"].shape
    N, G = c["N"], c["G"]
    Q = min(64, L)
    pos, valid = _order(s, B, L)
    per = lambda t: t.repeat_interleave(H // G, 2)                                   # [B,L,G,N] -> [B,L,H,N]
    u = _pieces(_take(tok["u"], pos, valid), Q)                                      # [B,H,p,Q,P]
    Bm, Cm = (_pieces(per(_take(tok[k], pos, valid)), Q) for k in ("B", "C"))        # [B,H,p,Q,N]
    if c["fixed"]:
        e, dt = None, valid[..., None].float().expand(B, L, H)
    else:
        e = _take(tok["delta"], pos, valid) + s["delta_bias"]
        dt = torch.where(valid[..., None], torch.where(e > 20, e, torch.log1p(torch.exp(e))), 0.0)
    dt = _pieces(dt, Q)                                                              # [B,H,p,Q]
    A = s["A"][:, None, None]
    run_sum = (dt.double() * A[None]).cumsum(-1)
    M = _between(run_sum)                                                            # [B,H,p,Q,Q]
    into, left = torch.exp(run_sum).float(), torch.exp(run_sum[..., -1:] - run_sum).float()
    ud = dt[..., None] * u
    scores = Cm @ Bm.mT
    # states in front of each piece: its own and all earlier pieces' inputs, decayed
    inputs = (left[..., None] * ud).mT @ Bm                                          # [B,H,p,P,N]
    h0 = torch.zeros(B, H, P, N, device="cuda") if s["state"] is None else s["state"]
    total = torch.nn.functional.pad(run_sum[..., -1].cumsum(-1), (1, 0))
    far = _between(total)                                                            # [B,H,p+1,p+1]
    states = (far @ torch.cat([h0[:, :, None], inputs], 2).flatten(3)).unflatten(3, (P, N))
    y = (scores * M) @ ud + into[..., None] * (Cm @ states[:, :, :-1].mT)
    if s["D"] is not None:
        y = y + s["D"][:, None, None, None] * u
    out = {"y": _put_back(_whole(y, L), pos, valid, T), "final": None if s["final"] is None else states[:, :, -1].clone()}
    if step:
        out["y"] = out["y"][:, 0]
    if c["mode"] != "train":
        return out
    dy = _pieces(_take(s["dy"], pos, valid), Q)
    last = torch.zeros(B, H, P, N, device="cuda") if s["dfinal"] is None else s["dfinal"]
    # gradients of the states behind each piece
    outputs = (into[..., None] * dy).mT @ Cm                                         # [B,H,p,P,N]
    g = (far.mT @ torch.cat([outputs, last[:, :, None]], 2).flatten(3)).unflatten(3, (P, N))
    after, before = g[:, :, 1:], states[:, :, :-1]
    R = dy @ ud.mT
    pairs = scores * M * R                                                           # what each pair of steps adds to the result
    dud = (scores * M).mT @ dy + left[..., None] * (Bm @ after.mT)
    dB = (R * M).mT @ Cm + left[..., None] * (ud @ after)
    dC = (R * M) @ Bm + into[..., None] * (dy @ before)
    du = dt[..., None] * dud
    if s["D"] is not None:
        du = du + s["D"][:, None, None, None] * dy
    # a step's log decay has a part in all that passes it: pairs from before it to it or after, states into and out of the piece
    come = into * (dy * (Cm @ before.mT)).sum(-1)
    go = left * (ud * (Bm @ after.mT)).sum(-1)
    through = (torch.exp(run_sum[..., -1]).float() * (after * before).sum((-1, -2)))[..., None]
    dsum = pairs.double().sum(-1) - pairs.double().sum(-2) + come - go
    dlog = (dsum.flip(-1).cumsum(-1).flip(-1) + go.double().sum(-1, keepdim=True) + through).float()
    add = lambda t: t.unflatten(2, (G, H // G)).sum(3)
    out["du"] = _put_back(_whole(du, L), pos, valid, T)
    out["dB"], out["dC"] = (_put_back(add(_whole(t, L)), pos, valid, T) for t in (dB, dC))
    out["dA"] = (dt * dlog).double().sum((0, 2, 3)).float()
    out["dD"] = None if s["D"] is None else (u * dy).double().sum((0, 2, 3, 4)).float()
    out["dstate"] = None if s["state"] is None else g[:, :, 0].clone()
    out["ddelta"] = out["ddelta_bias"] = None
    if not c["fixed"]:
        ddelta = _whole(A[None] * dlog + (u * dud).sum(-1), L) * torch.sigmoid(e)
        ddelta = torch.where(valid[..., None], ddelta, 0.0)
        out["ddelta"], out["ddelta_bias"] = _put_back(ddelta, pos, valid, T), ddelta.double().sum((0, 1)).float()
    return out


def _plain_quantize(x):
    """e4m3 codes [M,K] and scales [M,ceil(K/128)]: the largest magnitude of a block becomes the largest code."""
    M, K = x.shape
    blocks = torch.nn.functional.pad(x.float(), (0, -K % BLOCK)).unflatten(1, (-1, BLOCK))
    top = blocks.abs().amax(2).clamp(min=LEAST)
    codes = (blocks * (E4M3_MAX / top)[..., None]).clamp(-E4M3_MAX, E4M3_MAX).flatten(1).to(E4M3)
    rows = torch.nn.functional.pad(codes.view(torch.uint8)[:, :K], (0, -K % 16)).view(E4M3)
    return rows[:, :K], (top / E4M3_MAX).t().contiguous().t()


def _plain_product(a, a_scales, w, w_scales, bias, dtype):
    K, N = a.shape[1], w.shape[0]
    a = a.float() * a_scales.repeat_interleave(BLOCK, 1)[:, :K]
    w = w.float() * w_scales.repeat_interleave(BLOCK, 1)[:, :K].repeat_interleave(BLOCK, 0)[:N]
    y = a @ w.t()
    return (y if bias is None else y + bias).to(dtype)


def _plain_fp8(s):
    c = s["case"]
    if c["mode"] == "quantize":
        codes, scales = _plain_quantize(s["x"])
        return {"codes": codes, "scales": scales}
    a = (s["a"], s["a_scales"]) if c["mode"] == "product" else _plain_quantize(s["x"])
    return {"y": _plain_product(*a, s["w"], s["w_scales"], s["bias"], TYPES[c["dtype"]])}


# ---------------------------------------------------------------------------------------------------------- exact values
def exact(case, seed):
    """The definitions in 64 bits: the recurrence token by token, the product of what the codes stand for."""
    s = prepare(case, seed)
    d = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    return _exact_heads(case, d) if case["family"] == "heads" else _exact_fp8(case, d)


def _exact_heads(case, s):
    B, L, H, P, N, G, step = (*(case[k] for k in "BLHPNG"), case["mode"] == "step")
    if step:
        s = {**s, **{k: None if s[k] is None else s[k][:, None] for k in ("u", "delta", "B", "C")}}
    f64 = dict(dtype=torch.float64, device="cuda")
    rows, group = torch.arange(B, device="cuda"), torch.arange(H, device="cuda") // (H // G)
    n = torch.full((B,), L, device="cuda") if s["lengths"] is None else s["lengths"].long()
    train = case["mode"] == "train"
    zero = torch.zeros((), **f64)

    def at(i):
        on = i < n
        return torch.where(on, n - 1 - i, 0) if case["reverse"] else torch.full_like(n, i), on

    def put(t, p, on, v):
        t.index_put_((rows, p), torch.where(on.reshape((-1,) + (1,) * (v.dim() - 1)), v, t[rows, p]))

    def token(p):
        e = None if s["delta"] is None else s["delta"][rows, p] + s["delta_bias"]
        dt = torch.ones(B, H, **f64) if e is None else torch.clamp(e, min=0.0) + torch.log1p(torch.exp(-e.abs()))
        return e, dt, torch.exp(dt * s["A"]), s["u"][rows, p], s["B"][rows, p][:, group], s["C"][rows, p][:, group]

    h = torch.zeros(B, H, P, N, **f64) if s["state"] is None else s["state"]
    y, kept = torch.zeros(B, L, H, P, **f64), []
    for i in range(L):
        p, on = at(i)
        _, dt, a, u, Bt, Ct = token(p)
        if train:
            kept.append(h)
        new = a[..., None, None] * h + (dt[..., None] * u)[..., None] * Bt[:, :, None]
        h = torch.where(on[:, None, None, None], new, h)
        o = (h @ Ct[..., None])[..., 0]
        put(y, p, on, o if s["D"] is None else o + s["D"][:, None] * u)
    out = {"y": y[:, 0] if step else y, "final": None if s["final"] is None else h}
    if not train:
        return out
    du, dd = torch.zeros(B, L, H, P, **f64), torch.zeros(B, L, H, **f64)
    dB, dC = torch.zeros(B, L, G, N, **f64), torch.zeros(B, L, G, N, **f64)
    dA, dD, db = torch.zeros(H, **f64), torch.zeros(H, **f64), torch.zeros(H, **f64)
    gh = torch.zeros_like(h) if s["dfinal"] is None else s["dfinal"]
    for i in reversed(range(L)):
        p, on = at(i)
        e, dt, a, u, Bt, Ct = token(p)
        before = kept.pop()
        dy = torch.where(on[:, None, None], s["dy"][rows, p], zero)
        now = a[..., None, None] * before + (dt[..., None] * u)[..., None] * Bt[:, :, None]
        g = gh + dy[..., None] * Ct[:, :, None]
        g = torch.where(on[:, None, None, None], g, zero)
        gb = (g @ Bt[..., None])[..., 0]                                             # [B,H,P]
        q = a * (g * before).sum((-1, -2))                                           # gradient of the log decay
        put(du, p, on, dt[..., None] * gb + (0.0 if s["D"] is None else s["D"][:, None] * dy))
        put(dB, p, on, torch.einsum("bhpn,bhp->bhn", g, dt[..., None] * u).unflatten(1, (G, -1)).sum(2))
        put(dC, p, on, torch.einsum("bhpn,bhp->bhn", now, dy).unflatten(1, (G, -1)).sum(2))
        dA += (dt * q).sum(0)
        dD += (dy * u).sum((0, 2))
        if e is not None:
            de = (s["A"] * q + (gb * u).sum(-1)) / (1 + torch.exp(-e))
            put(dd, p, on, de)
            db += torch.where(on[:, None], de, zero).sum(0)
        gh = torch.where(on[:, None, None, None], a[..., None, None] * g, gh)
    fixed = s["delta"] is None
    out.update(du=du, ddelta=None if fixed else dd, dA=dA, dB=dB, dC=dC, dD=None if s["D"] is None else dD, ddelta_bias=None if fixed else db,
               dstate=None if s["state"] is None else gh)
    return out


def _exact_fp8(case, s):
    quantized = case["mode"] == "product"
    if quantized:
        a, sa = s["a"], s["a_scales"]
    else:
        M, K = s["x"].shape
        kb = -(-K // BLOCK)
        block = torch.arange(K, device="cuda") // BLOCK
        sa = torch.zeros(M, kb, dtype=torch.float64, device="cuda").index_reduce_(1, block, s["x"].abs(), "amax").clamp(min=LEAST) / E4M3_MAX
        a = s["x"] / sa[:, block]
        # to the nearest multiple of 2^-3 of its power of two, 2^-9 at least
        grid = torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=2.0 ** -6))) - 3)
        a = (torch.round(a / grid) * grid).clamp(-E4M3_MAX, E4M3_MAX)
    if case["mode"] == "quantize":
        return {"codes": a, "scales": sa}
    k, n = torch.arange(a.shape[1], device="cuda") // BLOCK, torch.arange(s["w"].shape[0], device="cuda") // BLOCK
    y = (a * sa[:, k]) @ (s["w"] * s["w_scales"][n][:, k]).t()
    return {"y": y if s["bias"] is None else y + s["bias"]}


# ---------------------------------------------------------------------------------------------------------- work
def work(case):
    e, train = BYTES[case["dtype"]], case["mode"] == "train"
    if case["family"] == "heads":
        B, L, H, P, N, G = (case[k] for k in "BLHPNG")
        el, bc, dl, st = B * L * H * P, 2 * B * L * G * N, B * L * H * int(not case["fixed"]), B * H * P * N * int(case["state"])
        bytes_ = e * (2 * el + bc + dl) + 4 * (2 * st + 3 * H)
        flops = el * N * 5 + el * 2                        # decay, input and output of the recurrence
        if train:                                          # the backward pass reads the same again, and dy
            bytes_ += e * (3 * el + 2 * bc + 2 * dl) + 4 * (3 * st + 6 * H)
            flops += el * N * 12 + el * 4
        return {"bytes": bytes_, "flops": flops}
    M, K, N = case["M"], case["K"], case["N"]
    kb = -(-K // BLOCK)
    if case["mode"] == "quantize":
        return {"bytes": M * K * (e + 1) + 4 * M * kb, "flops": 4 * M * K}
    weights = N * K + 4 * kb * -(-N // BLOCK) + 4 * N * int(case["bias"])
    inputs = M * K + 4 * M * kb if case["mode"] == "product" else M * K * e
    return {"bytes": inputs + weights + M * N * e, "flops": 2 * M * N * K}
