"""gated_scan, gated_scan_backward and gated_scan_step against the recurrence in 64 bits."""
import math
import random

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


def make(seed, dtype, B, L, D, N, G=None, gate=True, skip=True, bias=True, state=False, lengths=None, odd=False, ungrouped=False):
    """Inputs as a block has them: u and z the halves of one tensor, B and C the columns of another; `odd` shifts every row by one element."""
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    G = G or 1
    pad = 1 if odd else 0
    xz, dl = r(B, L, 2 * D + pad).to(dtype).cuda(), r(B, L, D + pad).to(dtype).cuda() * 0.5
    bc = r(B, L, 2 * G * N + 4 + pad).to(dtype).cuda()
    t = {"u": xz[..., pad:D + pad], "delta": dl[..., pad:], "z": xz[..., D + pad:] if gate else None,
         "A": (-torch.arange(1, N + 1) * torch.exp(0.3 * r(D, N))).cuda(),
         "B": bc[..., pad:G * N + pad].unflatten(-1, (G, N)), "C": bc[..., 4 + pad + G * N:].unflatten(-1, (G, N)),
         "D": r(D).cuda() if skip else None, "delta_bias": (r(D) - 3.0).cuda() if bias else None,
         "state": r(B, D, N).cuda() if state else None}
    if ungrouped:
        t["B"], t["C"] = t["B"][:, :, 0], t["C"][:, :, 0]
    t["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    if lengths is not None:                                  # what lies behind the ends is not read
        for b, n in enumerate(lengths):
            for k in ("u", "delta", "z", "B", "C"):
                if t[k] is not None:
                    t[k][b, max(n, 0):] = float("nan")
    return t


FLOATS = ("u", "delta", "A", "B", "C", "D", "z", "delta_bias", "state")


def call(ptq, t, reverse=False, softplus=True, **kw):
    return ptq.gated_scan(t["u"], t["delta"], t["A"], t["B"], t["C"], D=t["D"], z=t["z"], delta_bias=t["delta_bias"], state=t["state"],
                          lengths=t["lengths"], reverse=reverse, softplus=softplus, **kw)


def reference(t, reverse, softplus, dy=None, dfinal=None, absolute=False):
    """y, final state and (with dy) gradients; `absolute`: the scale of the tolerances, everything but A positive and no cancellation."""
    x = ref.leaves({k: t[k] for k in FLOATS})
    pick = {k: x.get(k) for k in FLOATS}
    if absolute:
        # dt, decays and gates as they are; u, B, C, D, state and cotangents by magnitude
        pick = {k: v if v is None or k in ("A", "delta", "delta_bias", "z") else v.abs() for k, v in pick.items()}
    y, final = ref.scan(*(pick[k] for k in ("u", "delta", "A", "B", "C")), D=pick["D"], z=None if absolute else pick["z"],
                        delta_bias=pick["delta_bias"], state=pick["state"], lengths=t["lengths"], softplus=softplus, reverse=reverse)
    if dy is None:
        return y, final, None
    return y, final, ref.gradients((y, final), (dy, dfinal), x)


def scales(t, reverse, softplus, dy, dfinal, z):
    """Per output the bound that the factor multiplies: every sum by magnitude, which for the gradients is written out here."""
    x = {k: None if t[k] is None else torch.nan_to_num(t[k].double().cpu(), 0.0).abs() for k in FLOATS}
    x["A"], x["delta"], x["delta_bias"] = -x["A"], torch.nan_to_num(t["delta"].double().cpu()), None if t["delta_bias"] is None else t["delta_bias"].double().cpu()
    B, L, D = x["u"].shape
    Bm, Cm = (v[:, :, None] if v.dim() == 3 else v for v in (x["B"], x["C"]))
    G = Bm.shape[2]
    heads = torch.arange(D) // (D // G)
    dy = dy.double().cpu().abs()
    gate = 1.0 if z is None else (z * torch.sigmoid(z)).abs()
    out = {k: torch.zeros_like(v) for k, v in (("u", x["u"]), ("delta", x["u"]), ("z", x["u"]), ("A", x["A"]), ("B", Bm), ("C", Cm))}
    out["D"], out["delta_bias"] = torch.zeros(D, dtype=torch.float64), torch.zeros(D, dtype=torch.float64)
    out["state"] = torch.zeros(B, D, x["A"].shape[1], dtype=torch.float64)
    for b, order in enumerate(ref.positions(B, L, t["lengths"], reverse)):
        h = torch.zeros(D, x["A"].shape[1], dtype=torch.float64) if x["state"] is None else x["state"][b]
        kept = []
        for p in order:
            e = x["delta"][b, p] + (0.0 if x["delta_bias"] is None else x["delta_bias"])
            dt = torch.nn.functional.softplus(e, threshold=1e9) if softplus else e.abs()
            a = torch.exp((dt if softplus else e)[:, None] * t["A"].double().cpu())
            kept.append((p, dt, a, h))
            h = a * h + (dt * x["u"][b, p])[:, None] * Bm[b, p][heads]
            kept[-1] += (h,)
        e_g = torch.zeros_like(h) if dfinal is None else dfinal[b].double().cpu().abs()
        for p, dt, a, before, now in reversed(kept):
            do = dy[b, p] * (gate if z is None else gate[b, p])
            g = e_g + do[:, None] * Cm[b, p][heads]
            q = g * a * before
            gb = (g * Bm[b, p][heads]).sum(-1)
            skip = 0.0 if x["D"] is None else x["D"]
            dd = x["u"][b, p] * gb + (q * -x["A"]).sum(-1)
            out["u"][b, p] = dt * gb + skip * do
            out["delta"][b, p] = dd
            out["z"][b, p] = 1.2 * dy[b, p] * ((now * Cm[b, p][heads]).sum(-1) + skip * x["u"][b, p])
            out["A"] += q * dt[:, None]
            out["B"][b, p] = torch.zeros_like(Bm[b, p]).index_add_(0, heads, g * (dt * x["u"][b, p])[:, None])
            out["C"][b, p] = torch.zeros_like(Cm[b, p]).index_add_(0, heads, now * do[:, None])
            out["D"] += x["u"][b, p] * do
            out["delta_bias"] += dd
            e_g = g * a
        out["state"][b] = e_g
    if t["B"].dim() == 3:
        out["B"], out["C"] = out["B"][:, :, 0], out["C"][:, :, 0]
    return out


def check(ptq, t, reverse=False, softplus=True, train=True, dfinal=True, seed=7):
    u = t["u"]
    B, L, D = u.shape
    N = t["A"].shape[1]
    x64 = {k: None if t[k] is None else torch.nan_to_num(t[k].double().cpu(), 0.0) for k in FLOATS}
    factor = ref.scan_factor(x64["u"], x64["delta"], x64["A"], x64["delta_bias"], softplus, t["lengths"], reverse)
    final = torch.full((B, D, N), 7.0, device="cuda")
    history = ptq.scan_history(u, N) if train else None
    y = call(ptq, t, reverse, softplus, final_state=final, history=history)
    gen = torch.Generator().manual_seed(seed)
    dy = torch.randn(B, L, D, generator=gen).to(u.dtype).cuda() if train else None
    df = torch.randn(B, D, N, generator=gen).cuda() if train and dfinal else None
    y64, final64, g64 = reference(t, reverse, softplus, dy, df)
    y_abs, final_abs, _ = reference(t, reverse, softplus, absolute=True)
    gate = 1.0 if t["z"] is None else (x64["z"] * torch.sigmoid(x64["z"])).abs()
    ref.close(y, y64, y_abs * gate, factor, "y")
    ref.close(final, final64, final_abs, factor, "final state")
    if not train:
        return
    got = ptq.gated_scan_backward(dy, u, t["delta"], t["A"], t["B"], t["C"], history, D=t["D"], z=t["z"], delta_bias=t["delta_bias"], state=t["state"],
                                  lengths=t["lengths"], softplus=softplus, reverse=reverse, dfinal=df)
    bound = scales(t, reverse, softplus, dy, df, x64["z"])
    for k in FLOATS:
        if t[k] is None:
            assert got[k] is None
            continue
        assert got[k].dtype == t[k].dtype
        ref.close(got[k], g64[k], bound[k], factor, "gradient of " + k)


@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 8, 11, 16, 17, 24, 32])
@pytest.mark.parametrize("dtype", [ref.F32, ref.F16, ref.BF16], ids=["f32", "f16", "bf16"])
def test_states(ptq, N, dtype):
    """Every split of the states over lanes, each type, both directions."""
    check(ptq, make(N, dtype, 2, 37, 24, N, state=True), reverse=N % 2 == 0)


@pytest.mark.parametrize("L", [1, 2, 7, 8, 9, 31, 32, 33, 64, 65, 96, 130])
def test_lengths_at_tile_and_stretch_ends(ptq, L):
    check(ptq, make(L, ref.F32, 1, L, 40, 16, state=L % 2 == 0), reverse=L % 3 == 0)
    check(ptq, make(L, ref.BF16, 2, L, 9, 6, skip=False), reverse=L % 3 == 1)


@pytest.mark.parametrize("D,G", [(1, 1), (3, 3), (8, 1), (15, 1), (16, 2), (33, 1), (66, 2), (130, 1), (200, 4), (12, 6)])
@pytest.mark.parametrize("odd", [False, True])
def test_channels_groups_and_row_alignment(ptq, D, G, odd):
    """Groups that end inside a warp's channels; rows at any address."""
    check(ptq, make(D, ref.F16, 2, 21, D, 16, G=G, odd=odd, gate=D % 2 == 0))
    check(ptq, make(D, ref.F32, 1, 40, D, 4, G=G, odd=odd, state=True), reverse=True)


@pytest.mark.parametrize("lengths", [[0, 0, 0], [1, 0, 33], [50, 17, 8], [49, 200, -3], [7, 50, 16]])
@pytest.mark.parametrize("reverse", [False, True])
def test_padded_batches(ptq, lengths, reverse):
    """Empty sequences, ends inside tiles, lengths out of range; NaN behind the ends stays there, gradients there are zeros."""
    for N, dtype, state in ((16, ref.F32, True), (3, ref.BF16, False)):
        t = make(sum(map(abs, lengths)), dtype, 3, 50, 20, N, G=2, state=state, lengths=lengths)
        check(ptq, t, reverse=reverse)
        y = torch.full((3, 50, 20), 3.0, dtype=dtype, device="cuda")
        assert call(ptq, t, reverse, y=y) is y
        for b, n in enumerate(lengths):
            assert (y[b, max(n, 0):] == 3.0).all()           # left as they were


@pytest.mark.parametrize("flags", [dict(gate=False), dict(skip=False), dict(bias=False), dict(gate=False, skip=False, bias=False), dict(state=True)])
def test_optional_inputs(ptq, flags):
    check(ptq, make(3, ref.F32, 2, 20, 17, 16, **flags))
    check(ptq, make(4, ref.F32, 1, 20, 17, 16, ungrouped=True, **flags), dfinal=False)


def test_without_softplus(ptq):
    t = make(5, ref.F32, 2, 30, 24, 8, bias=False, state=True)
    t["delta"] = t["delta"].abs() * 0.2
    check(ptq, t, softplus=False)


@pytest.mark.parametrize("B,L,D,N", [(1, 700, 16, 16), (2, 413, 24, 4), (1, 1100, 8, 1), (1, 300, 8, 32)])
def test_few_rows_are_cut_into_chunks(ptq, B, L, D, N):
    """Few channels: the sequence is cut, with and without padding, and the final state may replace the first one."""
    from paper_2412_20386_b200 import binding
    from parity_util import launches
    t = make(L, ref.F32, B, L, D, N, state=True)
    assert launches(ptq, lambda: call(ptq, t)) == 2
    check(ptq, t, reverse=B == 2)
    t = make(L + 1, ref.BF16, B, L, D, N, state=True, lengths=[L - 100] * B)
    check(ptq, t, reverse=B == 1)
    want = torch.empty_like(t["state"])
    y1 = call(ptq, t, final_state=want)
    t["state"] = t["state"].clone()
    y2 = call(ptq, t, final_state=t["state"])
    assert torch.equal(t["state"], want)
    assert torch.equal(torch.nan_to_num(y1.float()), torch.nan_to_num(y2.float()))
    assert binding.kernel_launch_count() > 0


def test_many_rows_take_one_pass(ptq):
    from parity_util import launches
    t = make(1, ref.F16, 160, 33, 384, 16)
    assert launches(ptq, lambda: call(ptq, t)) == 1
    for b in (0, 77, 159):
        one = {k: v[b:b + 1] if torch.is_tensor(v) and v.dim() > 2 else v for k, v in t.items()}
        ref.close(call(ptq, t)[b], call(ptq, one)[0], 1.0, 2.0 ** -10)
    sub = {k: v[:2] if torch.is_tensor(v) and v.dim() > 2 else v for k, v in t.items()}
    check(ptq, sub)


def test_slow_decays_keep_their_precision(ptq):
    """Thousands of steps with decays of 0.999 and more: errors of the power of two add up over the whole memory, so their mean has to
    vanish.  Bound: as everywhere, here with a memory of about a thousand steps."""
    t = make(9, ref.F32, 1, 3000, 8, 2, gate=False)
    t["A"] = -torch.rand(8, 2, device="cuda") * 0.02 - 0.001
    check(ptq, t, train=False)
    history = ptq.scan_history(t["u"], 2)
    y = call(ptq, t, history=history)
    y64, _, _ = reference(t, False, True)
    y64 = y64.detach()
    assert float((y.double().cpu() - y64).norm() / y64.norm()) < 3e-6


def test_large_and_special_values(ptq):
    """dt from underflow to where softplus is the identity; A = -inf forgets, A = 0 keeps; a zero dt keeps the state."""
    t = make(11, ref.F32, 1, 12, 16, 16, gate=True, state=True)
    t["delta"] = torch.linspace(-120, 60, 12 * 16, device="cuda").reshape(1, 12, 16).contiguous()
    t["delta_bias"] = None
    t["A"][:, 0] = 0.0
    y = call(ptq, t, final_state=(final := torch.empty_like(t["state"])))
    y64, final64, _ = reference(t, False, True)
    ya, fa, _ = reference(t, False, True, absolute=True)
    gate = (t["z"].double().cpu() * torch.sigmoid(t["z"].double().cpu())).abs()
    # dt reaches 60 and |A| about 40: the argument's rounding, |dt A| 2^-21, matters only where exp(dt A) is not zero in binary32 (|dt A| < 104)
    ref.close(y, y64, ya * gate, 2.0 ** -20 * (8 + 4 * 12) * 105, "y")
    ref.close(final, final64, fa, 2.0 ** -20 * (8 + 4 * 12) * 105, "final state")
    t["delta"] = torch.zeros_like(t["delta"])
    t["A"] = torch.full_like(t["A"], -math.inf)
    call(ptq, t, softplus=True, final_state=final)
    u, B = t["u"].double().cpu(), t["B"].double().cpu()[:, :, 0]
    ref.close(final, (math.log(2.0) * u[:, -1])[..., None] * B[:, -1][:, None], 1.0, 2.0 ** -20, "only the last input is left")
    t["A"] = -torch.rand_like(t["A"])
    call(ptq, t, softplus=False, final_state=final)
    assert torch.equal(final, t["state"])                    # dt = 0: exactly as it was


def test_infinities_and_nan_stay_in_their_channel(ptq):
    t = make(12, ref.F32, 2, 40, 24, 16)
    clean = call(ptq, t)
    t["u"][0, 5, 3] = float("inf")
    t["delta"][1, 7, 9] = float("nan")
    y = call(ptq, t)
    mask = torch.ones(2, 40, 24, dtype=torch.bool)
    mask[0, 5:, 3] = False
    mask[1, 7:, 9] = False
    assert torch.equal(y.cpu()[mask], clean.cpu()[mask])
    assert not torch.isfinite(y[0, 5, 3]) and torch.isnan(y[1, 7:, 9]).all()
    t = make(13, ref.F32, 1, 9, 16, 16)
    t["A"][4, 2] = float("nan")
    y = call(ptq, t)
    assert torch.isnan(y[0, :, 4]).all() and torch.isfinite(y[0, :, :4]).all() and torch.isfinite(y[0, :, 5:]).all()


@pytest.mark.parametrize("N", [1, 2, 4, 7, 16, 20, 32])
@pytest.mark.parametrize("dtype", [ref.F32, ref.F16, ref.BF16], ids=["f32", "f16", "bf16"])
def test_single_tokens(ptq, N, dtype):
    """The step's own kernel: odd batches and channels, in place and not, and the same as the scan of length 1."""
    for B, D, G in ((1, 8, 1), (5, 33, 1), (9, 70, 2), (131, 16, 1)):
        t = make(N + B, dtype, B, 1, D, N, G=G, state=True, odd=B == 5)
        one = {k: None if t[k] is None else t[k][:, 0] for k in ("u", "delta", "z", "B", "C")}
        args = (one["u"], one["delta"], t["A"], one["B"], one["C"])
        kw = dict(D=t["D"], z=t["z"][:, 0], delta_bias=t["delta_bias"])
        new = torch.empty_like(t["state"])
        y = ptq.gated_scan_step(t["state"], *args, **kw, new_state=new)
        x64 = {k: None if t[k] is None else t[k].double().cpu() for k in FLOATS}
        factor = ref.scan_factor(x64["u"], x64["delta"], x64["A"], x64["delta_bias"], True, None, False)
        y64, f64, _ = reference(t, False, True)
        ya, fa, _ = reference(t, False, True, absolute=True)
        ref.close(y, y64[:, 0], (ya * (x64["z"] * torch.sigmoid(x64["z"])).abs())[:, 0], factor, "y")
        ref.close(new, f64, fa, factor, "state")
        state = t["state"].clone()
        assert torch.equal(ptq.gated_scan_step(state, *args, **kw), y) and torch.equal(state, new)
        lengths = torch.tensor([b % 2 for b in range(B)], dtype=torch.int32, device="cuda")
        t["lengths"], final = lengths, torch.empty_like(state)
        yl = call(ptq, t, final_state=final)
        for b in range(B):
            assert torch.equal(final[b], new[b] if b % 2 else t["state"][b])
            assert torch.equal(yl[b, 0], y[b] if b % 2 else torch.zeros_like(y[b]))


def test_pieces_of_a_sequence_and_tokens_one_by_one(ptq):
    """A sequence in one call, in pieces that hand the state on, and token by token."""
    t = make(21, ref.F32, 2, 90, 24, 16, state=True)
    final = torch.empty_like(t["state"])
    whole = call(ptq, t, final_state=final)
    for cuts in ([1, 50, 90], [64, 89, 90], list(range(1, 91))):
        state, at, parts = t["state"].clone(), 0, []
        for end in cuts:
            piece = {k: v[:, at:end] if k in ("u", "delta", "z", "B", "C") else v for k, v in t.items()}
            piece["state"] = state
            parts.append(call(ptq, piece, final_state=state))
            at = end
        got = torch.cat(parts, 1)
        assert torch.allclose(got, whole, rtol=1e-4, atol=1e-5) and torch.allclose(state, final, rtol=1e-4, atol=1e-5)


def test_gradients_against_differences(ptq):
    """Along a random direction in all inputs the kernels' gradients give the difference quotient of the 64-bit recurrence.  Step 1e-5: the
    quotient's own error is about 1e-10 of third derivatives; the kernels' is what `factor` allows on the sum of magnitudes."""
    t = make(31, ref.F32, 2, 25, 12, 8, G=2, state=True)
    history = ptq.scan_history(t["u"], 8)
    call(ptq, t, history=history)
    gen = torch.Generator().manual_seed(1)
    dy, df = torch.randn(2, 25, 12, generator=gen).cuda(), torch.randn(2, 12, 8, generator=gen).cuda()
    g = ptq.gated_scan_backward(dy, t["u"], t["delta"], t["A"], t["B"], t["C"], history, D=t["D"], z=t["z"], delta_bias=t["delta_bias"], state=t["state"],
                                dfinal=df)
    x = {k: t[k].double().cpu() for k in FLOATS}
    for k in FLOATS:
        v = torch.randn(x[k].shape, generator=gen, dtype=torch.float64)

        def loss(s):
            y = {**x, k: x[k] + s * v}
            out, fin = ref.scan(*(y[n] for n in ("u", "delta", "A", "B", "C")), D=y["D"], z=y["z"], delta_bias=y["delta_bias"], state=y["state"])
            return float((out * dy.double().cpu()).sum() + (fin * df.double().cpu()).sum())
        slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
        got = g[k].double().cpu() * v
        assert abs(float(got.sum()) - slope) <= 2.0 ** -13 * float(got.abs().sum()), k


def test_same_bits_every_time(ptq):
    t = make(41, ref.BF16, 3, 300, 96, 16, G=2, state=True)
    history = ptq.scan_history(t["u"], 16)
    y = call(ptq, t, history=history)
    dy = torch.randn_like(y)
    run = lambda: ptq.gated_scan_backward(dy, t["u"], t["delta"], t["A"], t["B"], t["C"], history, D=t["D"], z=t["z"], delta_bias=t["delta_bias"],
                                          state=t["state"])
    first = run()
    for _ in range(3):
        assert torch.equal(call(ptq, t), y)
        again = run()
        for k in FLOATS:
            assert torch.equal(first[k], again[k])


def test_cases_cover_every_random_shape(ptq):
    """Random calls over the whole range of arguments."""
    rng = random.Random(5)
    for i in range(40):
        G = rng.choice([1, 1, 2, 3])
        D, N, B, L = G * rng.randint(1, 40), rng.randint(1, 32), rng.randint(1, 4), rng.randint(1, 70)
        lengths = [rng.randint(0, L) for _ in range(B)] if rng.random() < 0.4 else None
        t = make(100 + i, rng.choice([ref.F32, ref.F16, ref.BF16]), B, L, D, N, G=G, gate=rng.random() < 0.6, skip=rng.random() < 0.6,
                 bias=rng.random() < 0.8, state=rng.random() < 0.5, lengths=lengths, odd=rng.random() < 0.4)
        check(ptq, t, reverse=rng.random() < 0.5, dfinal=rng.random() < 0.6)
