"""head_scan, head_scan_backward and head_scan_step against the recurrence in 64 bits."""
import pytest
import torch

import heads_ref as ref
from block_ref import BF16, F16, F32, close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ptq():
    import __graft_entry__ as entry
    entry.build()
    import paper_2412_20386_b200 as p
    torch.cuda.set_device(0)
    return p


def make(seed, dtype, B, L, H, P, N, G=1, skip=True, state=False, lengths=None, odd=0, ungrouped=False, fixed=False, bias=True, decay=4.0):
    """Inputs as a block has them: u, B and C the columns of one tensor; `odd` shifts and widens its rows by so many elements."""
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    xbc = r(B, L, H * P + 2 * G * N + odd).to(dtype).cuda()[..., odd:]
    dl = (r(B, L, H + odd) * 0.5).to(dtype).cuda()[..., odd:]
    t = {"u": xbc[..., :H * P].unflatten(-1, (H, P)), "delta": None if fixed else dl,
         "A": (-decay * torch.rand(H, generator=gen) * (0.05 if fixed else 1.0)).cuda(),
         "B": xbc[..., H * P:H * P + G * N].unflatten(-1, (G, N)), "C": xbc[..., H * P + G * N:].unflatten(-1, (G, N)),
         "D": r(H).cuda() if skip else None, "delta_bias": None if fixed or not bias else (r(H) - 3.0).cuda(),
         "state": r(B, H, P, N).cuda() if state else None}
    if ungrouped:
        t["B"], t["C"] = t["B"][:, :, 0], t["C"][:, :, 0]
    t["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    if lengths is not None:                                  # what lies behind the ends is not read
        for b, n in enumerate(lengths):
            for k in ("u", "delta", "B", "C"):
                if t[k] is not None:
                    t[k][b, max(n, 0):] = float("nan")
    return t


def call(ptq, t, **kw):
    return ptq.head_scan(t["u"], t["delta"], t["A"], t["B"], t["C"], D=t["D"], delta_bias=t["delta_bias"], state=t["state"], lengths=t["lengths"], **kw)


def back(ptq, t, dy, history, **kw):
    return ptq.head_scan_backward(dy, t["u"], t["delta"], t["A"], t["B"], t["C"], history, D=t["D"], delta_bias=t["delta_bias"], state=t["state"],
                                  lengths=t["lengths"], **kw)


def check(ptq, t, train=True, seed=7, **kw):
    B, L, H, P = t["u"].shape
    N, T = t["B"].shape[-1], t["u"].dtype
    gen = torch.Generator().manual_seed(seed)
    dy = torch.randn(B, L, H, P, generator=gen).to(T).cuda()
    dfinal = torch.randn(B, H, P, N, generator=gen).cuda() if t["state"] is not None else None
    value, scale, F = ref.solve(t, dy=dy if train else None, dfinal=dfinal, **kw)
    final = torch.full((B, H, P, N), 7.0, device="cuda")
    history = ptq.head_scan_history(t["u"], N) if train else None
    y = call(ptq, t, final_state=final, history=history, **kw)
    close(y, value["y"], scale["y"], ref.factor("y", T, F), "y")
    close(final, value["final"], scale["final"], ref.factor("final", F32, F), "final state")
    if not train:
        return
    g = back(ptq, t, dy, history, dfinal=dfinal, **kw)
    for k, v in g.items():
        if t[k] is None:
            assert v is None, k
        else:
            assert v.shape == t[k].shape and v.is_contiguous() and v.dtype == (T if k in ("u", "delta", "B", "C") else F32), k
            close(v, value[k], scale[k], ref.factor(k, v.dtype, F), "d" + k)
    again = back(ptq, t, dy, history, dfinal=dfinal, **kw)
    assert all(v is None or torch.equal(v, again[k]) for k, v in g.items())               # the same call, the same bits


SHAPES = [
    # B, L, H, P, N, more
    (2, 64, 2, 64, 64, {}),
    (1, 1, 1, 1, 1, {}),
    (2, 1, 3, 64, 16, dict(state=True)),
    (1, 63, 2, 16, 32, dict(state=True)),
    (1, 65, 2, 33, 33, dict(state=True, G=2)),
    (2, 130, 4, 64, 128, dict(G=2, skip=False)),
    (1, 197, 2, 128, 16, dict(state=True, ungrouped=True)),
    (2, 100, 3, 65, 7, dict(state=True, odd=1)),
    (1, 80, 2, 130, 100, dict(odd=2, state=True)),
    (1, 70, 2, 200, 24, dict(odd=4)),
    (1, 72, 1, 256, 128, dict(state=True)),
    (4, 90, 2, 50, 24, dict(lengths=[90, 0, 1, 65], state=True)),
    (3, 150, 2, 24, 40, dict(lengths=[64, 200, -3], odd=1)),
    (2, 140, 3, 40, 64, dict(fixed=True, state=True)),
    (2, 66, 2, 64, 64, dict(bias=False)),
]


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:5])))
@pytest.mark.parametrize("reverse", [False, True], ids=["first to last", "last to first"])
def test_values_and_gradients(ptq, shape, dtype, reverse):
    B, L, H, P, N, more = shape
    check(ptq, make(1, dtype, B, L, H, P, N, **more), reverse=reverse)


@pytest.mark.parametrize("kw", [dict(softplus=False), dict(scale_input=False), dict(softplus=False, scale_input=False)], ids=str)
@pytest.mark.parametrize("dtype", [F16, F32], ids=["fp16", "fp32"])
def test_flags(ptq, kw, dtype):
    t = make(2, dtype, 2, 100, 2, 64, 32, state=True)
    if not kw.get("softplus", True):
        t["delta"], t["delta_bias"] = t["delta"].abs() * 0.2, t["delta_bias"].abs() * 0.02
    check(ptq, t, **kw)


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("more", [dict(state=True), dict(lengths=[1500, 700], state=True), dict()], ids=["state", "lengths", "zeros"])
def test_long_sequences_are_cut_into_segments(ptq, dtype, more):
    """Two heads of two sequences: far fewer than the GPU holds at once, so the sequences are cut; states join them, decays of seconds do not fade."""
    t = make(3, dtype, 2, 1500, 2, 16, 16, decay=0.5, **more)
    check(ptq, t, reverse=True)
    if t["state"] is not None:                               # the final state may be written over the first one
        final = torch.empty_like(t["state"])
        y = call(ptq, t, final_state=final)
        state = t["state"].clone()
        assert torch.equal(call(ptq, {**t, "state": state}, final_state=state), y) and torch.equal(state, final)


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("P,N,odd", [(64, 128, 0), (37, 19, 0), (130, 64, 0), (16, 4, 1), (1, 1, 0)])
def test_single_tokens(ptq, dtype, P, N, odd):
    """A step is binary32 throughout: y is off by half a step of its type and a sum of N products."""
    t = make(4, dtype, 3, 5, 4, P, N, G=2, state=True, odd=odd)
    state = t["state"].clone()
    for i in range(5):
        before = state.clone()
        one = {**t, "state": before, **{k: t[k][:, i:i + 1] for k in ("u", "delta", "B", "C")}}
        value, scale, F = ref.solve(one)
        y = ptq.head_scan_step(state, t["u"][:, i], t["delta"][:, i], t["A"], t["B"][:, i], t["C"][:, i], D=t["D"], delta_bias=t["delta_bias"])
        close(y[:, None], value["y"], scale["y"], F, "y")
        close(state, value["final"], scale["final"], F, "state")
        new = torch.empty_like(state)
        y2 = ptq.head_scan_step(before, t["u"][:, i], t["delta"][:, i], t["A"], t["B"][:, i], t["C"][:, i], D=t["D"], delta_bias=t["delta_bias"], new_state=new)
        assert torch.equal(y, y2) and torch.equal(new, state)


def test_tokens_follow_the_whole_sequence(ptq):
    t = make(5, BF16, 2, 70, 4, 64, 64, state=True)
    final, state = torch.empty_like(t["state"]), t["state"].clone()
    y = call(ptq, t, final_state=final)
    value, scale, F = ref.solve(t)
    for i in range(70):
        yi = ptq.head_scan_step(state, t["u"][:, i], t["delta"][:, i], t["A"], t["B"][:, i], t["C"][:, i], D=t["D"], delta_bias=t["delta_bias"])
        close(yi, value["y"][:, i], scale["y"][:, i], F, "token")
        close(y[:, i], value["y"][:, i], scale["y"][:, i], ref.factor("y", BF16, F), "sequence")
    close(state, value["final"], scale["final"], F, "state")


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")], ids=str)
@pytest.mark.parametrize("where", ["u", "B", "C", "delta"])
@pytest.mark.parametrize("at", [0, 5, 63, 64, 100])
def test_values_that_are_not_finite_reach_no_earlier_token(ptq, dtype, bad, where, at):
    t = make(6, dtype, 2, 130, 2, 64, 32, state=True)
    wfinal = torch.empty_like(t["state"])
    want = call(ptq, t, final_state=wfinal)
    t[where][1, at, 1 if where in ("u", "delta") else 0, ...][() if where == "delta" else 3] = bad
    final = torch.empty_like(wfinal)
    y = call(ptq, t, final_state=final)
    assert torch.equal(y[1, :at], want[1, :at]) and torch.equal(y[0], want[0]) and torch.equal(final[0], wfinal[0])
    # log(1 + e^-inf) is 0: a step that leaves the state as it is
    assert torch.isfinite(y[1, at, 1]).all() == (where == "delta" and bad == -float("inf"))
    if where == "u":                                         # and no other column than its own
        rest = [c for c in range(64) if c != 3]
        assert torch.isfinite(y[1][:, :, rest]).all() and torch.isfinite(final[1][:, rest]).all() and not torch.isfinite(final[1, 1, 3]).any()
    if where == "C":                                         # and no other token
        assert torch.equal(y[1, at + 1:], want[1, at + 1:]) and torch.equal(final, wfinal)


def test_extreme_decays(ptq):
    for dtype in (F16, F32):
        t = make(7, dtype, 2, 130, 4, 32, 16, state=True)
        t["A"] = torch.tensor([-float("inf"), -1e4, 0.0, -1e-30], device="cuda")
        keep = {**t, "A": torch.tensor([-1e30, -1e4, 0.0, -1e-30], device="cuda")}       # 64 bits: the same decays
        value, scale, F = ref.solve(keep)
        F = 2.0 ** -16 * (1 + 130 / 64)
        final = torch.empty_like(t["state"])
        y = call(ptq, t, final_state=final)
        close(y, value["y"], scale["y"], ref.factor("y", dtype, F), "y")
        close(final, value["final"], scale["final"], F, "final")
        h = ptq.head_scan_history(t["u"], 16)
        call(ptq, t, history=h)
        assert all(torch.isfinite(v).all() for k, v in back(ptq, t, y, h).items())


def test_binary16_keeps_its_range(ptq):
    """Products of operands that binary16 cannot hold, and columns 2^16 apart: the small ones are not lost beside the large ones."""
    t = make(8, F16, 1, 130, 2, 64, 32, state=True)
    t["u"][..., 5] = (t["u"][..., 5] * 2e4).clamp(-6e4, 6e4)
    t["B"] *= 60.0
    t["C"][:, 64:] *= 1.0 / 4096
    t["state"][:, :, 7] *= 1e-3
    t["D"] = None
    value, scale, F = ref.solve(t)
    final = torch.empty_like(t["state"])
    y = call(ptq, t, final_state=final)
    close(final, value["final"], scale["final"], F, "final")
    finite = value["y"].abs() < 65504
    # an operand is rounded by half a step, or by 2^-25 of the largest of its 16 columns (16 steps)
    top = scale["y"].unflatten(-1, (4, 16)).amax(-1, keepdim=True).expand(1, 130, 2, 4, 16).flatten(-2)
    lim = 2.0 ** -11 * value["y"].abs() + (2.0 ** -11 + F) * scale["y"] + 2.0 ** -20 * top + 2.0 ** -24
    assert ((y.double().cpu() - value["y"]).abs() <= lim)[finite].all()


def test_padding_is_left_alone(ptq):
    t = make(9, BF16, 3, 100, 2, 32, 16, lengths=[100, 30, 0], state=True)
    y, final = torch.full((3, 100, 2, 32), 9.0, dtype=BF16, device="cuda"), torch.empty_like(t["state"])
    history = torch.full((3, 2, 2, 32, 16), 9.0, device="cuda")
    assert call(ptq, t, y=y, final_state=final, history=history) is y
    assert (y[1, 30:] == 9).all() and (y[2] == 9).all() and torch.equal(final[2], t["state"][2])
    assert (history[1, 1] == 9).all() and (history[2] == 9).all() and torch.equal(history[:2, 0], t["state"][:2])
    fresh = call(ptq, t)
    assert (fresh[1, 30:] == 0).all() and (fresh[2] == 0).all()
    g = back(ptq, t, torch.full_like(y, float("nan")).masked_fill_((torch.arange(100, device="cuda")[None] < t["lengths"][:, None])[..., None, None], 1.0), history)
    assert all(torch.isfinite(v).all() for v in g.values())
    assert all((g[k][1, 30:] == 0).all() and (g[k][2] == 0).all() for k in ("u", "delta", "B", "C"))


def test_gradients_against_differences(ptq):
    """Along random directions: (loss(x + h d) - loss(x - h d)) / 2h in 64 bits against the kernels' gradients, binary32."""
    t = make(10, F32, 1, 70, 2, 8, 8, state=True)
    gen = torch.Generator().manual_seed(3)
    dy, dfinal = torch.randn(1, 70, 2, 8, generator=gen), torch.randn(1, 2, 8, 8, generator=gen)
    history = ptq.head_scan_history(t["u"], 8)
    call(ptq, t, history=history)
    g = back(ptq, t, dy.cuda(), history, dfinal=dfinal.cuda())

    def loss(x):
        v, _, _ = ref.solve(x)
        return float((v["y"] * dy.double()).sum() + (v["final"] * dfinal.double()).sum())
    for k in ref.NAMES:
        d = torch.randn(t[k].shape, generator=gen, dtype=torch.float64)
        h = 1e-4
        near = [loss({**t, k: t[k].double().cpu() + s * h * d}) for s in (1, -1)]
        want, got = (near[0] - near[1]) / (2 * h), float((g[k].double().cpu() * d).sum())
        # second-order differences leave h^2 of the third derivative (below 1e3 of the loss's own size here); binary32 the rest
        size = float((g[k].double().cpu() * d).abs().sum())
        assert abs(got - want) <= 1e-4 * size + 1e-5 * abs(want), k
