"""Binary16 operands of linear attention that are formed in a call, 16 steps at a time, and brought into range by powers of two: sets of steps of very
different sizes.  Tolerances are those of heads_ref: half a step for the rounded operand, of 16 x 16 elements that are about as large, and F."""
import pytest
import torch

import heads_ref as ref
from block_ref import F16, close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ptq():
    import __graft_entry__ as entry
    entry.build()
    import paper_2412_20386_b200 as p
    torch.cuda.set_device(0)
    return p


def make(H=2, P=16, N=32, L=64):
    gen = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=gen)
    return {"u": r(1, L, H, P), "delta": None, "A": -torch.full((H,), 0.01), "B": r(1, L, N), "C": r(1, L, N), "D": None, "delta_bias": None, "state": None,
            "lengths": None}


def check(ptq, t, dy=None):
    t = {k: v if v is None else v.cuda() if k == "A" else v.half().cuda() for k, v in t.items()}
    dy = None if dy is None else dy.half()
    value, scale, F = ref.solve(t, dy=dy)
    assert value["y"].abs().max() < 65504
    history = None if dy is None else ptq.head_scan_history(t["u"], t["B"].shape[-1])
    y = ptq.head_scan(t["u"], None, t["A"], t["B"], t["C"], history=history)
    close(y, value["y"], scale["y"], ref.factor("y", F16, F), "y")
    if dy is not None:
        g = ptq.head_scan_backward(dy.cuda(), t["u"], None, t["A"], t["B"], t["C"], history)
        for k in ("u", "B", "C", "A"):
            close(g[k], value[k], scale[k], ref.factor(k, g[k].dtype, F), "d" + k)


@pytest.mark.parametrize("first", [0, 16, 32])
@pytest.mark.parametrize("front", ["B is zero", "u is zero"])
def test_small_scores_behind_a_set_that_gives_nothing(ptq, first, front):
    """Scores of about 2^-19 times u of about 2^11, behind 16 steps whose scores are zero, or large, of inputs that are zero."""
    t = make()
    t["B"] *= 2.0 ** -11
    t["C"] *= 2.0 ** -11
    t["u"] *= 2.0 ** 11
    if front == "B is zero":
        t["B"][:, first:first + 16] = 0
    else:
        t["B"][:, first:first + 16] *= 2.0 ** 24
        t["u"][:, first:first + 16] = 0
    check(ptq, t)


@pytest.mark.parametrize("at", [0, 20, 40, 63])
def test_a_small_loss_on_one_token(ptq, at):
    """dy . u of about 2^-19 times C of about 2^8 (dB) and B of about 2^2 (dC)."""
    t = make()
    t["u"] *= 2.0 ** -3
    t["B"] *= 2.0 ** 2
    t["C"] *= 2.0 ** 8
    dy = torch.zeros(1, 64, 2, 16)
    dy[:, at] = make()["u"][:, at] * 2.0 ** -18
    check(ptq, t, dy)


@pytest.mark.parametrize("first", [0, 16, 32])
@pytest.mark.parametrize("front", ["u is zero", "C is zero", "dy is zero"])
def test_small_gradients_beside_a_set_that_gives_nothing(ptq, first, front):
    """The same in the backward pass's products: 16 steps without u, C or dy among ones with small products."""
    t = make()
    t["u"] *= 2.0 ** -4
    t["B"] *= 2.0 ** 3
    t["C"] *= 2.0 ** 8
    dy = make()["u"].flip(1) * 2.0 ** -18
    if front == "u is zero":
        t["u"][:, first:first + 16] = 0
    elif front == "C is zero":
        t["C"][:, first:first + 16] = 0
        t["B"] *= 2.0 ** -14
        t["C"] *= 2.0 ** -17
        dy *= 2.0 ** 25
        t["u"] *= 2.0 ** -6
    else:
        dy[:, first:first + 16] = 0
    check(ptq, t, dy)


@pytest.mark.parametrize("first", [0, 16, 32, 48])
@pytest.mark.parametrize("front", ["u is zero", "B is zero", "u is small"])
def test_states_of_steps_among_ones_that_give_nothing(ptq, first, front):
    """Sixteen steps decide the final state, by a decay of up to 2^-46 beside what others would, and the gradient of the first one, by as much."""
    t = make()
    t["A"] = -torch.full((2,), 0.5)
    other = torch.ones(64, dtype=torch.bool)
    other[first:first + 16] = False
    dy = make()["u"].flip(1)
    if front == "u is small":
        t["u"][:, other] *= 2.0 ** -20
        dy[:, other] *= 2.0 ** -20
    else:
        t["u" if front == "u is zero" else "B"][:, other] = 0
        if front == "u is zero":
            dy[:, other] = 0
        else:
            t["C"][:, other] = 0
    t = {k: v if v is None else v.cuda() if k == "A" else v.half().cuda() for k, v in t.items()}
    t["state"] = torch.zeros(1, 2, 16, 32, device="cuda")
    value, scale, F = ref.solve(t, dy=dy.half())
    final, history = torch.empty_like(t["state"]), ptq.head_scan_history(t["u"], 32)
    ptq.head_scan(t["u"], None, t["A"], t["B"], t["C"], state=t["state"], final_state=final, history=history)
    close(final, value["final"], scale["final"], F, "final state")
    g = ptq.head_scan_backward(dy.half().cuda(), t["u"], None, t["A"], t["B"], t["C"], history, state=t["state"])
    close(g["state"], value["state"], scale["state"], F, "dstate")
