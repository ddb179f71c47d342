"""Steps of decays so strong that they leave nothing of the state, among steps that leave nearly all of it.

Tolerances do not grow with the strong steps: what is off by their argument is nothing.  Of one chunk of 64 steps in binary32, relative to the sums over
absolute values: operands have 22 bits and the product of their lower parts is left out (3 x 2^-22), 6 partial sums of 16 terms are cut off (6 x 2^-23), up to 4 of them
are added (4 x 2^-24): 2^-19.1 a product.  A factor is off by its power of two (2^-22) and its argument, x 2^-24 e^-x at most: 2^-21.4.  y and the final state take two
products and a factor: 2^-17.9.  R = dy . u and P = C . B, a factor and one more product make du, dB and dC: the same.  Gradients of delta
and A add products of three, 64 steps and the states of a head in a row (64 x 2^-24 each), to what dw adds: 2^-15.5.  Activations of 16 bits: a strong step
counts as 2^-256 at least, so behind up to 8 of them in 16 steps the sums of logarithms are little more than 2^11; two of them rounded are off by 2^-12, a factor by
ln 2 times that: 2^-12.5 more."""
import pytest
import torch

import heads_ref as ref
from block_ref import BF16, F16, F32, close

pytestmark = pytest.mark.gpu
KW = dict(softplus=False, scale_input=False)
Y, GRADS, MORE = 2.0 ** -17.9, 2.0 ** -15.5, 2.0 ** -12.5


@pytest.fixture(scope="module")
def ptq():
    import __graft_entry__ as entry
    entry.build()
    import paper_2412_20386_b200 as p
    torch.cuda.set_device(0)
    return p


def make(dtype, strong, at, L=64, H=2, P=16, N=16):
    gen = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=gen)
    delta = torch.rand(1, L, H, generator=gen) * 0.1 + 0.01
    delta[:, at] = strong
    return {"u": r(1, L, H, P).to(dtype).cuda(), "delta": delta.to(dtype).cuda(), "A": torch.tensor([-1.0, -0.7])[:H].cuda(), "B": r(1, L, N).to(dtype).cuda(),
            "C": r(1, L, N).to(dtype).cuda(), "D": None, "delta_bias": None, "state": None, "lengths": None}


@pytest.mark.parametrize("reverse", [False, True], ids=["first to last", "last to first"])
@pytest.mark.parametrize("at", [[3], [0, 1, 2, 3, 4, 5, 6, 7], [17, 18, 40, 41, 42, 43, 44, 45, 46, 47, 48, 49, 50, 63]], ids=["one", "eight", "many"])
@pytest.mark.parametrize("strong", [70.0, 300.0, 5000.0, 60000.0])
@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
def test_weak_steps_beside_strong_ones(ptq, dtype, strong, at, reverse):
    t = make(dtype, strong, at)
    more = 0.0 if dtype == F32 else MORE
    gen = torch.Generator().manual_seed(6)
    dy, dfinal = torch.randn(1, 64, 2, 16, generator=gen).to(dtype), torch.randn(1, 2, 16, 16, generator=gen)
    value, scale, _ = ref.solve(t, dy=dy, dfinal=dfinal, reverse=reverse, **KW)
    final, history = torch.empty(1, 2, 16, 16, device="cuda"), ptq.head_scan_history(t["u"], 16)
    y = ptq.head_scan(t["u"], t["delta"], t["A"], t["B"], t["C"], final_state=final, history=history, reverse=reverse, **KW)
    close(y, value["y"], scale["y"], ref.factor("y", dtype, Y + more), "y")
    close(final, value["final"], scale["final"], Y, "final state")
    g = ptq.head_scan_backward(dy.cuda(), t["u"], t["delta"], t["A"], t["B"], t["C"], history, reverse=reverse, dfinal=dfinal.cuda(), **KW)
    for k in ("u", "B", "C"):
        close(g[k], value[k], scale[k], ref.factor(k, dtype, Y + more), "d" + k)
    for k in ("delta", "A"):
        close(g[k], value[k], scale[k], GRADS + more, "d" + k)


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("none", [-200.0, -float("inf")], ids=str)
def test_steps_of_no_length_with_an_infinite_rate(ptq, dtype, none):
    """A = -inf: a step leaves nothing of the state, unless softplus gives it no length in binary32; then it leaves the state as it is, and delta has no gradient."""
    at = [0, 5, 6, 40, 41, 42, 43, 44, 45, 46, 47, 48, 63]
    t = make(dtype, -200.0, at)
    t["A"] = torch.tensor([-float("inf"), -0.7], device="cuda")
    t["delta_bias"] = torch.tensor([-1.0, 0.5], device="cuda")
    gen = torch.Generator().manual_seed(6)
    dy = torch.randn(1, 64, 2, 16, generator=gen).to(dtype)
    value, scale, _ = ref.solve({**t, "A": torch.tensor([-1e30, -0.7])}, dy=dy)              # 64 bits: the same decays
    t["delta"][:, at] = none
    history = ptq.head_scan_history(t["u"], 16)
    y = ptq.head_scan(t["u"], t["delta"], t["A"], t["B"], t["C"], delta_bias=t["delta_bias"], history=history)
    close(y, value["y"], scale["y"], ref.factor("y", dtype, Y), "y")
    g = ptq.head_scan_backward(dy.cuda(), t["u"], t["delta"], t["A"], t["B"], t["C"], history, delta_bias=t["delta_bias"])
    for k in ("u", "B", "C"):
        close(g[k], value[k], scale[k], ref.factor(k, dtype, Y), "d" + k)
    for k in ("delta", "A", "delta_bias"):
        close(g[k], value[k], scale[k], GRADS, "d" + k)
