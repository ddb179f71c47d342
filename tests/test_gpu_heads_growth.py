"""Decays above 1 (A < 0 with negative dt here): growth that binary32 holds over 64 steps, across sequences that are cut into segments.

Tolerances.  Errors are relative to the recurrence over absolute values: a chunk of 64 steps adds 2^-16 (1 + max |dt A|) of it at most (heads_ref: F without its
memory, which growth makes as large as the growth), and what a chunk is off by grows as that recurrence does: 2^-16 (1 + chunks) (1 + max |dt A|) in all."""
import pytest
import torch

import heads_ref as ref
from block_ref import BF16, F16, F32, close

pytestmark = pytest.mark.gpu
KW = dict(softplus=False, scale_input=False)                 # dt = delta, inputs u B^T


@pytest.fixture(scope="module")
def ptq():
    import __graft_entry__ as entry
    entry.build()
    import paper_2412_20386_b200 as p
    torch.cuda.set_device(0)
    return p


def make(dtype, L, H, P, N, seed=1):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    return {"u": r(1, L, H, P).to(dtype).cuda(), "delta": torch.full((1, L, H), 0.0625).to(dtype).cuda(), "A": -torch.linspace(0.9, 1.0, H).cuda(),
            "B": r(1, L, N).to(dtype).cuda(), "C": r(1, L, N).to(dtype).cuda(), "D": r(H).cuda(), "delta_bias": None, "state": None, "lengths": None}


def forward(ptq, t, **more):
    return ptq.head_scan(t["u"], t["delta"], t["A"], t["B"], t["C"], D=t["D"], state=t["state"], **KW, **more)


def limit(L, most=1.0):
    return 2.0 ** -16 * (1 + -(-L // 64)) * (1 + most)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("start", [0.0, 1e-25], ids=["nothing to grow", "small to grow"])
def test_growth_over_a_segment(ptq, dtype, start):
    """3000 steps of two heads are cut into segments of 128.  The state grows by e^52 per 64 steps, e^104 (2^150) in all, from step 128 on; it
    shrinks from 256 on."""
    L = 3000
    t = make(dtype, L, 2, 16, 16)
    t["u"][:, :256] = 0
    t["delta"][:, 128:256] = -0.8125
    t["delta"][:, 256:640] = 0.125
    t["state"] = torch.randn(1, 2, 16, 16, device="cuda") * start
    value, scale, _ = ref.solve(t, **KW)
    assert torch.isfinite(value["y"]).all() and value["y"].abs().max() < 1e30
    final = torch.empty_like(t["state"])
    y = forward(ptq, t, final_state=final)
    close(y, value["y"], scale["y"], ref.factor("y", dtype, limit(L)), "y")
    close(final, value["final"], scale["final"], limit(L), "final state")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("end", [0.0, 1e-25], ids=["loss on early tokens", "small gradients behind"])
def test_gradients_grow_over_a_segment(ptq, dtype, end):
    """As many heads as make it worth cutting 1024 steps into segments of 256 (binary32: 128) for the backward pass.  States shrink by e^60 and more, then
    grow by e^104 (2^150) within a segment."""
    L, H = 1024, 155 if dtype == F32 else 310
    t = make(dtype, L, H, 4, 4)
    t["delta"][:, 320:512] = 0.3125
    t["u"][:, 320:] = 0
    t["delta"][:, 640:768] = -0.8125
    gen = torch.Generator().manual_seed(2)
    dy = torch.randn(1, L, H, 4, generator=gen).to(dtype)
    dy[:, 320:] = 0
    dfinal = torch.randn(1, H, 4, 4, generator=gen) * end
    value, scale, _ = ref.solve(t, dy=dy, dfinal=dfinal, **KW)
    history = ptq.head_scan_history(t["u"], 4)
    y = forward(ptq, t, history=history)
    close(y, value["y"], scale["y"], ref.factor("y", dtype, limit(L)), "y")
    g = ptq.head_scan_backward(dy.cuda(), t["u"], t["delta"], t["A"], t["B"], t["C"], history, D=t["D"], dfinal=dfinal.cuda(), **KW)
    for k, v in g.items():
        if v is not None:
            close(v, value[k], scale[k], ref.factor(k, v.dtype, limit(L)), "d" + k)


@pytest.mark.parametrize("H", [2, 160], ids=["few heads", "many heads"])
def test_binary16_operands_of_growth(ptq, H):
    """Factors of up to 2^83 within 64 steps, of inputs that are zero and of ones that are as small as binary16 has them, and states that are as large."""
    L = 256
    t = make(F16, L, H, 8, 32)
    t["delta"][:, 64:128] = -0.90625
    t["delta"][:, 128:192] = 1.0
    t["u"][:, 64:192] = 0
    t["u"][:, 66, ::2] = 2.0 ** -24                          # grows to 2^57, and shrinks to 2^-35
    t["u"][:, :64] = 0
    t["C"][:, 64:192:2] = 0                                  # y of the others would be more than binary16 holds:
    value, scale, _ = ref.solve(t, **KW)
    final = torch.empty(1, H, 8, 32, device="cuda")
    y = forward(ptq, t, final_state=final)
    held = value["y"].abs() < 65504
    assert held[:, ::2].all() and held[:, :, 1::2].all() and not held.all()
    assert torch.isfinite(y.cpu()[held]).all()
    close(torch.where(held.cuda(), y, 0), torch.where(held, value["y"], 0.0), torch.where(held, scale["y"], 1.0), ref.factor("y", F16, limit(L)), "y")
    close(final, value["final"], scale["final"], limit(L), "final state")
    # the gradients of a loss on the tokens in front of the growth and behind it
    gen = torch.Generator().manual_seed(2)
    dy = torch.randn(1, L, H, 8, generator=gen).half()
    dy[:, 64:192] = 0
    value, scale, _ = ref.solve(t, dy=dy, **KW)
    history = ptq.head_scan_history(t["u"], 32)
    forward(ptq, t, history=history)
    g = ptq.head_scan_backward(dy.cuda(), t["u"], t["delta"], t["A"], t["B"], t["C"], history, D=t["D"], **KW)
    for k, v in g.items():
        if v is not None:
            assert value[k].abs().max() < 65504
            close(v, value[k], scale[k], ref.factor(k, v.dtype, limit(L)), "d" + k)


def test_binary16_growth_over_a_segment(ptq):
    """test_growth_over_a_segment in binary16, which cannot hold what grows: nothing does."""
    L = 3000
    t = make(F16, L, 2, 16, 16)
    t["u"][:, :256] = 0
    t["delta"][:, 128:256] = -0.90625
    value, scale, _ = ref.solve(t, **KW)
    final = torch.empty(1, 2, 16, 16, device="cuda")
    y = forward(ptq, t, final_state=final)
    close(y, value["y"], scale["y"], ref.factor("y", F16, limit(L)), "y")
    close(final, value["final"], scale["final"], limit(L), "final state")
