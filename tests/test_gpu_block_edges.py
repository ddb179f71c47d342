"""Calls of the operators between a block's linears at the edges of what their documents allow, against 64 bits."""
import ctypes
import itertools

import pytest
import torch

import block_ref as ref
from parity_util import launches
from test_block_host import Norm
from test_gpu_block_norm import make as make_norm
from test_gpu_block_norm_stream import check as check_norm
from test_gpu_block_scan import check as check_scan, make as make_scan

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ptq():
    import __graft_entry__ as entry
    entry.build()
    import paper_2412_20386_b200 as p
    torch.cuda.set_device(0)
    return p


@pytest.mark.parametrize("kind,gate_at", list(itertools.product(["rms", "layer"], ["in", "out"])))
def test_norm_without_eps_and_an_incomplete_last_set_of_rows(ptq, kind, gate_at):
    """Rows are taken two at a time from 1185 on; with eps = 0 a row that is not there has no finite 1 / rms."""
    for M, D in ((1185, 72), (1187, 264), (1187, 35)):
        check_norm(ptq, make_norm(M, ref.BF16, M, D, None, True, True), kind, gate_at, ref.BF16, eps=0.0)
    check_norm(ptq, make_norm(1, ref.F32, 1185, 40, None), kind, gate_at, None, eps=0.0)


def growing(L, D, N):
    """Rates above zero without softplus: dt is delta."""
    gen = torch.Generator().manual_seed(L)
    r = lambda *s: torch.rand(*s, generator=gen) * 0.5 + 0.5
    t = {"u": r(1, L, D), "delta": torch.full((1, L, D), 3.0), "A": torch.ones(D, N), "B": r(1, L, N), "C": r(1, L, N)}
    return {k: v.cuda() for k, v in t.items()}


def test_states_that_grow_beyond_binary32_within_a_chunk_but_start_from_nothing(ptq):
    """32 steps of e^3 are 2^138, more than binary32 holds; nothing comes in that they would multiply, in either direction, and the last eight
    steps give e^21.  Bound: all terms are positive; a step's decay is off by 2^-22 + 3 (2^-21 + 2^-24), at most 2^-19, over eight steps."""
    t = growing(200, 8, 16)
    t["u"][:, :192] = 0.0
    args = [t[k] for k in ("u", "delta", "A", "B", "C")]
    final, history = torch.empty(1, 8, 16, device="cuda"), ptq.scan_history(t["u"], 16)
    assert launches(ptq, lambda: ptq.gated_scan(*args, softplus=False)) == 2             # cut into chunks
    y = ptq.gated_scan(*args, softplus=False, final_state=final, history=history)
    x64 = ref.leaves(t)
    y64, f64 = ref.scan(*(x64[k] for k in ("u", "delta", "A", "B", "C")), softplus=False)
    ref.close(y, y64, y64.abs(), 2.0 ** -16, "y")
    ref.close(final, f64, f64.abs(), 2.0 ** -16, "final state")
    dy = torch.rand(1, 200, 8, device="cuda") + 0.5
    dy[:, 8:] = 0.0                                         # the gradient of the state grows from here to the front
    want = ref.gradients((y64, f64), (dy, None), x64)
    got = ptq.gated_scan_backward(dy, *args, history, softplus=False)
    for k in ("u", "delta", "A", "B", "C"):
        ref.close(got[k], want[k], want[k].abs(), 2.0 ** -16, "gradient of " + k)


def test_a_small_state_that_grows_by_more_than_binary32_holds(ptq):
    """1e-20 times e^96 in one chunk of 32 steps.  Bound: 32 steps of 2^-19."""
    t = growing(200, 8, 16)
    t["delta"].zero_()
    t["delta"][:, 0], t["delta"][:, 32:64] = 1.0, 3.0
    t["u"].zero_()
    t["u"][:, 0] = 1e-20
    args = [t[k] for k in ("u", "delta", "A", "B", "C")]
    final = torch.empty(1, 8, 16, device="cuda")
    y = ptq.gated_scan(*args, softplus=False, final_state=final)
    y64, f64 = ref.scan(*(v.double().cpu() for v in args), softplus=False)
    ref.close(y, y64, y64.abs(), 2.0 ** -14, "y")
    ref.close(final, f64, f64.abs(), 2.0 ** -14, "final state")


def test_the_gradient_of_a_scale_that_is_not_given(ptq):
    """C ABI: like the weight, a scale that is NULL is 1 and has a gradient if one is asked for."""
    from paper_2412_20386_b200 import binding
    lib = binding.load_library()
    lib.ptq_norm_workspace_bytes.restype = ctypes.c_size_t
    rows, cols = 37, 72
    x, gate, dy = (torch.randn(rows, cols, device="cuda") for _ in range(3))
    one, dx, dgate = torch.ones(cols, device="cuda"), torch.empty_like(x), torch.empty_like(x)
    got = []
    for scale in (one, None):
        n = Norm(dtype=2, residual_dtype=2, rows=rows, cols=cols, eps=1e-5, x=x.data_ptr(), x_pitch=cols, gate=gate.data_ptr(), gate_pitch=cols,
                 scale=None if scale is None else scale.data_ptr())
        space = torch.empty(lib.ptq_norm_workspace_bytes(ctypes.byref(n)), dtype=torch.uint8, device="cuda")
        sums = torch.full((3, cols), 7.0, device="cuda")
        grads = (ctypes.c_void_p * 6)(dx.data_ptr(), dgate.data_ptr(), None, *(s.data_ptr() for s in sums))
        st = lib.ptq_norm_backward(ctypes.byref(n), ctypes.c_void_p(dy.data_ptr()), None, grads, ctypes.c_void_p(space.data_ptr()),
                                   ctypes.c_size_t(space.numel()), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert st == 0
        got.append(sums)
    assert torch.equal(*got) and (got[0][2].abs() > 0).any()


def test_a_binary32_stream_that_begins_beside_16_bit_activations(ptq):
    """The first block of a network: its x begins a residual stream of binary32, whose gradient comes back as binary32."""
    for dtype, D in ((ref.BF16, 72), (ref.F16, 35)):
        t = make_norm(D, dtype, 40, D, None, True, True)
        out = torch.empty(40, D, device="cuda")
        y, r = ptq.block_norm(t["x"], t["weight"], t["bias"], scale=t["scale"], gate=t["gate"], residual_out=out)
        _, r64 = ref.norm(t["x"].double().cpu(), scale=t["scale"].double().cpu(), gate=t["gate"].double().cpu())
        assert r is out
        ref.close(r, r64, r64.abs(), 2.0 ** -19, "r")
        assert torch.equal(y, ptq.block_norm(t["x"], t["weight"], t["bias"], scale=t["scale"], gate=t["gate"]))
        for kind, gate_at in itertools.product(["rms", "layer"], ["in", "out"]):
            check_norm(ptq, t, kind, gate_at, ref.F32)
    wide = make_norm(9, ref.BF16, 1300, 2056, None, True)
    check_norm(ptq, wide, "layer", "in", ref.F32)
    for bad in (torch.empty(40, 35, device="cuda", dtype=torch.bfloat16), torch.empty(40, 35, device="cuda", dtype=torch.float64)):
        with pytest.raises(ValueError):
            ptq.block_norm(t["x"], residual_out=bad)
        with pytest.raises(ValueError):
            ptq.block_norm_backward(t["x"].contiguous(), t["x"], dresidual_out=bad)


def test_single_tokens_of_empty_sequences(ptq):
    """What belongs to a sequence of no tokens is not read: it may be anything."""
    for N, B in ((16, 9), (2, 3), (32, 20)):
        t = make_scan(N, ref.BF16, B, 1, 40, N, state=True, lengths=[b % 2 for b in range(B)])
        check_scan(ptq, t, train=False)


def test_padded_reversed_groups_in_many_chunks(ptq):
    t = make_scan(77, ref.F32, 3, 1100, 12, 16, G=2, state=True, lengths=[1100, 555, 3])
    check_scan(ptq, t, reverse=True)
    t = make_scan(78, ref.BF16, 2, 900, 18, 8, G=3, odd=True, lengths=[33, 890])
    check_scan(ptq, t, reverse=True, dfinal=False)
