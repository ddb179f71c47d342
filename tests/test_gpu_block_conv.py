"""short_conv and short_conv_backward against the formula in 64 bits."""
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


def make(seed, dtype, B, L, D, W, bias=True, state=False, lengths=None, pad=0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    x = r(B, L, D + pad).to(dtype).cuda()[..., pad:]
    t = {"x": x, "weight": r(D, W).cuda(), "bias": r(D).cuda() if bias else None, "state": r(B, W - 1, D).to(dtype).cuda() if state else None}
    lengths_t = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    if lengths is not None:
        for b, n in enumerate(lengths):
            x[b, max(n, 0):] = float("nan")
    return t, lengths_t


def check(ptq, t, lengths=None, silu=True, reverse=False, dfinal=True, seed=4):
    B, L, D = t["x"].shape
    W = t["weight"].shape[1]
    kw = dict(lengths=lengths, silu=silu, reverse=reverse)
    final = torch.full((B, W - 1, D), 9.0, dtype=t["x"].dtype, device="cuda")
    y = ptq.short_conv(t["x"], t["weight"], t["bias"], t["state"], **kw, final_state=final)
    x64 = ref.leaves(t)
    y64, f64 = ref.conv(x64["x"], x64["weight"], x64.get("bias"), x64.get("state"), **kw)
    mag = {k: v.detach().abs() for k, v in x64.items()}
    pre_abs, _ = ref.conv(mag["x"], mag["weight"], mag.get("bias"), mag.get("state"), lengths=lengths, silu=False, reverse=reverse)
    f = 2.0 ** -19
    ref.close(y, y64, pre_abs * 1.2, f, "y")
    assert torch.equal(final.double().cpu(), f64.detach()), "final state"
    gen = torch.Generator().manual_seed(seed)
    dy = torch.randn(B, L, D, generator=gen).to(t["x"].dtype).cuda()
    df = torch.randn(B, W - 1, D, generator=gen).to(t["x"].dtype).cuda() if dfinal else None
    g64 = ref.gradients((y64, f64), (dy, df), x64)
    got = ptq.short_conv_backward(dy, t["x"], t["weight"], t["bias"], t["state"], **kw, dfinal=df)
    # by magnitude: the gradient of the linear convolution of magnitudes, with dpre off by f (1 + pre) relative to dy
    m = {k: v.clone().requires_grad_() for k, v in mag.items()}
    lin, fin = ref.conv(m["x"], m["weight"], m.get("bias"), m.get("state"), lengths=lengths, silu=False, reverse=reverse)
    bound = ref.gradients((lin, fin), (dy.double().cpu().abs() * (2 + pre_abs), None if df is None else df.abs()), m)
    for k in t:
        if t[k] is None:
            assert got[k] is None
            continue
        assert got[k].dtype == t[k].dtype
        ref.close(got[k], g64[k], bound[k], f, "gradient of " + k)


@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("L", [1, 2, 3, 4, 5, 8, 9, 33, 130])
@pytest.mark.parametrize("dtype", [ref.F32, ref.F16, ref.BF16], ids=["f32", "f16", "bf16"])
def test_taps_lengths_and_types(ptq, W, L, dtype):
    t, _ = make(W * 100 + L, dtype, 2, L, 24, W, state=L % 2 == 0)
    check(ptq, t, silu=L != 5, reverse=W == 3)


@pytest.mark.parametrize("D", [1, 2, 3, 4, 7, 8, 20, 127, 128, 129, 260])
@pytest.mark.parametrize("pad", [0, 1, 4])
def test_channels_and_row_alignment(ptq, D, pad):
    t, _ = make(D, ref.F16, 3, 19, D, 4, state=True, pad=pad)
    check(ptq, t)
    t, _ = make(D, ref.F32, 2, 11, D, 3, bias=False, pad=pad)
    check(ptq, t, reverse=True, dfinal=False)


@pytest.mark.parametrize("lengths", [[0, 0, 0], [1, 0, 40], [2, 3, 16], [39, 100, -1], [17, 40, 15]])
@pytest.mark.parametrize("reverse", [False, True])
def test_padded_batches(ptq, lengths, reverse):
    for W, state in ((4, True), (2, False)):
        t, n = make(sum(map(abs, lengths)), ref.BF16, 3, 40, 33, W, state=state, lengths=lengths)
        check(ptq, t, n, reverse=reverse)
        y = torch.full((3, 40, 33), 5.0, dtype=ref.BF16, device="cuda")
        assert ptq.short_conv(t["x"], t["weight"], state=t["state"], lengths=n, reverse=reverse, y=y) is y
        for b, k in enumerate(lengths):
            assert (y[b, max(k, 0):] == 5.0).all()


def test_long_sequences_and_many(ptq):
    t, _ = make(1, ref.F32, 1, 1500, 8, 4, state=True)
    check(ptq, t)
    t, _ = make(2, ref.F16, 130, 9, 12, 4)
    check(ptq, t, reverse=True)


def test_pieces_tokens_and_states_in_place(ptq):
    """One call, pieces that hand the state on, tokens one by one (a state that is replaced each time): the same values."""
    t, _ = make(3, ref.BF16, 3, 50, 40, 4, state=True)
    final = torch.empty_like(t["state"])
    whole = ptq.short_conv(t["x"], t["weight"], t["bias"], t["state"], final_state=final)
    for cuts in ([2, 3, 30, 50], list(range(1, 51))):
        state, at, parts = t["state"].clone(), 0, []
        for end in cuts:
            parts.append(ptq.short_conv(t["x"][:, at:end], t["weight"], t["bias"], state, final_state=state))
            at = end
        assert torch.equal(torch.cat(parts, 1), whole) and torch.equal(state, final)
    state = t["state"].clone()                                # many segments, and the state is still read before it is replaced
    assert torch.equal(ptq.short_conv(t["x"], t["weight"], t["bias"], state, final_state=state), whole) and torch.equal(state, final)


def test_nan_reaches_its_taps_only(ptq):
    t, _ = make(4, ref.F32, 1, 20, 16, 4)
    clean = ptq.short_conv(t["x"], t["weight"], t["bias"])
    t["x"][0, 7, 5] = float("nan")
    y = ptq.short_conv(t["x"], t["weight"], t["bias"])
    mask = torch.ones(1, 20, 16, dtype=torch.bool)
    mask[0, 7:11, 5] = False
    assert torch.equal(y.cpu()[mask], clean.cpu()[mask]) and torch.isnan(y[0, 7:11, 5]).all()


def test_gradients_against_differences(ptq):
    t, _ = make(5, ref.F32, 2, 13, 12, 4, state=True)
    gen = torch.Generator().manual_seed(2)
    dy, df = torch.randn(2, 13, 12, generator=gen).cuda(), torch.randn(2, 3, 12, generator=gen).cuda()
    g = ptq.short_conv_backward(dy, **t, dfinal=df)
    x = {k: v.double().cpu() for k, v in t.items()}
    for k in t:
        v = torch.randn(x[k].shape, generator=gen, dtype=torch.float64)

        def loss(s):
            y, f = ref.conv(**{**x, k: x[k] + s * v})
            return float((y * dy.double().cpu()).sum() + (f * df.double().cpu()).sum())
        got = g[k].double().cpu() * v
        assert abs(float(got.sum()) - (loss(1e-5) - loss(-1e-5)) / 2e-5) <= 2.0 ** -15 * float(got.abs().sum()), k


def test_random_calls(ptq):
    rng = random.Random(6)
    for i in range(40):
        B, L, D, W = rng.randint(1, 5), rng.randint(1, 60), rng.randint(1, 70), rng.randint(2, 4)
        lengths = [rng.randint(0, L) for _ in range(B)] if rng.random() < 0.4 else None
        t, n = make(50 + i, rng.choice([ref.F32, ref.F16, ref.BF16]), B, L, D, W, rng.random() < 0.7, rng.random() < 0.5, lengths, rng.choice([0, 0, 3]))
        check(ptq, t, n, silu=rng.random() < 0.7, reverse=rng.random() < 0.5, dfinal=rng.random() < 0.6)
