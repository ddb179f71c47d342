"""fp8_linear at the ends of its sizes, against 64 bits on what fp8_quantize gives.  Tolerances as for its other sizes: 2^-21 + 2^-24 ceil(K / 128) of the magnitudes."""
import pytest
import torch

from block_ref import BF16, F16, F32, close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ptq():
    import __graft_entry__ as entry
    entry.build()
    import paper_2412_20386_b200 as p
    torch.cuda.set_device(0)
    yield p
    p.fp8_device_status()


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("M,K,N", [(1, 65536, 130), (16, 65536, 257), (17, 65535, 130), (2, 40, 1 << 20), ((1 << 20) + 3, 24, 8), (1 << 16, 1, 1), (150000, 200, 129)])
def test_the_ends_of_the_sizes(ptq, dtype, M, K, N):
    gen = torch.Generator(device="cuda").manual_seed(M + K)
    x = torch.randn(M, K, generator=gen, device="cuda").to(dtype)
    w, ws = ptq.fp8_quantize_weight(torch.randn(N, K, generator=gen, device="cuda") / K ** 0.5)
    b = torch.randn(N, generator=gen, device="cuda")
    y = ptq.fp8_linear(x, w, ws, b)
    a, sa = ptq.fp8_quantize(x)
    two = ptq.fp8_matmul(a, sa, w, ws, b, dtype=dtype)
    assert M <= 16 or torch.equal(y, two)
    a = a.float().double() * sa.double().repeat_interleave(128, 1)[:, :K]
    w = w.float().double() * ws.double().repeat_interleave(128, 1)[:, :K].repeat_interleave(128, 0)[:N]
    factor = 2.0 ** -21 + 2.0 ** -24 * (-(-K // 128))
    for m in range(0, M, 1 << 17):                           # a part of the rows at a time
        rows = slice(m, m + (1 << 17))
        want, scale = a[rows] @ w.t() + b.double(), a[rows].abs() @ w.abs().t() + b.double().abs()
        for got in (y, two):
            close(got[rows], want.cpu(), scale.cpu(), factor, "y")


def test_weights_that_are_not_finite_make_their_128_columns_nan(ptq):
    """In every form of the product."""
    w = torch.randn(600, 300, device="cuda")
    x = torch.randn(5000, 300, device="cuda", dtype=BF16)
    codes, scales = ptq.fp8_quantize_weight(w)
    for value in (float("nan"), float("inf")):
        bad = w.clone()
        bad[130, 257] = value
        c, s = ptq.fp8_quantize_weight(bad)
        for M in (1, 16, 17, 60, 300, 5000):
            want, got = ptq.fp8_linear(x[:M], codes, scales), ptq.fp8_linear(x[:M], c, s)
            assert torch.isnan(got[:, 128:256]).all() and torch.equal(got[:, :128], want[:, :128]) and torch.equal(got[:, 256:], want[:, 256:])
