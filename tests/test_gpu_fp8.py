"""fp8_quantize, fp8_quantize_weight, fp8_matmul and fp8_linear against 64 bits.

Tolerances.  Scales: a maximum and one division, 2^-24 (and as much for the reference's cast).  Codes: none, the definition's two binary32 roundings (448 / top, and
x times that) are made here too.  Products: codes are exact operands, 128 products sum
in binary32 on the tensor cores (four partial sums, cut off: 4 x 2^-23 of the magnitudes), each times two scales (2^-23) and added to at most 8 parts of up to
64 blocks (2^-24 each): 2^-21 + 2^-24 ceil(K / 128) of the magnitudes."""
import pytest
import torch

from block_ref import BF16, F16, F32, close

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
TYPES = pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])


@pytest.fixture(scope="module")
def ptq():
    import __graft_entry__ as entry
    entry.build()
    import paper_2412_20386_b200 as p
    torch.cuda.set_device(0)
    yield p
    p.fp8_device_status()                                    # no kernel gave up a wait


def values():
    """All finite magnitudes of e4m3, from its definition."""
    return torch.tensor(sorted({m * 2.0 ** -9 for m in range(8)} | {(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)}),
                        dtype=torch.float64)


def check_codes(codes, x, top):
    """codes are nearest to x (448 / top), of two as near the even one; x and top binary32 (in 64 bits)."""
    v = values()
    got = codes.float().double().cpu().flatten()
    x = (x.float() * torch.full_like(top, 448.0, dtype=torch.float32).div(top.float())).double().flatten()      # (448.0 / t would be a reciprocal, times 448)
    i = torch.searchsorted(v, x.abs().clamp(max=448.0)).clamp(1, len(v) - 1)
    down, up = x.abs().clamp(max=448.0) - v[i - 1], v[i] - x.abs().clamp(max=448.0)
    lower = (down < up) | ((down == up) & ((i - 1) % 2 == 0))
    assert torch.equal(got, torch.sign(x) * torch.where(lower, v[i - 1], v[i]))


def blocks(x):
    """[M, K] -> [M, blocks, 128], zeros behind the end, 64 bits."""
    x = x.double().cpu()
    return torch.nn.functional.pad(x, (0, -x.shape[1] % 128)).unflatten(1, (-1, 128))


@TYPES
@pytest.mark.parametrize("M,K,odd", [(1, 1, 0), (1, 768, 0), (17, 129, 0), (33, 127, 1), (16, 128, 8), (50, 1000, 4), (3, 640, 0), (200, 384, 1), (5, 4104, 0)])
def test_quantize(ptq, dtype, M, K, odd):
    gen = torch.Generator().manual_seed(K)
    x = (torch.randn(M, K + odd, generator=gen) * torch.exp(2 * torch.randn(M, K + odd, generator=gen))).to(dtype).cuda()[:, odd:]
    codes, scales = ptq.fp8_quantize(x)
    assert codes.dtype == E4M3 and codes.shape == (M, K) and codes.stride(0) % 16 == 0 and scales.shape == (M, -(-K // 128))
    top = blocks(x).abs().amax(-1).clamp(min=2.0 ** -100)
    assert ((scales.double().cpu() - top / 448).abs() <= 2.0 ** -23 * top / 448).all()
    check_codes(codes, x.double().cpu(), top.repeat_interleave(128, 1)[:, :K])
    mine = torch.zeros(M, -(-K // 16) * 16 + 16, dtype=torch.uint8, device="cuda").view(E4M3)[:, :K]
    other = torch.full((M, 2 * scales.shape[1]), 5.0, device="cuda")
    got = ptq.fp8_quantize(x, codes=mine, scales=other[:, ::2])                         # the caller's own, any distances apart
    assert got[0] is not codes and torch.equal(mine.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(other[:, ::2], scales)
    assert (other[:, 1::2] == 5).all() and (mine.as_strided((M, mine.stride(0) - K), (mine.stride(0), 1), K).view(torch.uint8) == 0).all()
    three = ptq.fp8_quantize(x[None].expand(2, M, K).contiguous())                      # leading dimensions
    assert three[1].shape == (2, M, scales.shape[1]) and torch.equal(three[1][1], scales)


@TYPES
def test_quantize_values_at_the_borders(ptq, dtype):
    x = torch.zeros(6, 256, dtype=dtype)
    x[1, :128] = torch.finfo(dtype).tiny                     # small, of one size
    x[2, 3], x[2, 4] = float("inf"), 1.0
    x[3, 200] = float("nan")
    x[4, :128] = torch.linspace(-1, 1, 128).to(dtype)
    x[5, 0] = -torch.finfo(dtype).max
    codes, scales = ptq.fp8_quantize(x.cuda())
    c, s = codes.float().cpu(), scales.cpu()
    assert (c[0] == 0).all() and (s[0] > 0).all() and torch.isfinite(s[0]).all()
    assert (c[1, 128:] == 0).all() and torch.isfinite(c[1]).all()
    assert torch.isnan(c[2, 3]) and (c[2, 4:] == 0).all() and torch.isinf(s[2, 0]) and torch.isfinite(s[2, 1])
    assert torch.isnan(c[3, 128:]).all() and torch.isnan(s[3, 1]) and (c[3, :128] == 0).all()
    assert c[4, 0] == -448 and c[4, 127] == 448 and c[5, 0] == -448
    w, ws = ptq.fp8_quantize_weight(torch.randn(4, 256).to(dtype).cuda())
    y = ptq.fp8_linear(x.cuda(), w, ws).cpu()
    assert torch.isnan(y[2:4]).all() and torch.isfinite(y[[0, 1, 4]]).all() and (y[0] == 0).all()


@TYPES
@pytest.mark.parametrize("N,K", [(1, 1), (128, 128), (130, 257), (384, 768), (77, 1000)])
def test_quantize_weight(ptq, dtype, N, K):
    w = torch.randn(N, K + 3).to(dtype).cuda()[:, 3:]
    codes, scales = ptq.fp8_quantize_weight(w)
    pad = torch.nn.functional.pad(w.double().cpu(), (0, -K % 128, 0, -N % 128)).unflatten(1, (-1, 128)).unflatten(0, (-1, 128))
    top = pad.abs().amax((1, 3)).clamp(min=2.0 ** -100)
    assert scales.shape == top.shape and ((scales.double().cpu() - top / 448).abs() <= 2.0 ** -23 * top / 448).all()
    check_codes(codes, w.double().cpu(), top.repeat_interleave(128, 1)[:, :K].repeat_interleave(128, 0)[:N])


def operands(seed, M, K, N, bias=False):
    gen = torch.Generator().manual_seed(seed)
    a = (torch.randn(M, K, generator=gen) * 100).clamp(-448, 448).to(E4M3)
    w = (torch.randn(N, K, generator=gen) * 100).clamp(-448, 448).to(E4M3)
    pitch = -(-K // 16) * 16
    put = lambda v: torch.full((v.shape[0], pitch), 0x7f, dtype=torch.uint8).index_copy_(1, torch.arange(K), v.view(torch.uint8)).cuda().view(E4M3)[:, :K]
    kb, nb = -(-K // 128), -(-N // 128)
    sa, sw = torch.rand(M, kb, generator=gen) + 0.01, torch.rand(nb, kb, generator=gen) / 100 + 1e-4
    b = torch.randn(N, generator=gen).cuda() if bias else None
    return put(a), sa.cuda(), put(w), sw.cuda(), b


def product(a, sa, w, sw, b):
    K, N = a.shape[1], w.shape[0]
    a = a.float().double().cpu() * sa.double().cpu().repeat_interleave(128, 1)[:, :K]
    w = w.float().double().cpu() * sw.double().cpu().repeat_interleave(128, 1)[:, :K].repeat_interleave(128, 0)[:N]
    y, scale = a @ w.t(), a.abs() @ w.abs().t()
    return (y, scale) if b is None else (y + b.double().cpu(), scale + b.double().cpu().abs())


@TYPES
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 768, 384), (1, 5000, 128), (3, 129, 8), (16, 128, 127), (17, 1000, 130), (33, 127, 1000), (64, 384, 128),
                                   (65, 640, 257), (129, 4096, 64), (300, 1000, 1111), (1000, 16, 600), (2000, 384, 776), (5000, 512, 1040), (1, 65536, 40)])
def test_matmul(ptq, dtype, M, K, N):
    """Codes beyond K, up to the pitch, are NaN here: they are not read.  Sizes reach every form of the product and cuts into up to eight parts."""
    a, sa, w, sw, b = operands(M + K + N, M, K, N, bias=N % 2 == 0)
    want, scale = product(a, sa, w, sw, b)
    factor = 2.0 ** -21 + 2.0 ** -24 * (-(-K // 128))
    y = ptq.fp8_matmul(a, sa, w, sw, b, dtype=dtype)
    assert y.shape == (M, N) and y.dtype == dtype
    close(y, want, scale, factor, "y")
    assert torch.equal(ptq.fp8_matmul(a, sa.t().contiguous().t(), w, sw, b, dtype=dtype), y)            # the scales' order does not matter
    wide = torch.full((M, N + 11), 3.0, dtype=dtype, device="cuda")
    assert ptq.fp8_matmul(a, sa, w, sw, b, y=wide[:, 5:5 + N]).data_ptr() == wide[:, 5:].data_ptr()
    close(wide[:, 5:5 + N], want, scale, factor, "y in a slice")
    assert (wide[:, :5] == 3).all() and (wide[:, 5 + N:] == 3).all()


@TYPES
@pytest.mark.parametrize("M,K,N", [(1, 768, 384), (2, 130, 100), (16, 1000, 1111), (17, 1000, 1111), (7, 8192, 300), (64, 768, 384), (400, 257, 129), (3000, 384, 768)])
def test_linear_is_quantize_and_matmul(ptq, dtype, M, K, N):
    gen = torch.Generator().manual_seed(M)
    x = torch.randn(M, K, generator=gen).to(dtype).cuda()
    w, sw = ptq.fp8_quantize_weight(torch.randn(N, K, generator=gen).cuda())
    b = torch.randn(N, generator=gen).cuda()
    a, sa = ptq.fp8_quantize(x)
    y, two = ptq.fp8_linear(x, w, sw, b), ptq.fp8_matmul(a, sa, w, sw, b, dtype=dtype)
    if M > 16:
        assert torch.equal(y, two)
    want, scale = product(a, sa, w, sw, b)
    close(y, want, scale, 2.0 ** -21 + 2.0 ** -24 * (-(-K // 128)), "y")
    assert torch.equal(ptq.fp8_linear(x[None], w, sw, b)[0], y)
    odd = torch.zeros(M, K + 1, dtype=dtype, device="cuda")[:, 1:].copy_(x)             # rows that begin anywhere
    assert torch.equal(ptq.fp8_linear(odd, w, sw, b), y)


def test_rows_of_one_call_do_not_see_each_other(ptq):
    """A row's result is that of the row alone, whatever stands beside it: NaN, infinities, sizes 2^80 apart."""
    w, sw = ptq.fp8_quantize_weight(torch.randn(200, 300, device="cuda"))
    for M in (5, 40, 700):
        x = torch.randn(M, 300, device="cuda")
        want = ptq.fp8_linear(x, w, sw)
        x[0], x[1, 7], x[2] = float("nan"), float("inf"), x[2] * 2.0 ** 80
        got = ptq.fp8_linear(x, w, sw)
        assert torch.equal(got[3:], want[3:]) and torch.isnan(got[:2]).all() and torch.isfinite(got[2]).all()
