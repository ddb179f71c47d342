"""Calls with more heads than the GPU has SMs, where the forward pass shares its work otherwise, and cut sequences of heads that are wider than a CTA's columns."""
import pytest
import torch

from block_ref import BF16, F16, F32
from test_gpu_heads import check, make, ptq                  # noqa: F401 (ptq: a fixture)

pytestmark = pytest.mark.gpu

SHAPES = [
    # B, L, H, P, N, more
    (2, 70, 150, 8, 64, dict(state=True)),
    (1, 130, 160, 8, 128, dict(G=4)),
    (2, 66, 80, 72, 16, dict(state=True, odd=1)),            # two tiles of columns
    (3, 100, 110, 5, 100, dict(lengths=[100, 33, 0], state=True, odd=2)),
    (1, 197, 170, 16, 48, dict(state=True, bias=False)),
    (1, 65, 600, 8, 16, dict(G=2, state=True)),
]


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:5])))
def test_more_heads_than_the_gpu_has_sms(ptq, shape, dtype):             # noqa: F811
    B, L, H, P, N, more = shape
    check(ptq, make(21, dtype, B, L, H, P, N, **more), reverse=L % 2 == 0)


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("P,N,more", [(72, 16, dict(state=True)), (130, 24, dict(lengths=[1400, 300], state=True, odd=1)), (65, 8, {})], ids=["two", "three", "odd"])
def test_cut_sequences_of_wide_heads(ptq, dtype, P, N, more):           # noqa: F811
    check(ptq, make(22, dtype, 2, 1400, 1, P, N, decay=0.5, **more))
