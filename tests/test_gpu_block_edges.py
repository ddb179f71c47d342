"""Calls of the operators between a block's linears at the edges of what their documents allow, against 64 bits."""
import itertools

import pytest
import torch

import block_ref as ref
from test_gpu_block_norm import make as make_norm
from test_gpu_block_norm_stream import check as check_norm

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
