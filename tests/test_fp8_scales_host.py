"""Which layouts of scales fp8_quantize takes: each scale in a place of its own.  Checked on the host, so it needs no GPU."""
import ctypes
import itertools

import pytest
import torch

from test_heads_fp8_host import ARCH, CUDA, P, SHAPE, i64, inp, lib, vp          # noqa: F401 (lib: a fixture)


def quantize(lib, rows, blocks, row, block):                 # noqa: F811
    cols = 128 * (blocks - 1) + 1
    return lib.ptq_fp8_quantize(ctypes.byref(inp(rows=rows, cols=cols, x_pitch=cols)), vp(P), i64(cols + 15 & ~15), vp(P), (i64 * 2)(row, block), None)


def test_places_that_coincide_are_refused(lib):              # noqa: F811
    """All pitches up to 9 of up to 5 rows and blocks, against a list of the places."""
    if torch.cuda.is_available():
        pytest.skip("a call that is not refused would run")
    for rows, blocks, row, block in itertools.product(range(1, 6), range(1, 6), range(10), range(10)):
        places = [m * row + b * block for m in range(rows) for b in range(blocks)]
        got = quantize(lib, rows, blocks, row, block)
        assert got in (ARCH, CUDA) if len(set(places)) == len(places) else got == SHAPE, (rows, blocks, row, block)


def test_large_layouts(lib):                                 # noqa: F811
    """Products of pitches and counts beyond 64 bits."""
    if torch.cuda.is_available():
        pytest.skip("a call that is not refused would run")
    far = (1 << 62) + 1
    refused = [(5, 5, 0, 0), (1 << 30, 512, 1, 1), (1 << 30, 512, 1, (1 << 30) - 1), (1 << 30, 512, 511, 1), (3, 3, far, far), (1 << 30, 512, 1 << 40, 1 << 41)]
    for case in refused:
        assert quantize(lib, *case) == SHAPE, case
    for case in [(1 << 30, 512, 1, 1 << 30), (1 << 30, 512, 512, 1), (3, 3, far, 1), (1 << 30, 512, 1 << 40, (1 << 60) + (1 << 20))]:
        assert quantize(lib, *case) in (ARCH, CUDA), case
