"""A product's wait that runs out, without a GPU fault: a barrier expects an arrival that
does not come.  The outputs concerned are NaN, the others right, and the context stays
usable."""
import os
import re

import numpy as np
import pytest
import torch

from kv_case import bits, tensor
from paper_2608_23805_gb300 import api
from paper_2608_23805_gb300 import native as N

SHORT = 2_000_000  # clock64 cycles, about a millisecond


def stalled(lin, x, where, dtype):
    api.Q4Linear.set_wait_cycles(SHORT)
    api.Q4Linear.inject_stall(where)
    try:
        return lin(x, dtype=dtype)
    finally:
        api.Q4Linear.set_wait_cycles(0)


def product(rows, n_in, n_out, group):
    rng = np.random.default_rng([rows, n_in, n_out])
    codes = rng.integers(0, 256, (n_out, n_in // 2), dtype=np.uint8)
    scales = rng.uniform(0.01, 0.02, (n_out, n_in // group)).astype(np.float16)
    return api.Q4Linear(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()), tensor(bits(rng.standard_normal((rows, n_in))))


@pytest.mark.gpu
@pytest.mark.parametrize("where", [N.MSI_Q4_STALL_CODES, N.MSI_Q4_STALL_ROWS])
@pytest.mark.parametrize("rows,n_in,n_out,group", [(1, 32, 5, 32), (3, 2048, 100, 64), (8, 8192, 2000, 128), (16, 4096, 333, 32), (40, 512, 500, 64),
                                                   (8, 1024, 20000, 32)])
def test_tiles_by_themselves(rows, n_in, n_out, group, where):
    """The first tile's outputs, of the first rows, whatever its other warps have."""
    lin, x = product(rows, n_in, n_out, group)
    for dtype in (torch.bfloat16, torch.float32):
        want = lin(x, dtype=dtype)
        got = stalled(lin, x, where, dtype)
        lost = torch.zeros_like(got, dtype=torch.bool)
        lost[:8 if rows <= 8 else 16 if rows <= 16 else 32, :16] = True
        assert torch.equal(got.isnan(), lost) and torch.equal(got[~lost], want[~lost])
        assert torch.equal(lin(x, dtype=dtype), want)  # the request was for one call


@pytest.mark.gpu
@pytest.mark.parametrize("where", [N.MSI_Q4_STALL_CODES, N.MSI_Q4_STALL_ROWS])
@pytest.mark.parametrize("rows,n_in,n_out,group", [(9, 512, 15001, 128), (16, 2048, 15001, 32), (13, 4096, 30000, 64), (16, 1280, 20000, 32),
                                                   (50, 2048, 15001, 64), (33, 768, 16000, 128)])
def test_rows_shared_by_the_warps_of_a_cta(rows, n_in, n_out, group, where):
    """A warp that gives up frees no slot: the others of its part give up in turn, and
    where they had all they needed, their outputs are right."""
    lin, x = product(rows, n_in, n_out, group)
    want = lin(x)
    got = stalled(lin, x, where, torch.bfloat16)
    nan = got.isnan()
    first = nan[:16 if rows <= 16 else 32]
    assert torch.equal(first, first[:1].expand_as(first)) and not nan[first.shape[0]:].any()
    lost = first[0].nonzero()[:, 0]
    assert lost.numel() % 16 == 0 and 16 <= lost.numel() <= 14 * 16 and int(lost[-1]) - int(lost[0]) + 1 == lost.numel()
    turns = -(-n_in // 256) // 2  # of the first part: two wait in the slots
    if where == N.MSI_Q4_STALL_ROWS or turns > 2:
        assert int(lost[0]) == 0 and lost.numel() > 16
    else:
        assert lost.numel() == 16 and int(lost[0]) > 0
    assert torch.equal(got[~nan], want[~nan])
    assert torch.equal(lin(x), want)


@pytest.mark.gpu
def test_a_stall_taken_back():
    lin, x = product(4, 512, 64, 32)
    want = lin(x)
    api.Q4Linear.inject_stall(N.MSI_Q4_STALL_CODES)
    api.Q4Linear.inject_stall(0)
    assert torch.equal(lin(x), want)


def test_refusals_and_constants():
    for bad in (-1, 3):
        assert N.lib().msi_q4_inject_stall(bad) == N.MSI_ERR_INVALID_ARG
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "msi.h")) as f:
        text = f.read()
    for name in ("MSI_Q4_STALL_CODES", "MSI_Q4_STALL_ROWS"):
        assert int(re.search(name + r" = (\d)", text).group(1)) == getattr(N, name)
