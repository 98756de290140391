"""A wait of the chunk form's kernel that runs out, without a GPU fault: one warp
waits on a barrier that nothing arrives at.  Every warp of both CTAs of its pair
stops, TMEM is freed, no row of the call can be read as an answer, and the cache
and the context stay usable."""
import os
import re

import pytest
import torch

from kv_case import KvCase, ints, tensor
from paper_2608_23805_gb300 import native as N

SHORT = 2_000_000  # clock64 cycles, about a millisecond
WHERE = [N.MSI_KV_STALL_SOFTMAX, N.MSI_KV_STALL_MMA, N.MSI_KV_STALL_CONVERSION]


@pytest.mark.gpu
@pytest.mark.parametrize("where", WHERE)
@pytest.mark.parametrize("D,fmt", [(64, N.MSI_KV_Q8), (128, N.MSI_KV_Q8), (256, N.MSI_KV_E4M3)])
@pytest.mark.parametrize("softcap", [0.0, 20.0])
def test_expired_wait_fails_closed_then_recovers(D, fmt, softcap, where):
    """Items that one CTA pair has whole are among the call's: nothing joins those."""
    n = 90
    c = KvCase(n_seqs=n, K=2, D=D, P=16, fmt=fmt, max_blocks=32, n_blocks=n * 10)
    c.append(list(range(n)), [60 + i for i in range(n)])
    rows = 60 * n
    cu = ints(range(0, rows + 1, 60))
    q = tensor(c.rows(rows, 4))
    want, want_lse = c.cache.attention(q, cu, 60, softcap=softcap)
    out, lse = torch.full_like(want, 7.0), torch.full_like(want_lse, 7.0)
    c.cache.set_wait_cycles(SHORT)
    c.cache.inject_stall(where)
    c.cache.attention(q, cu, 60, softcap=softcap, out=out, lse=lse)
    assert c.cache.status() == N.MSI_ERR_TIMEOUT
    assert out.isnan().all() and lse.isnan().all()
    c.cache.set_wait_cycles(0)
    c.cache.attention(q, cu, 60, softcap=softcap, out=out, lse=lse)  # the request was for one call
    assert c.cache.status() == N.MSI_OK
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    c.check_state()


@pytest.mark.gpu
def test_stall_is_of_chunk_calls_and_refused_otherwise():
    c = KvCase(n_seqs=1, K=1, D=64, P=16)
    c.append([0], [100])
    c.cache.inject_stall(N.MSI_KV_STALL_MMA)
    c.attend([0], [1], 4)  # decode form: not touched
    assert c.cache.status() == N.MSI_OK
    c.cache.inject_stall(0)
    c.attend([0], [90], 4)
    assert c.cache.status() == N.MSI_OK
    for bad in (-1, 4):
        with pytest.raises(N.MsiError) as e:
            c.cache.inject_stall(bad)
        assert e.value.status == N.MSI_ERR_INVALID_ARG


def test_constants():
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "msi.h")) as f:
        text = f.read()
    for name in ("MSI_KV_STALL_SOFTMAX", "MSI_KV_STALL_MMA", "MSI_KV_STALL_CONVERSION"):
        assert int(re.search(name + r" = (\d)", text).group(1)) == getattr(N, name)
