"""Appends that meet a block number out of range in the free list or in a table:
that block alone is skipped, everything else of the call is done and committed,
and what would read the block is NaN."""
import numpy as np
import pytest
import torch

from kv_case import KvCase, ints, tensor
from paper_2608_23805_gb300 import native as N

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [-7, 4000, 2 ** 31 - 1])
@pytest.mark.parametrize("n,rows", [(3, 40), (500, 70)])
def test_wrong_free_entry(n, rows, bad):
    c = KvCase(n_seqs=n, K=1, D=64, P=16, max_blocks=8, n_blocks=4000)
    at = 2  # the first sequence's third block
    c.cache.free_ids[4000 - 1 - at] = bad
    c.model.free[4000 - 1 - at] = bad
    c.model.weight = dict.fromkeys(c.model.free, 0.0)
    c.cache.table.fill_(1)  # what an entry that nobody writes would name: another sequence's block
    cu = np.arange(n + 1) * rows
    k, v = c.rows(cu[-1]), c.rows(cu[-1])
    c.cache.append(tensor(k), tensor(v), ints(cu))
    assert c.model.append(list(range(n)), cu, k, v)
    assert c.cache.status() == N.MSI_ERR_INVALID_ARG
    c.check_state()
    c.check_values(list(range(1, n)))
    k, v = c.cache.read(ints([0, rows]), rows)
    assert k[32:min(48, rows)].isnan().all() and not k[:32].isnan().any() and not k[48:].isnan().any()
    assert c.cache.status() == N.MSI_ERR_INVALID_ARG
    out, _ = c.cache.attention(tensor(c.rows(1, 4)), ints([0, 1]), 1)
    assert out.isnan().all() and c.cache.status() == N.MSI_ERR_INVALID_ARG
    c.attend([1, 2], [1, 1], 4)


@pytest.mark.parametrize("bad", [-1, 4000])
def test_wrong_table_entry_of_a_growing_block(bad):
    n = 500
    c = KvCase(n_seqs=n, K=1, D=64, P=16, max_blocks=8, n_blocks=4000)
    c.append(list(range(n)), [20] * n)
    c.cache.table[3, 1] = bad
    c.model.table[3][1] = bad
    c.model.weight = dict.fromkeys(c.model.free, 0.0)
    c.append(list(range(n)), [30] * n)
    assert c.cache.status() == N.MSI_ERR_INVALID_ARG
    c.check_state()
    c.check_values([s for s in range(n) if s != 3])
    k, _ = c.cache.read(ints([0, 50]), 50, seqs=ints([3]))
    assert k[16:32].isnan().all() and not k[:16].isnan().any() and not k[32:].isnan().any()
    assert c.cache.status() == N.MSI_ERR_INVALID_ARG
