"""Windows up to the largest number."""
import numpy as np
import pytest
import torch

from kv_case import KvCase, ints, tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 3, 2 ** 30, 4096])
@pytest.mark.parametrize("rows", [64, 300])
def test_windows_without_end(rows, window):
    """A window as long as what a sequence can hold, or longer, is none; more rows than tokens."""
    c = KvCase(n_seqs=2, K=1, D=64, P=16, max_blocks=64)
    c.append([0, 1], [3, 500])
    q = c.rows(2 * rows, 1)
    out, lse = c.cache.attention(tensor(q), ints([0, rows, 2 * rows]), rows)
    got, got_lse = c.cache.attention(tensor(q), ints([0, rows, 2 * rows]), rows, window=window)
    assert torch.equal(got, out) and torch.equal(got_lse, lse)
    assert bool((lse[rows - 3:rows] > -1e30).all()) and bool((lse[:rows - 3] == -np.inf).all())
    c.attend([0, 1], [rows, rows], 1, window=window, q=q)
