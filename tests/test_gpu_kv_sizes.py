"""What the wrapper keeps of calls' shapes."""
import numpy as np
import pytest

from kv_case import KvCase, ints, tensor

pytestmark = pytest.mark.gpu


def test_sizes_of_workspaces_are_not_kept_without_end():
    c = KvCase(n_seqs=1, K=1, D=64, P=16)
    c.append([0], [900])
    for n in range(1, 700):
        c.cache.attention(tensor(np.zeros((n, 1, 64), np.uint16)), ints([0, n]), n)
    assert len(c.cache._need) <= 256 and c.cache.status() == 0
