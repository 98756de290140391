"""Query rows whose memory overlaps."""
import pytest
import torch

from kv_case import KvCase, ints, tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [2, 3, 200])
@pytest.mark.parametrize("stride", [0, 128, 256])
def test_overlapping_query_rows(rows, stride):
    """Rows that share memory (a stride below a row's length): the output that
    the call makes is packed, and each row's answer is its own."""
    c = KvCase(n_seqs=1, K=1, D=128, P=16, seed=stride)
    c.append([0], [300])
    base = tensor(c.rows(2 * rows + 4, 1)).reshape(-1)
    q = base.as_strided((rows, 3, 128), (stride, 128, 1))
    out, lse = c.cache.attention(q, ints([0, rows]), rows)
    ref, ref_lse = c.cache.attention(q.contiguous(), ints([0, rows]), rows)
    assert out.is_contiguous() and torch.equal(out, ref) and torch.equal(lse, ref_lse)
