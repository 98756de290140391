"""Decode-form attention over the 8-bit cache with more query rows of a head than
one group holds: groups of rows of a sequence are worked on apart."""
import numpy as np
import pytest
import torch

from kv_case import KvCase, ints, tensor
from paper_2608_23805_gb300 import native as N

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,fmt", [(64, N.MSI_KV_E4M3), (128, N.MSI_KV_Q8), (256, N.MSI_KV_Q8), (256, N.MSI_KV_E4M3)])
@pytest.mark.parametrize("G,rows", [(8, 3), (8, 4), (1, 17), (5, 6), (32, 1)])
@pytest.mark.parametrize("softcap,window", [(0.0, 0), (4.0, 25)])
def test_groups(D, fmt, G, rows, softcap, window):
    c = KvCase(D=D, fmt=fmt, K=2, P=16, max_blocks=64, n_blocks=160, seed=G * rows)
    c.append([0, 1, 2, 3], [700, 33, 5, 150])
    # a whole sequence of new rows, some of them, one, and a sequence that held fewer tokens than rows
    c.attend([0, 1, 2, 3], [rows, 1, rows, max(1, rows - 1)], 2 * G, softcap=softcap, window=window)


@pytest.mark.parametrize("D", [128, 256])
@pytest.mark.parametrize("n", [1, 4])
def test_groups_observed(D, n):
    c = KvCase(D=D, K=3, P=32, n_seqs=4, max_blocks=40, n_blocks=120, seed=n)
    c.append(list(range(n)), [900, 31, 640, 1][:n])
    c.attend(list(range(n)), [5, 2, 1, 1][:n], 15, observe=True)
    w = c.cache.weight.cpu().numpy().astype(np.float64)
    for s in range(n):
        ids = c.model.table[s]
        # sums of up to 25 rows' weights in fp32: each weight off by 2^-11 and the scores' error
        np.testing.assert_allclose(w[ids], c.model.weight[ids], rtol=2.0 ** -9, atol=1e-4)


def test_groups_do_not_depend_on_the_others():
    """A head's first 16 rows have the same answer whether 16 more stand beside
    them, where the runs are cut alike (one CTA's worth of tokens)."""
    c = KvCase(D=128, K=1, P=16, n_seqs=1, max_blocks=8, n_blocks=8, seed=3)
    c.append([0], [40])
    q = c.rows(4, 8)
    both = c.cache.attention(tensor(q), ints([0, 4]), 4)[0].float()
    again = c.cache.attention(tensor(q), ints([0, 4]), 4)[0].float()
    assert torch.equal(both, again)
    # rows 2, 3 of four are the last two tokens of the same sequence
    two = c.cache.attention(tensor(q[2:]), ints([0, 2]), 2)[0].float()
    assert float((both[2:] - two).abs().max()) <= 2.0 ** -7 * float(two.abs().max())


def test_chunk_of_many_sequences():
    """Chunk form with more items than a pass of its plan, and CTAs with parts of
    many of them."""
    c = KvCase(n_seqs=300, K=4, D=64, P=16, n_blocks=2100, max_blocks=8)
    order = c.rng.permutation(300).tolist()
    c.append(order, [80] * 300)
    c.attend(order, [65 + i % 2 for i in range(300)], 4)


@pytest.mark.parametrize("D,most", [(64, 64), (128, 64), (256, 48)])
def test_the_largest_decode_call_and_the_next(D, most):
    for rows in (most, most + 1):
        c = KvCase(D=D, K=1, P=32, seed=rows)
        c.append([0, 1], [333, rows])
        c.attend([0, 1], [rows, 1], 1, observe=rows == most)
        if rows > most:
            with pytest.raises(N.MsiError) as e:
                c.cache.attention(tensor(c.rows(rows, 1)), ints([0, rows]), rows, observe=True)
            assert e.value.status == N.MSI_ERR_UNSUPPORTED
