"""A pool of more than 4 GB of codes: blocks at its far end, where offsets pass 32 bits."""
import pytest
import torch

from kv_case import KvCase

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,P,K,n_blocks", [(128, 32, 2, 600_000), (256, 16, 1, 1_200_000)])
def test_blocks_past_four_gigabytes(D, P, K, n_blocks):
    assert n_blocks * K * P * D > 2 ** 32
    c = KvCase(n_seqs=2, max_blocks=40, n_blocks=n_blocks, D=D, P=P, K=K)
    c.cache.free_ids.copy_(torch.arange(n_blocks, dtype=torch.int32))  # the last block is taken first
    c.model.free = list(range(n_blocks))
    c.append([1, 0], [333, 150])
    c.check_values()
    c.attend([0, 1], [1, 2], 4 * K, observe=True)  # decode form
    c.attend([0, 1], [150, 200], 4 * K)            # chunk form
    c.cache.evict(2, 5, 1, 1)
    c.model.evict([0, 1], 5, 1, 1)
    c.append([0, 1], [3, 40])
    assert c.cache.seq_state[:, 0].tolist() == [c.model.held(s) for s in range(2)]
    assert c.cache.status() == 0
    del c
    torch.cuda.empty_cache()
