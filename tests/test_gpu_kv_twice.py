"""Sequences named twice in a call."""
import pytest
import torch

from kv_case import KvCase, ints, tensor
from paper_2608_23805_gb300 import native as N

pytestmark = pytest.mark.gpu


def test_sequences_named_twice():
    """Observed attention refuses them (two entries would add to one block's
    weight); without observation each entry has its answer."""
    c = KvCase(n_seqs=3, K=1, D=64, P=16)
    c.append([0, 1], [50, 30])
    q = tensor(c.rows(3, 4))
    cu, seqs = ints([0, 1, 2, 3]), ints([0, 1, 0])
    out, lse = c.cache.attention(q, cu, 1, seqs=seqs)
    for b, s in enumerate([0, 1, 0]):
        one, one_lse = c.cache.attention(q[b:b + 1], ints([0, 1]), 1, seqs=ints([s]))
        assert (out[b:b + 1].float() - one.float()).abs().max() <= 2.0 ** -7 * one.float().abs().max()
        assert (lse[b:b + 1] - one_lse).abs().max() < 1e-5
    assert c.cache.status() == 0
    before = c.cache.weight.clone()
    out, lse = c.cache.attention(q, cu, 1, seqs=seqs, observe=True)
    assert c.cache.status() == N.MSI_ERR_INVALID_ARG
    assert out.isnan().all() and lse.isnan().all() and torch.equal(c.cache.weight, before)
    c.attend([0, 1], [1, 1], 4, observe=True)
