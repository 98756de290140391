"""Block weights that attention adds up, as closely as its arithmetic allows: they
are taken from the fp32 weights, before those are rounded for the products."""
import numpy as np
import pytest

from kv_case import KvCase
from oracle.moe import bf16_to_f64
from paper_2608_23805_gb300 import native as N

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,fmt", [(64, N.MSI_KV_E4M3), (128, N.MSI_KV_Q8), (256, N.MSI_KV_Q8)])
@pytest.mark.parametrize("G,counts", [(5, [5, 2, 1, 1]), (8, [1, 1, 1, 1]), (12, [4, 4, 4, 4])])
@pytest.mark.parametrize("softcap,window", [(0.0, 0), (20.0, 100)])
def test_weights(D, fmt, G, counts, softcap, window):
    c = KvCase(D=D, fmt=fmt, K=3, P=32, n_seqs=4, max_blocks=40, n_blocks=120, seed=G)
    c.append([0, 1, 2, 3], [900, 31, 640, 1])
    q = c.rows(sum(counts), 3 * G)
    c.attend([0, 1, 2, 3], counts, 3 * G, observe=True, q=q, softcap=softcap, window=window)
    # a score's error (kv_case) moves a weight and its row's sum by as much each; sums of up to
    # 16 rows, tokens and heads, exponents of up to 7 bits before the point, in fp32
    size = max(c.model.attention(s, bf16_to_f64(q[sum(counts[:s]):sum(counts[:s + 1])]), D ** -0.5)["size"].max() for s in range(4))
    ds = (2 * D + 10) * 2.0 ** -24 * (size + softcap + 1.0) + 2.0 ** -20
    np.testing.assert_allclose(c.cache.weight.cpu().numpy(), c.model.weight, rtol=4 * ds + 2.0 ** -16, atol=1e-6)
