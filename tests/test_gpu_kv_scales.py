"""Blocks whose value scales lie far apart."""
import numpy as np
import pytest

from kv_case import KvCase, bits, check_rows, ints, tensor
from oracle.moe import bf16_to_f64
from paper_2608_23805_gb300 import native as N

pytestmark = pytest.mark.gpu
FORMATS = [N.MSI_KV_Q8, N.MSI_KV_E4M3]
# the least scale is 1e-20 / 448, so the first set spans 2^89
SETS = {"small": [0.0, 1e-30, 1e-19, 1e-3, 1.0, 30.0, 1e3, 1e6], "middle": [1.0, 1e4, 1e8, 1e12, 1e17, 1e21, 1e25, 3.0],
        "large": [2e11, 1e13, 1e18, 1e23, 1e28, 1e33, 1e36, 2e37]}


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("scales", sorted(SETS))
@pytest.mark.parametrize("order", ["up", "down", "mixed", "ends"])
@pytest.mark.parametrize("rows,D", [(1, 64), (1, 128), (2, 256), (90, 64), (90, 128), (90, 256)])
def test_value_scales_far_apart(D, rows, order, scales, fmt):
    """Within 2^90: every token counts in the sum by its score alone, and so in lse and in the outputs."""
    P, s = 16, SETS[scales]
    c = KvCase(n_seqs=1, K=1, D=D, P=P, fmt=fmt, seed=7)
    s = {"up": s, "down": s[::-1], "mixed": [s[i] for i in (5, 0, 7, 3, 1, 6, 2, 4)], "ends": [s[7], s[0]] * 4}[order]
    v = c.rng.standard_normal((len(s) * P, 1, D)).clip(-4, 4) * np.repeat(s, P)[:, None, None]
    c.append([0], [len(s) * P], v=bits(v))
    q = c.rows(rows, 4)
    observe = rows < 8
    c.attend([0], [rows], 4, q=q, observe=observe)
    assert c.cache.status() == N.MSI_OK
    if observe:
        # a weight is off by twice its score's error, and so is its row's sum
        ds = (2 * D + 10) * 2.0 ** -24 * (c.model.attention(0, bf16_to_f64(q), D ** -0.5)["size"].max() + 1.0) + 2.0 ** -20
        np.testing.assert_allclose(c.cache.weight.cpu().numpy(), c.model.weight, rtol=4 * ds, atol=1e-9)


@pytest.mark.parametrize("rows", [1, 90])
def test_in_parts(rows):
    """The same over parts of a long sequence that several CTAs take."""
    n = 3000
    c = KvCase(n_seqs=1, K=1, D=64, P=16, max_blocks=200, n_blocks=200, seed=9)
    v = c.rng.standard_normal((n, 1, 64)).clip(-4, 4) * np.where(np.arange(n) < n // 2, 0.0, 1e6)[:, None, None]
    c.append([0], [n], v=bits(v))
    c.attend([0], [rows], 4)
    c.append([0], [n // 4], start=[0])
    c.attend([0], [rows], 4)


@pytest.mark.parametrize("seqs,rows", [(1, 1), (48, 1), (1, 90), (3, 90)])
def test_too_far_apart(seqs, rows):
    """Beyond: an answer that holds, or none and the error."""
    c = KvCase(n_seqs=seqs, K=1, D=64, P=16, max_blocks=64, n_blocks=64 * seqs, seed=seqs)
    n = 1000
    v = c.rng.standard_normal((n * seqs, 1, 64)).clip(-4, 4) * 1e30
    v.reshape(seqs, n, 64)[:, np.arange(n) // 16 % 3 == 0] = 0.0  # whole blocks of zeros among the others
    c.append(list(range(seqs)), [n] * seqs, v=bits(v))
    q = c.rows(seqs * rows, 4)
    cu = ints(range(0, seqs * rows + 1, rows))
    out, lse = c.cache.attention(tensor(q), cu, rows)
    status = c.cache.status()
    assert status in (N.MSI_OK, N.MSI_ERR_UNSUPPORTED)
    if seqs > 1 or rows > 1:
        assert status == N.MSI_ERR_UNSUPPORTED
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for s in range(seqs):
        at = slice(s * rows, (s + 1) * rows)
        if status != N.MSI_OK and rows > 1:
            assert np.isnan(out[at]).all() and np.isnan(lse[at]).all()
        elif not np.isnan(lse[at]).all():
            check_rows(out[at], lse[at], c.model.attention(s, bf16_to_f64(q[at]), 0.125), 64, 0.0)
    c.check_state()
