"""Caps far above every score, and near it."""
import pytest

from kv_case import KvCase, check_rows, ints, tensor
from oracle.moe import bf16_to_f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [1e-39, 2.0, 50.0, 64.0, 65.0, 1e3, 1e4, 1e6, 1e8, 1e30])
@pytest.mark.parametrize("rows,D", [(1, 64), (1, 128), (2, 256), (90, 64), (90, 128), (90, 256)])
def test_caps_of_every_size(D, rows, cap):
    """cap tanh(score / cap) to the score's own precision: the bound has no term of the cap."""
    c = KvCase(n_seqs=1, K=1, D=D, P=16, seed=5)
    c.append([0], [333])
    q = c.rows(rows, 4, 3.0)
    out, lse = c.cache.attention(tensor(q), ints([0, rows]), rows, softcap=cap)
    ref = c.model.attention(0, bf16_to_f64(q), D ** -0.5, cap)
    check_rows(out.double().cpu().numpy(), lse.double().cpu().numpy(), ref, D, 0.0)
