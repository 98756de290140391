"""What pins the plain model of the 8-bit key-value cache (oracle/kv.py): torch's
e4m3 cast, hand-worked blocks, scipy's softmax, and a small hand-worked history."""
import numpy as np
import pytest
import torch
from scipy.special import logsumexp, softmax

from oracle import kv as M
from oracle.moe import bf16_to_f64


def bf16(x):
    return torch.tensor(np.asarray(x, np.float32)).bfloat16().view(torch.int16).numpy().view(np.uint16)


def test_e4m3_is_torchs_cast():
    grid = torch.arange(0, 0x7F, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert grid[-1] == 448.0
    ties = (grid[1:] + grid[:-1]) / 2
    x = np.concatenate([grid, ties, np.nextafter(ties, np.float32(0)), np.nextafter(ties, np.float32(1e9))])
    x = np.concatenate([x, -x]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(M.round_e4m3(x), want)
    assert M.round_e4m3(np.float32([500, -1e6])).tolist() == [448.0, -448.0]


def test_q8_block_by_hand():
    rows = np.zeros((16, 2, 64), np.float32)
    rows[0, 0, :3] = [127, -127, 2.5]  # a = 127: codes are the numbers rounded to even
    rows[5, 0, 0] = -63.5
    code, scale = M.round_block(rows, M.Q8)
    assert code[0, 0, :3].tolist() == [127, -127, 2] and code[5, 0, 0] == -64
    assert scale[0] == np.float32(127) * np.float32(1 / np.float32(127))
    assert (code[:, 1] == 0).all() and 0 < scale[1] < 1e-21  # an empty head: a = 1e-20


@pytest.mark.parametrize("fmt,top", [(M.Q8, 127.0), (M.E4M3, 448.0)])
def test_block_is_near_its_rows(fmt, top):
    rows = np.random.default_rng(0).standard_normal((32, 3, 64)).astype(np.float32)
    code, scale = M.round_block(rows, fmt)
    assert np.abs(code).max() == top
    # half a step of the format at each number
    step = 1.0 if fmt == M.Q8 else 2.0 ** (np.floor(np.log2(np.maximum(np.abs(code), 2.0 ** -6))) - 3)
    err = np.abs(code * scale.astype(np.float64)[None, :, None] - rows)
    assert (err <= 0.5001 * step * scale[None, :, None] + 1e-6 * np.abs(rows)).all()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_block_that_is_not_finite(bad):
    rows = np.ones((16, 2, 64), np.float32)
    rows[3, 1, 7] = bad
    _, scale = M.round_block(rows, M.Q8)
    assert np.isfinite(scale[0]) and np.isnan(scale[1])


def filled(tokens, K=2, D=64, P=16, seed=0):
    m = M.KvModel(1, 32, 32, K, D, P, M.Q8)
    rng = np.random.default_rng(seed)
    k, v = bf16(rng.standard_normal((tokens, K, D))), bf16(rng.standard_normal((tokens, K, D)))
    assert m.append([0], [0, tokens], k, v)
    return m, rng, k, v


@pytest.mark.parametrize("softcap,window", [(0.0, 0), (3.0, 0), (0.0, 7), (2.0, 1)])
def test_attention_is_a_masked_softmax(softcap, window):
    m, rng, _, _ = filled(45)
    q = rng.standard_normal((6, 4, 64))
    got = m.attention(0, q, 0.125, softcap, window)
    k, v = m.values(0)
    for i in range(6):
        at = 45 - 6 + i
        sees = np.arange(45) <= at
        if window:
            sees &= np.arange(45) > at - window
        for h in range(4):
            s = k[:, h // 2] @ q[i, h] * 0.125
            s = softcap * np.tanh(s / softcap) if softcap else s
            s = np.where(sees, s, -np.inf)
            np.testing.assert_allclose(got["out"][i, h], softmax(s) @ v[:, h // 2], atol=1e-13)
            np.testing.assert_allclose(got["weights"][h, i], softmax(s), atol=1e-14)
            np.testing.assert_allclose(got["lse"][i, h], logsumexp(s), atol=1e-12)


def test_rows_before_the_first_token_see_nothing():
    m, rng, _, _ = filled(3)
    got = m.attention(0, rng.standard_normal((5, 2, 64)), 0.125)
    assert np.isneginf(got["lse"][:2]).all() and (got["out"][:2] == 0).all()
    assert np.isfinite(got["lse"][2:]).all()


def test_values_do_not_depend_on_the_pieces():
    m, _, k, v = filled(45)
    other = M.KvModel(1, 32, 32, 2, 64, 16, M.Q8)
    for a, b in [(0, 1), (1, 20), (20, 45)]:
        assert other.append([0], [0, b - a], k[a:b], v[a:b])
    for x, y in zip(m.values(0), other.values(0)):
        np.testing.assert_array_equal(x, y)
    err = np.abs(m.values(0)[0] - bf16_to_f64(k)).max()
    assert 0 < err <= np.abs(bf16_to_f64(k)).max() / 127 / 2 * 1.001


def test_history_by_hand():
    m = M.KvModel(2, 4, 6, 1, 64, 16, M.Q8)
    rows = bf16(np.random.default_rng(1).standard_normal((64, 1, 64)))
    assert m.append([0, 1], [0, 40, 50], rows[:50], rows[:50])  # 3 blocks, 1 block
    assert m.table == [[0, 1, 2], [3]] and m.free == [5, 4] and m.pos == [40, 10]
    assert not m.append([1], [0, 40], rows[:40], rows[:40])      # 4 blocks, 3 more than the one: 2 are free
    assert m.table == [[0, 1, 2], [3]] and m.held(1) == 10
    assert not m.append([0], [0, 25], rows[:25], rows[:25])      # 65 tokens: more than the table's 4 blocks
    m.weight[:] = [0.1, 0.3, 9, 9, 9, 9]
    m.evict([0, 1], keep=2, sinks=0, recent=1)                   # the lighter of blocks 0 and 1 goes
    assert m.table[0] == [1, 2] and m.free == [5, 4, 0] and m.held(0) == 24 and m.pos[0] == 40
    assert m.append([0], [0, 9], rows[:9], rows[:9], start=[23])  # the last token again, then 8 more
    assert m.table[0] == [1, 2] and m.held(0) == 32 and m.pos[0] == 48
    assert m.append([0], [0, 1], rows[:1], rows[:1])
    assert m.table[0] == [1, 2, 0] and m.weight[0] == 0.0
    m.release([1])
    assert m.table[1] == [] and m.free == [5, 4, 3] and m.pos[1] == 0


def test_evict_ties_keep_the_earlier_block():
    m, _, _, _ = filled(6 * 16)
    m.weight[:6] = [5, 1, 1, 1, 7, 0]
    m.evict([0], keep=4, sinks=1, recent=1)
    assert m.table[0] == [0, 1, 4, 5]
