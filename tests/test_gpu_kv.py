"""The 8-bit key-value cache against its plain model: what append, rollback,
eviction and release leave held, bit for bit; attention in decode form within
bounds derived from its roundings; refusals on the host and on the GPU."""
import ctypes

import numpy as np
import pytest
import torch

from kv_case import KvCase, bits, ints, tensor
from oracle.moe import bf16_to_f64
from paper_2608_23805_gb300 import api
from paper_2608_23805_gb300 import native as N

pytestmark = pytest.mark.gpu
FORMATS = [N.MSI_KV_Q8, N.MSI_KV_E4M3]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,P,K", [(64, 16, 1), (64, 128, 3), (128, 32, 2), (256, 16, 1), (256, 64, 2), (256, 128, 1)])
def test_append_in_pieces(D, P, K, fmt):
    """Ragged pieces, empty ones among them, in any sequence order."""
    c = KvCase(K=K, D=D, P=P, fmt=fmt, max_blocks=16, n_blocks=64)
    for seqs, counts in [([2, 0], [P + 3, 1]), ([0, 3, 2], [2, 0, P - 3]), ([1, 2], [3 * P, 2 * P + 5]), ([2], [1]),
                         ([3, 2, 1, 0], [7, P, 1, 5 * P - 1])]:
        assert c.append(seqs, counts)
        c.check_state()
        c.check_values()


def test_one_by_one_equals_at_once():
    a, b = KvCase(seed=1), KvCase(seed=1)
    k, v = a.rows(75), a.rows(75)
    a.append([0], [75], k=k, v=v)
    for i in range(75):
        b.append([0], [1], k=k[i:i + 1], v=v[i:i + 1])
    b.check_state()
    for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
        x, y = getattr(a.cache, name), getattr(b.cache, name)
        n = a.cache.table[0, :3].long()
        assert torch.equal(x[n], y[b.cache.table[0, :3].long()]), name


@pytest.mark.parametrize("P", [16, 32])
def test_rollback(P):
    """Rejected tokens taken back: within a block, across a block's boundary,
    to nothing, and to a boundary far back; freed blocks return."""
    c = KvCase(P=P, D=64, max_blocks=32, n_blocks=64)
    c.append([0, 1], [2 * P - 1, 3 * P])
    for start, n in [((2 * P - 1, 3 * P - 4), (4, 2)), ((2 * P, 2 * P + 1), (3, 0)), ((P + 2, 2 * P + 1), (P + 9, 1)),
                     ((P + 2, P + 1), (0, 1)), ((P, 0), (2 * P + 3, 5)), ((P, 3), (0, 0)), ((0, 3), (0, 5 * P))]:
        assert c.append([0, 1], list(n), start=list(start))
        c.check_state()
        c.check_values()
    # rows of an older block are gone: refused, nothing changes
    before = c.cache.seq_state.clone()
    c.cache.append(tensor(c.rows(1)), tensor(c.rows(1)), ints([0, 1]), seqs=ints([1]), start=ints([P + 1]))
    assert c.cache.status() == N.MSI_ERR_INVALID_ARG
    assert torch.equal(c.cache.seq_state, before)
    c.check_state()
    c.check_values()


def test_many_sequences():
    """More sequences than a CTA has threads."""
    c = KvCase(n_seqs=700, max_blocks=4, n_blocks=2000, D=64, K=1, P=16)
    order = c.rng.permutation(700)[:650].tolist()
    assert c.append(order, c.rng.integers(0, 40, 650).tolist())
    assert c.append(order[::-1], c.rng.integers(0, 20, 650).tolist())
    c.check_state()
    c.check_values()


def test_full_pool_and_full_table():
    c = KvCase(n_seqs=2, max_blocks=3, n_blocks=4, P=16, D=64)
    assert c.append([0, 1], [32, 20])
    for seqs, counts in [([0, 1], [1, 13]), ([0], [17])]:
        assert not c.append(seqs, counts)
        assert c.cache.status() == N.MSI_ERR_NOT_RESIDENT
        c.check_state()
        c.check_values()
    # until the word is read, attention answers NaN and append does nothing
    assert not c.append([0, 1], [1, 13])
    c.cache.append(tensor(c.rows(1)), tensor(c.rows(1)), ints([0, 1]), seqs=ints([1]))
    out, lse = c.cache.attention(tensor(c.rows(1, 4)), ints([0, 1]), 1, seqs=ints([1]))
    assert out.isnan().all() and lse.isnan().all()
    assert c.cache.status() == N.MSI_ERR_NOT_RESIDENT
    c.check_state()
    c.attend([1], [1], 4)


@pytest.mark.parametrize("fmt", FORMATS)
def test_extreme_values(fmt):
    """Zero blocks, the smallest and largest bf16 numbers, one large value among small ones."""
    c = KvCase(D=64, P=16, fmt=fmt, n_seqs=1)
    x = np.zeros((64, 2, 64), np.float32)
    x[16:32] = c.rng.standard_normal((16, 2, 64)) * 1e-38
    x[32:48] = c.rng.standard_normal((16, 2, 64)) * 1e37
    x[48:] = c.rng.standard_normal((16, 2, 64)) * 1e-3
    x[50, 1, 3] = -900.0
    c.append([0], [64], k=bits(x), v=bits(x[::-1]))
    c.check_state()
    c.check_values()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("bad", [np.inf, np.nan])
@pytest.mark.parametrize("where", ["k", "v"])
def test_not_finite(fmt, bad, where):
    """A block with an infinity or NaN: rows that see it are NaN, others are as without it."""
    c = KvCase(D=64, P=16, K=1, fmt=fmt, n_seqs=2)
    k, v = c.rows(40), c.rows(40)
    (k if where == "k" else v)[33, 0, 5] = bits([bad])[0]
    c.append([0], [40], k=k, v=v)
    c.append([1], [32], k=k[:32], v=v[:32])
    q = c.rows(10, 2)
    out, lse = c.cache.attention(tensor(q), ints([0, 10]), 10, seqs=ints([0]))
    ref, ref_lse = c.cache.attention(tensor(q[:2]), ints([0, 2]), 2, seqs=ints([1]))
    assert out[2:].isnan().all()           # tokens 32 .. 39
    assert torch.equal(out[:2], ref) and torch.equal(lse[:2], ref_lse)


LENGTHS = [1, 15, 16, 17, 100, 333]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("K,G", [(1, 1), (2, 8), (1, 7), (3, 3), (1, 16)])
def test_decode(D, K, G, fmt):
    """Single tokens of ragged sequences, one of which holds nothing."""
    c = KvCase(n_seqs=8, K=K, D=D, P=16, fmt=fmt)
    seqs = [6, 0, 2, 1, 7, 4]
    c.append(seqs, LENGTHS)
    c.attend(seqs + [5], [1] * 7, K * G, q_scale=3.0)


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("softcap,window", [(0.0, 0), (5.0, 0), (0.0, 20), (30.0, 1), (0.0, 1000)])
def test_decode_drafts(P, softcap, window):
    """Several query rows a sequence, ragged, more than are held among them (rows that see nothing)."""
    c = KvCase(n_seqs=4, K=2, D=128, P=P)
    c.append([0, 1, 2, 3], [130, 2, 64, 41])
    c.attend([3, 1, 0, 2], [5, 4, 1, 0], 10, softcap=softcap, window=window, q_scale=2.0)


@pytest.mark.parametrize("n", [1, 3])
def test_decode_long(n):
    """Lengths that many CTAs share, their parts joined."""
    c = KvCase(n_seqs=n, K=1, D=64, P=64, n_blocks=400, max_blocks=200)
    c.append(list(range(n)), [9000, 1234, 4000][:n])
    c.attend(list(range(n)), [2] * n, 4, observe=True)
    w = c.cache.weight.cpu().numpy()
    np.testing.assert_allclose(w, c.model.weight, rtol=2e-5, atol=1e-9)


def test_decode_is_deterministic_and_strided():
    c = KvCase(n_seqs=3, K=2, D=128)
    c.append([0, 1, 2], [900, 70, 512])
    q = tensor(c.rows(3, 16))
    cu, seqs = ints([0, 1, 2, 3]), ints([0, 1, 2])
    out, lse = c.cache.attention(q, cu, 1, seqs=seqs)
    wide = torch.full((3, 40, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:24] = q
    res = torch.zeros((3, 20, 128), dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        c.cache.attention(wide[:, 8:24], cu, 1, seqs=seqs, out=res[:, 2:18], stream=side)
        side.synchronize()
        assert torch.equal(res[:, 2:18], out)
    assert (res[:, :2] == 0).all() and (res[:, 18:] == 0).all()


def test_query_range():
    """Query rows of zeros, of the smallest numbers, and with one infinity."""
    c = KvCase(n_seqs=1, K=1, D=64, P=16)
    c.append([0], [50])
    q = c.rows(1, 4)
    q[0, 1] = 0
    q[0, 2] = bits(bf16_to_f64(q[0, 2]) * 1e-38)
    bad = q.copy()
    bad[0, 3, 7] = bits([np.inf])[0]
    c.attend([0], [1], 4, q=q, scale=10.0)
    out, _ = c.cache.attention(tensor(bad), ints([0, 1]), 1, seqs=ints([0]), scale=10.0)
    good, _ = c.cache.attention(tensor(q), ints([0, 1]), 1, seqs=ints([0]), scale=10.0)
    assert torch.equal(out[:, :3], good[:, :3]) and out[:, 3].isnan().all()


def test_large_scores():
    """Scores of thousands: the greatest takes all, nothing overflows."""
    c = KvCase(n_seqs=2, K=1, D=128, P=32)
    c.append([0, 1], [300, 40])
    c.attend([0, 1], [1, 1], 8, q_scale=300.0)


@pytest.mark.parametrize("P,n", [(16, 9), (32, 40), (128, 7)])
def test_evict(P, n):
    """Weights of ties, zeros, an infinity and NaN; sinks and recent blocks stay; then the cache is used on."""
    c = KvCase(n_seqs=3, K=1, D=64, P=P, n_blocks=3 * n + 2, max_blocks=n + 2)
    c.append([2, 0, 1], [n * P, n * P - 3, 2 * P])
    w = np.round(c.rng.random(c.model.weight.size) * 5).astype(np.float32)  # ties
    w[c.model.table[0][3]] = np.inf
    c.cache.weight.copy_(torch.from_numpy(w))
    c.model.weight[:] = w
    for keep, sinks, recent in [(n - 1, 0, 1), (n - 2, 2, 2), (5, 1, 1), (4, 1, 3), (2, 0, 1), (1, 0, 1)]:
        c.cache.evict(ints([1, 0, 2]), keep, sinks, recent)
        c.model.evict([1, 0, 2], keep, sinks, recent)
        c.check_state()
    c.check_values()
    c.append([0, 2], [P + 1, 2])
    c.check_state()
    c.check_values()
    c.attend([0, 1, 2], [1, 1, 1], 2)


def test_evict_long_tables():
    """Tables longer than a pass, and than the kernel holds keys of (40,000 blocks)."""
    c = KvCase(n_seqs=2, K=1, D=64, P=16, n_blocks=42100, max_blocks=40100)
    t0, t1 = np.arange(40000), np.arange(40000, 42000)
    c.cache.table[0, :40000] = ints(t0)
    c.cache.table[1, :2000] = ints(t1)
    c.cache.seq_state[:2, 0] = ints([40000 * 16, 2000 * 16])
    c.cache.seq_state[:2, 1] = c.cache.seq_state[:2, 0]
    c.cache.control[0] = 100
    w = c.rng.random(42100).astype(np.float32)
    w[::3] = 0.25
    c.cache.weight.copy_(torch.from_numpy(w))
    c.cache.evict(2, 1500, 3, 2)
    assert c.cache.status() == 0
    for s, t in ((0, t0), (1, t1)):
        mid = t[3:-2]
        keep = np.sort(mid[np.lexsort((mid, -w[mid]))][:1495])
        want = np.concatenate([t[:3], keep, t[-2:]])
        assert c.cache.table[s, :1500].cpu().numpy().tolist() == want.tolist()
    free = c.cache.free_ids.cpu().numpy()[100:int(c.cache.control[0])]
    assert free.size == 40000 - 1500 + 500 and len(set(free.tolist())) == free.size
    assert (np.diff(free[:38500]) > 0).all()  # in table order


def test_rollback_after_eviction():
    """With one recent block kept, the block before it is another: only its boundary can be gone back to."""
    c = KvCase(n_seqs=1, K=1, D=64, P=16)
    c.append([0], [70])
    c.cache.weight[:] = torch.arange(c.cache.weight.numel(), 0, -1, device="cuda")
    c.model.weight[:] = np.arange(c.model.weight.size, 0, -1)
    c.cache.evict(1, 3, 0, 1)
    c.model.evict([0], 3, 0, 1)
    c.check_state()
    c.cache.append(tensor(c.rows(1)), tensor(c.rows(1)), ints([0, 1]), start=ints([30]))
    assert c.cache.status() == N.MSI_ERR_INVALID_ARG
    c.append([0], [3], start=[34])
    c.append([0], [20], start=[32])
    c.append([0], [2], start=[16])
    c.check_state()
    c.check_values()


def test_release():
    c = KvCase(n_seqs=3, P=16, D=64, n_blocks=20, max_blocks=10)
    c.append([0, 1, 2], [100, 33, 1])
    c.cache.release(ints([1, 0]))
    c.model.release([1, 0])
    c.check_state()
    c.append([1, 0], [120, 17])
    c.check_state()
    c.check_values()
    c.attend([0, 1, 2], [1, 1, 1], 4)


def test_observe_then_evict():
    """A bounded cache in use: append, attend, evict, as a decode loop does."""
    c = KvCase(n_seqs=2, K=2, D=64, P=16, n_blocks=24, max_blocks=10)
    c.append([0, 1], [100, 37])
    for _ in range(40):
        c.append([0, 1], [1, 1])
        c.attend([0, 1], [1, 1], 8, observe=True, q_scale=4.0)
        np.testing.assert_allclose(c.cache.weight.cpu().numpy(), c.model.weight, rtol=2e-5, atol=1e-9)
        c.cache.evict(ints([0, 1]), 6, 1, 2)
        c.model.evict([0, 1], 6, 1, 2)
        c.check_state()
    c.check_values()


def test_read_parts_and_refusal():
    c = KvCase(n_seqs=2, P=16, D=64)
    c.append([0, 1], [50, 20])
    k, v = c.cache.read(ints([0, 7, 7, 10])[[0, 1, 3]].contiguous(), 10, seqs=ints([1, 0]), first=ints([13, 47]))
    ref = [c.model.values(s) for s in (1, 0)]
    for w, x in enumerate((k, v)):
        want = np.concatenate([ref[0][w][13:20], ref[1][w][47:50]]).astype(np.float32)
        np.testing.assert_array_equal(x.float().cpu().numpy(), bf16_to_f64(bits(want)))
    k, v = c.cache.read(ints([0, 4]), 4, seqs=ints([1]), first=ints([18]))
    assert k[2:].isnan().all() and v[2:].isnan().all() and not k[:2].isnan().any()
    assert c.cache.status() == N.MSI_ERR_INVALID_ARG


@pytest.mark.parametrize("seqs,cu", [([0, 0], [0, 1, 2]), ([0, 4], [0, 1, 2]), ([-1, 1], [0, 1, 2]),
                                     ([0, 1], [0, 2, 1]), ([0, 1], [-1, 1, 2]), ([0, 1], [0, 1, 3])])
def test_device_refusals(seqs, cu):
    """Sequence numbers and row offsets out of range: nothing changes, attention answers NaN."""
    c = KvCase(n_seqs=4, D=64, P=16)
    c.append([0, 1], [20, 20])
    k = tensor(c.rows(2))
    c.cache.append(k, k, ints(cu), seqs=ints(seqs))
    assert c.cache.status() == N.MSI_ERR_INVALID_ARG
    c.check_state()
    c.check_values()
    if seqs != [0, 0]:
        out, lse = c.cache.attention(tensor(c.rows(2, 4)), ints(cu), 2, seqs=ints(seqs))
        assert out.isnan().all() and lse.isnan().all()
        assert c.cache.status() == N.MSI_ERR_INVALID_ARG
    if cu == [0, 1, 2]:
        c.cache.evict(ints(seqs), 1)
        assert c.cache.status() == N.MSI_ERR_INVALID_ARG
        c.cache.release(ints(seqs))
        assert c.cache.status() == N.MSI_ERR_INVALID_ARG
    c.check_state()


def test_wrong_table_entry():
    """A table that names a block the pool does not have: NaN and an error, no access."""
    c = KvCase(n_seqs=2, D=64, P=16)
    c.append([0, 1], [300, 20])
    c.cache.table[0, 9] = 1 << 20
    out, _ = c.cache.attention(tensor(c.rows(2, 4)), ints([0, 1, 2]), 1)
    assert out[0].isnan().all()
    assert c.cache.status() == N.MSI_ERR_INVALID_ARG
    k, _ = c.cache.read(ints([0, 300]), 300, seqs=ints([0]))
    assert k[144:160].isnan().all() and not k[:144].isnan().any()
    assert c.cache.status() == N.MSI_ERR_INVALID_ARG


def test_host_refusals():
    c = KvCase(n_seqs=2, D=64, P=16)
    l, h = N.lib(), c.cache.h
    good = {"n_seqs": 2, "max_blocks": 4, "n_blocks": 4, "n_kv_heads": 1, "head_dim": 64, "block_tokens": 16}
    for change, err in [({"head_dim": 96}, N.MSI_ERR_UNSUPPORTED), ({"block_tokens": 24}, N.MSI_ERR_UNSUPPORTED),
                        ({"n_seqs": 1025}, N.MSI_ERR_UNSUPPORTED), ({"n_kv_heads": 65}, N.MSI_ERR_UNSUPPORTED),
                        ({"fmt": 2}, N.MSI_ERR_INVALID_ARG)]:
        with pytest.raises(N.MsiError) as e:
            api.KvCache(**{**good, **change})
        assert e.value.status == err
    q = tensor(c.rows(2, 4))
    cu = ints([0, 1, 2])
    for kw, err in [({"scale": 0.0}, N.MSI_ERR_INVALID_ARG), ({"scale": float("inf")}, N.MSI_ERR_INVALID_ARG),
                    ({"softcap": -1.0}, N.MSI_ERR_INVALID_ARG), ({"window": -1}, N.MSI_ERR_INVALID_ARG)]:
        with pytest.raises(N.MsiError) as e:
            c.cache.attention(q, cu, 1, **kw)
        assert e.value.status == err
    with pytest.raises(N.MsiError):
        c.cache.attention(tensor(c.rows(2, 3)), cu, 1)              # 3 heads over 2
    with pytest.raises(N.MsiError):
        c.cache.attention(q, cu, 3)                                  # more rows than there are
    with pytest.raises(N.MsiError):
        c.cache.attention(tensor(c.rows(4, 4)), ints([0, 1, 1, 4]), 3)  # more sequences than the cache has
    for keep, sinks, recent in [(2, 2, 1), (1, 0, 0), (0, 0, 1), (3, -1, 1)]:
        with pytest.raises(N.MsiError):
            c.cache.evict(2, keep, sinks, recent)
    with pytest.raises(ValueError):
        c.cache.append(q, q, cu)
    with pytest.raises(ValueError):
        c.cache.attention(q, cu.long(), 1)
    a = N.msi_kv_attention_args(2, None, cu.data_ptr(), 2, 1, 4, q.data_ptr(), 256, q.data_ptr(), 256, None, 1.0, 0.0, 0, 0)
    n, form = ctypes.c_size_t(), ctypes.c_int()
    assert l.msi_kv_workspace_size(h, ctypes.byref(a), ctypes.byref(n), ctypes.byref(form)) == 0 and form.value == 1
    ws = torch.empty(n.value + 256, dtype=torch.uint8, device="cuda")
    assert l.msi_kv_attention(h, ctypes.byref(a), ws.data_ptr() + 16, n.value, None) == N.MSI_ERR_WORKSPACE
    assert l.msi_kv_attention(h, ctypes.byref(a), ws.data_ptr(), n.value - 1, None) == N.MSI_ERR_WORKSPACE
    assert l.msi_kv_attention(None, ctypes.byref(a), ws.data_ptr(), n.value, None) == N.MSI_ERR_INVALID_ARG
    a.flags = 2
    assert l.msi_kv_attention(h, ctypes.byref(a), ws.data_ptr(), n.value, None) == N.MSI_ERR_INVALID_ARG
    assert l.msi_kv_append(h, 3, None, cu.data_ptr(), None, q.data_ptr(), q.data_ptr(), 128, 2, None) == N.MSI_ERR_INVALID_ARG
    assert l.msi_kv_append(h, 2, None, cu.data_ptr(), None, q.data_ptr() + 2, q.data_ptr(), 128, 2, None) == N.MSI_ERR_INVALID_ARG
    assert l.msi_kv_append(h, 2, None, cu.data_ptr(), None, q.data_ptr(), q.data_ptr(), 127, 2, None) == N.MSI_ERR_INVALID_ARG
    assert c.cache.status() == 0 and c.cache.launches() == 1  # nothing was enqueued but init


def test_nothing_to_do():
    c = KvCase(n_seqs=2, D=64, P=16)
    c.append([0, 1], [0, 0])
    out, lse = c.cache.attention(tensor(c.rows(0, 4)), ints([0, 0, 0]), 0)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    c.cache.read(ints([0, 0]), 0)
    c.cache.evict(2, 1)
    c.cache.release(0)
    c.check_state()


def test_graph_replay():
    """A decode step captured once and replayed: all state is on the GPU."""
    c = KvCase(n_seqs=2, K=1, D=64, P=16, n_blocks=40, max_blocks=20)
    c.append([0, 1], [30, 5])
    k, v, q = (torch.zeros((2, h, 64), dtype=torch.bfloat16, device="cuda") for h in (1, 1, 4))
    cu = ints([0, 1, 2])
    out, lse = torch.empty_like(q), torch.empty((2, 4), dtype=torch.float32, device="cuda")
    c.cache.attention(q, cu, 1, out=out, lse=lse)  # the workspace is made
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.cache.append(k, v, cu)
        c.cache.attention(q, cu, 1, out=out, lse=lse)
    for _ in range(20):
        ks, vs, qs = c.rows(2), c.rows(2), c.rows(2, 4)
        for t, x in ((k, ks), (v, vs), (q, qs)):
            t.copy_(tensor(x))
        g.replay()
        torch.cuda.synchronize()
        c.model.append([0, 1], [0, 1, 2], ks, vs)
        from kv_case import check_rows
        for s in range(2):
            ref = c.model.attention(s, bf16_to_f64(qs[s:s + 1]), 64 ** -0.5)
            check_rows(out[s:s + 1].double().cpu().numpy(), lse[s:s + 1].double().cpu().numpy(), ref, 64, 0.0)
    c.check_state()
    c.check_values()


# -- chunk form: more rows a sequence and key-value head than decode form takes --

@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("K,G,P", [(1, 1, 16), (2, 4, 64), (1, 7, 32), (1, 16, 128)])
def test_chunk(D, K, G, P, fmt):
    """Ragged chunks of ragged sequences: a sequence that holds nothing, one
    whose chunk is all it holds, one without rows, one with a single row."""
    c = KvCase(n_seqs=8, K=K, D=D, P=P, fmt=fmt)
    seqs, held = [6, 0, 2, 1, 7], [300, 41, 129, 200, 70]
    c.append(seqs, held)
    c.attend([2, 5, 6, 0, 7, 1], [129, 3, 34, 41, 0, 1], K * G, q_scale=2.0)


@pytest.mark.parametrize("D", [64, 256])
@pytest.mark.parametrize("softcap,window", [(5.0, 0), (0.0, 1), (0.0, 100), (20.0, 33), (0.0, 5000)])
def test_chunk_scores(D, softcap, window):
    c = KvCase(n_seqs=2, K=2, D=D, P=16)
    c.append([0, 1], [700, 90])
    c.attend([1, 0], [60, 200], 4, softcap=softcap, window=window, q_scale=2.0)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_chunk_rows_that_see_nothing(D):
    """More rows than tokens: the first of them give 0 and -inf."""
    c = KvCase(n_seqs=2, K=1, D=D, P=16)
    c.append([0, 1], [20, 333])
    c.attend([0, 1], [300, 340], 2)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_chunk_rising_scores(D):
    """Keys that grow along the sequence: the running reference moves in most
    tiles, and scores reach thousands."""
    c = KvCase(n_seqs=1, K=1, D=D, P=16)
    k = bits(c.rng.standard_normal((1000, 1, D)) * np.linspace(0.1, 60, 1000)[:, None, None])
    c.append([0], [1000], k=k)
    c.attend([0], [70], 4, q_scale=8.0)


def test_chunk_many_sequences():
    """More items than a pass of the plan, and CTAs with parts of many of them."""
    c = KvCase(n_seqs=300, K=4, D=64, P=16, n_blocks=2000, max_blocks=8)
    order = c.rng.permutation(300).tolist()
    c.append(order, [40] * 300)
    c.attend(order, [33 + i % 2 for i in range(300)], 4)


@pytest.mark.parametrize("D,fmt", [(128, N.MSI_KV_Q8), (256, N.MSI_KV_E4M3)])
def test_chunk_not_finite(D, fmt):
    """A block with a NaN: the rows before its tokens are as without it."""
    c = KvCase(D=D, P=16, K=1, fmt=fmt, n_seqs=2)
    k, v = c.rows(200), c.rows(200)
    c.append([1], [200], k=k, v=v)
    v[100, 0, 5] = bits([np.nan])[0]
    c.append([0], [200], k=k, v=v)
    q = c.rows(200, 2)
    out, lse = c.cache.attention(tensor(q), ints([0, 200]), 200, seqs=ints([0]))
    ref, ref_lse = c.cache.attention(tensor(q), ints([0, 200]), 200, seqs=ints([1]))
    assert out[96:].isnan().all()
    assert torch.equal(out[:96], ref[:96]) and torch.equal(lse[:96], ref_lse[:96])


def test_chunk_equals_decode_and_is_deterministic():
    """A chunk's last row against the same row as a decode call, within both
    forms' roundings; strided rows, another stream, the same bits every time."""
    c = KvCase(n_seqs=3, K=2, D=128)
    c.append([0, 1, 2], [900, 70, 512])
    q = tensor(c.rows(180, 16))
    cu, seqs = ints([0, 100, 140, 180]), ints([0, 1, 2])
    out, lse = c.cache.attention(q, cu, 100, seqs=seqs)
    one, one_lse = c.cache.attention(q[[99, 139, 179]].contiguous(), ints([0, 1, 2, 3]), 1, seqs=seqs)
    last = out[[99, 139, 179]]
    assert (last.float() - one.float()).abs().max() <= 2.0 ** -7 * one.float().abs().max()
    assert (lse[[99, 139, 179]] - one_lse).abs().max() < 1e-5
    wide = torch.full((180, 40, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:24] = q
    res = torch.zeros((180, 20, 128), dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        c.cache.attention(wide[:, 8:24], cu, 100, seqs=seqs, out=res[:, 2:18], stream=side)
        side.synchronize()
        assert torch.equal(res[:, 2:18], out)
    assert (res[:, :2] == 0).all() and (res[:, 18:] == 0).all()


def test_chunk_refusals():
    c = KvCase(n_seqs=2, K=1, D=64, P=16)
    c.append([0, 1], [50, 60])
    q = tensor(c.rows(80, 2))
    with pytest.raises(N.MsiError) as e:
        c.cache.attention(q, ints([0, 40, 80]), 40, observe=True)
    assert e.value.status == N.MSI_ERR_UNSUPPORTED
    for seqs, cu in [([0, 2], [0, 40, 80]), ([0, 1], [0, 40, 81]), ([0, 1], [0, 41, 80])]:
        out, lse = c.cache.attention(q, ints(cu), 40, seqs=ints(seqs))
        assert out.isnan().all() and lse.isnan().all()
        assert c.cache.status() == N.MSI_ERR_INVALID_ARG
    c.cache.table[0, 1] = -5
    out, _ = c.cache.attention(q, ints([0, 40, 80]), 40)
    assert out[10:40].isnan().all()
    assert c.cache.status() == N.MSI_ERR_INVALID_ARG


def test_decode_parts_of_every_number():
    """Pairs cut into few and into many parts in one call: one long sequence
    among short ones (its parts are joined by whole CTAs, theirs by warps)."""
    c = KvCase(n_seqs=6, K=2, D=64, P=16, n_blocks=1500, max_blocks=1200)
    c.append(list(range(6)), [18000, 300, 40, 900, 16, 1])
    c.attend([3, 0, 5, 1, 2, 4], [1, 2, 1, 1, 2, 1], 4, observe=True)
    np.testing.assert_allclose(c.cache.weight.cpu().numpy(), c.model.weight, rtol=2e-5, atol=1e-9)
