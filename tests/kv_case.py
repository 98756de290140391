"""Shared setup of the key-value cache's GPU tests: a cache and its plain model
fed with the same rows, and the comparisons between them."""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv as M
from oracle.moe import bf16_to_f64
from paper_2608_23805_gb300 import api
from paper_2608_23805_gb300 import native as N


def bits(x):
    """fp32 array -> bf16 bits (ties to even)."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def tensor(b):
    return torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).view(torch.bfloat16).cuda()


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


class KvCase:
    def __init__(self, *, n_seqs=4, max_blocks=64, n_blocks=128, K=2, D=128, P=32, fmt=N.MSI_KV_Q8, seed=0):
        self.K, self.D, self.P, self.n_seqs = K, D, P, n_seqs
        self.cache = api.KvCache(n_seqs=n_seqs, max_blocks=max_blocks, n_blocks=n_blocks, n_kv_heads=K, head_dim=D,
                                 block_tokens=P, fmt=fmt)
        self.model = M.KvModel(n_seqs, max_blocks, n_blocks, K, D, P, fmt)
        self.rng = np.random.default_rng(seed)

    def rows(self, n, heads=None, scale=1.0):
        return bits(self.rng.standard_normal((n, self.K if heads is None else heads, self.D)) * scale)

    def append(self, seqs, counts, start=None, k=None, v=None, scale=1.0):
        """Append to both; returns whether the model had place."""
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(int)
        k = self.rows(cu[-1], scale=scale) if k is None else k
        v = self.rows(cu[-1], scale=scale) if v is None else v
        self.cache.append(tensor(k), tensor(v), ints(cu), seqs=ints(seqs), start=None if start is None else ints(start))
        return self.model.append(seqs, cu, k, v, start)

    def check_state(self):
        m, c = self.model, self.cache
        state, table = c.seq_state.cpu().numpy(), c.table.cpu().numpy()
        n_free, status = c.control.cpu().numpy()[:2]
        assert status == 0 and (c.control.cpu().numpy()[2:] == 0).all()
        assert c.free_ids.cpu().numpy()[:n_free].tolist() == m.free
        for s in range(self.n_seqs):
            assert state[s, 0] == m.held(s) and state[s, 1] == m.pos[s], s
            assert table[s, :len(m.table[s])].tolist() == m.table[s], s

    def check_values(self, seqs=None):
        """Every token read back equals the model's value, rounded to bf16."""
        seqs = list(range(self.n_seqs)) if seqs is None else seqs
        held = [self.model.held(s) for s in seqs]
        cu = np.concatenate([[0], np.cumsum(held)]).astype(int)
        got = self.cache.read(ints(cu), int(cu[-1]), seqs=ints(seqs))
        for i, s in enumerate(seqs):
            for w, ref in enumerate(self.model.values(s)):
                x = got[w][cu[i]:cu[i + 1]].float().cpu().numpy()
                want = bf16_to_f64(bits(ref.astype(np.float32)))
                np.testing.assert_array_equal(x, want.astype(np.float32))

    def attend(self, seqs, counts, heads, *, scale=None, softcap=0.0, window=0, observe=False, q=None, q_scale=1.0,
               max_rows=None, **kw):
        """Attention of both, compared within what the arithmetic allows."""
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(int)
        q = self.rows(cu[-1], heads, q_scale) if q is None else q
        out, lse = self.cache.attention(tensor(q), ints(cu), max(counts) if max_rows is None else max_rows, seqs=ints(seqs),
                                        scale=scale, softcap=softcap, window=window, observe=observe, **kw)
        out, lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
        scale = self.D ** -0.5 if scale is None else scale
        for i, s in enumerate(seqs):
            if counts[i] == 0:
                continue
            qs = bf16_to_f64(q[cu[i]:cu[i + 1]])
            ref = self.model.attention(s, qs, scale, softcap, window)
            check_rows(out[cu[i]:cu[i + 1]], lse[cu[i]:cu[i + 1]], ref, self.D, softcap)
            if observe:
                self.model.observe(s, ref["weights"])
        return out, lse


def check_rows(out, lse, ref, D, softcap):
    """Scores: fp32 sums of D exact products, ten more fp32 roundings of numbers
    no larger than the largest sum of absolute products (or the cap), and query
    elements under 2^-14 of a row's largest rounded to 2^-24 of it.  That error
    ds moves every weight by a factor 1 + 2 ds.  Weights: fp16, 2^-11 of each,
    and where fp16's exponents end (numbers under 2^-14 of the row's largest have
    a spacing of 2^-24 of it) 2^-25 of the largest; the sum in fp32.  Output: bf16, 8 significant bits, so 2^-8 of it."""
    ds = (2 * D + 10) * 2.0 ** -24 * (ref["size"] + softcap + 1.0) + 2.0 ** -20
    empty = np.isinf(ref["lse"])
    assert (np.isneginf(lse) == empty).all()
    assert (out[empty] == 0).all()
    got, want = lse[~empty], ref["lse"][~empty]
    assert (np.abs(got - want) <= (ds + 2.0 ** -22 * np.abs(ref["lse"]))[~empty]).all(), np.abs(got - want).max()
    own = (2.0 ** -11 + 2 * ds)[..., None] * ref["mag"] + 2.0 ** -25 * ref["bulk"][..., None] + 1e-30
    tol = 2.0 ** -8 * np.abs(ref["out"]) + 1.01 * own
    bad = np.abs(out - ref["out"]) > tol
    assert not bad.any(), (np.argwhere(bad)[:3], (np.abs(out - ref["out"]) / tol).max())
