"""Plain model of the 8-bit key-value cache, numpy on the CPU.

TEST INFRASTRUCTURE ONLY (see the package's docstring).  Blocks, tables and the
free list are lists; a block's rounding is the header's formula in fp32, one
operation at a time; attention is computed in fp64 from the values held.  The
paper leaves KV state to the native runtime: the definitions are those of
include/msi.h alone.
"""
from __future__ import annotations

import math

import numpy as np

from .moe import bf16_to_f64

Q8, E4M3 = 0, 1


def round_e4m3(y: np.ndarray) -> np.ndarray:
    """fp32 to the nearest e4m3 number (ties to even, above 448: 448), as fp64."""
    y = y.astype(np.float64)
    exp = np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6)))
    step = 2.0 ** (exp - 3)
    return np.clip(np.round(y / step) * step, -448.0, 448.0)


def round_block(rows: np.ndarray, fmt: int) -> tuple[np.ndarray, np.ndarray]:
    """rows fp32 [P, K, D] of a block -> (code values fp64 [P, K, D], scales fp32 [K])."""
    top = np.float32(127.0 if fmt == Q8 else 448.0)
    fine = np.isfinite(rows).all(axis=(0, 2))
    with np.errstate(invalid="ignore"):
        a = np.maximum(np.abs(rows).max(axis=(0, 2)), np.float32(1e-20)).astype(np.float32)
        inv = (top / a).astype(np.float32)
        y = (rows * inv[None, :, None]).astype(np.float32)
    y = np.where(fine[None, :, None], y, np.float32(0))
    scale = (a * (np.float32(1) / top)).astype(np.float32)
    code = np.round(y.astype(np.float64)) if fmt == Q8 else round_e4m3(y)
    return code, np.where(fine, scale, np.float32(np.nan))


class KvModel:
    """One cache.  Rows are uint16 bf16 bits [n, K, D]."""

    def __init__(self, n_seqs, max_blocks, n_blocks, K, D, P, fmt):
        self.max_blocks, self.K, self.D, self.P, self.fmt = max_blocks, K, D, P, fmt
        self.free = list(range(n_blocks - 1, -1, -1))
        self.weight = np.zeros(n_blocks, np.float64)
        self.table = [[] for _ in range(n_seqs)]
        self.rows = [[] for _ in range(n_seqs)]      # per sequence, per block: [2][rows][K, D] fp32
        self.pos = [0] * n_seqs

    def held(self, s):
        return sum(len(b[0]) for b in self.rows[s])

    def append(self, seqs, cu, k, v, start=None):
        """False (and nothing changed) when the pool or a table has no place."""
        spans = []
        need = 0
        for i, s in enumerate(seqs):
            at = self.held(s) if start is None else start[i]
            had = len(self.table[s])
            have = -(-(at + cu[i + 1] - cu[i]) // self.P)
            if have > self.max_blocks:
                return False
            need += max(0, have - had)
            spans.append((at, had, have))
        if need > len(self.free):
            return False
        drops = []
        for i, s in enumerate(seqs):
            at, had, have = spans[i]
            self.pos[s] += at + cu[i + 1] - cu[i] - self.held(s)
            n = -(-at // self.P)  # blocks that keep rows
            self.rows[s] = self.rows[s][:n]
            if at % self.P:
                self.rows[s][-1] = [x[:at % self.P] for x in self.rows[s][-1]]
            for r in range(cu[i], cu[i + 1]):
                if not self.rows[s] or len(self.rows[s][-1][0]) == self.P:
                    self.rows[s].append([[], []])
                for w, x in enumerate((k, v)):
                    self.rows[s][-1][w].append(bf16_to_f64(x[r]).astype(np.float32))
            drops += self.table[s][have:]
            self.table[s] = self.table[s][:have]
            while len(self.table[s]) < have:
                b = self.free.pop()
                self.weight[b] = 0.0
                self.table[s].append(b)
        self.free += drops
        return True

    def values(self, s):
        """(k, v) fp64 [held, K, D], the values that the codes stand for."""
        out = [[], []]
        for block in self.rows[s]:
            for w in range(2):
                full = np.zeros((self.P, self.K, self.D), np.float32)
                full[:len(block[w])] = np.stack(block[w])
                code, scale = round_block(full, self.fmt)
                out[w].append((code * scale.astype(np.float64)[None, :, None])[:len(block[w])])
        if not out[0]:
            return [np.zeros((0, self.K, self.D))] * 2
        return [np.concatenate(x) for x in out]

    def attention(self, s, q, scale, softcap=0.0, window=0):
        """q fp64 [r, H, D], the last tokens of sequence s -> dict of out
        [r, H, D], lse [r, H], weights [H, r, held], and what error bounds need:
        absolute weighted values [r, H, D], largest sum of |scale q k| [r, H] and
        number of tokens seen times their largest absolute value [r, H]."""
        k, v = self.values(s)
        r, H, D = q.shape
        G, L = H // self.K, k.shape[0]
        out, mag = np.zeros((r, H, D)), np.zeros((r, H, D))
        lse, size, bulk = np.full((r, H), -np.inf), np.zeros((r, H)), np.zeros((r, H))
        weights = np.zeros((H, r, L))
        for i in range(r):
            at = L - r + i
            lo = max(0, at - window + 1) if window else 0
            if at < lo:
                continue
            for h in range(H):
                kk, vv = k[lo:at + 1, h // G], v[lo:at + 1, h // G]
                x = kk @ q[i, h] * scale
                if softcap:
                    x = softcap * np.tanh(x / softcap)
                top = x.max()
                e = np.exp(x - top)
                p = e / e.sum()
                lse[i, h] = top + math.log(e.sum())
                out[i, h], mag[i, h] = p @ vv, p @ np.abs(vv)
                size[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
                bulk[i, h] = vv.shape[0] * np.abs(vv).max()
                weights[h, i, lo:at + 1] = p
        return {"out": out, "lse": lse, "weights": weights, "mag": mag, "size": size, "bulk": bulk}

    def observe(self, s, weights):
        """Add attention weights [H, r, held] up per block."""
        per = weights.sum((0, 1))
        for j, b in enumerate(self.table[s]):
            self.weight[b] += per[j * self.P:(j + 1) * self.P].sum()

    def evict(self, seqs, keep, sinks, recent):
        for s in seqs:
            n = len(self.table[s])
            if n <= keep:
                continue
            w = [self.weight[b] for b in self.table[s]]
            middle = sorted(range(sinks, n - recent), key=lambda j: (-w[j], j))[:keep - sinks - recent]
            kept = sorted(list(range(sinks)) + middle + list(range(n - recent, n)))
            gone = [j for j in range(n) if j not in set(kept)]
            self.free += [self.table[s][j] for j in gone]
            self.table[s] = [self.table[s][j] for j in kept]
            self.rows[s] = [self.rows[s][j] for j in kept]

    def release(self, seqs):
        for s in seqs:
            self.free += self.table[s]
            self.table[s], self.rows[s], self.pos[s] = [], [], 0
