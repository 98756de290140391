"""The decoder stack of examples/: chunk, decode, observation and eviction with
the MoE layer between them, every attention against the plain model."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from kv_case import check_rows
from oracle import kv as M
from oracle.moe import bf16_to_f64

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("decode_stack", os.path.join(ROOT, "examples", "decode_stack.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def host(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def test_stack_against_the_model():
    keep, P, D = 4, 16, 64
    stack = example().Stack(keep=keep, block_tokens=P, head_dim=D)
    models = [M.KvModel(2, 32, 64, 2, D, P, M.Q8) for _ in range(2)]
    counts = [70, 21]

    def seen(l, q, k, v, out, lse):
        cu = np.concatenate([[0], np.cumsum(counts)])
        assert models[l].append([0, 1], cu, host(k), host(v))
        got, sums, rows = bf16_to_f64(host(out)), lse.cpu().numpy(), bf16_to_f64(host(q))
        for s in range(2):
            part = slice(cu[s], cu[s + 1])
            ref = models[l].attention(s, rows[part], D ** -0.5)
            check_rows(got[part], sums[part], ref, D, 0.0)

    def blocks(l):  # what the device kept, then the model's
        cache = stack.caches[l]
        held = cache.seq_state[:, 0].cpu().numpy()
        return [cache.table[s, :-(-held[s] // P)].cpu().tolist() for s in range(2)]

    hidden = stack.w_qkv[0].shape[0]
    x = torch.randn((sum(counts), hidden), generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    cu = torch.tensor([0, 70, 91], dtype=torch.int32, device="cuda")
    x = stack.step(x, cu, 70, decode=False, seen=seen)[cu[1:].long() - 1]
    counts = [1, 1]
    one = torch.arange(3, dtype=torch.int32, device="cuda")
    for _ in range(40):
        x = stack.step(x, one, 1, decode=True, seen=seen)
        for l in range(2):
            # the choice itself is tested elsewhere: the model drops what the device dropped
            kept = blocks(l)
            m = models[l]
            for s in range(2):
                assert len(kept[s]) <= keep
                gone = [j for j, b in enumerate(m.table[s]) if b not in kept[s]]
                m.free += [m.table[s][j] for j in gone]
                m.rows[s] = [r for j, r in enumerate(m.rows[s]) if j not in gone]
                m.table[s] = kept[s]
    assert stack.status() == 0
    assert bool(torch.isfinite(x.float()).all())
    for l in range(2):
        assert stack.caches[l].seq_state[:, 1].tolist() == [110, 61]
        assert all(len(b) == keep for b in blocks(l))


def test_example_runs(monkeypatch):
    monkeypatch.setattr("sys.argv", ["decode_stack.py", "--steps", "3"])
    assert example().main() == 0
