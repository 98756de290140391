"""Captured decode steps among other calls on the same cache: a graph holds the
address of the workspace that it was captured with."""
import pytest
import torch

from kv_case import KvCase, ints, tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("side", [False, True])
def test_larger_call_after_capture(side):
    """A step is captured, a longer prompt than any before needs a larger
    workspace, other tensors are made, then the step is replayed: its answer is
    right, and it has written to nothing but its own memory."""
    c = KvCase(n_seqs=2, K=2, D=128, P=16, n_blocks=300, max_blocks=200)
    c.append([0, 1], [1000, 40])
    q, cu = tensor(c.rows(2, 16)), ints([0, 1, 2])
    out, lse = torch.empty_like(q), torch.empty((2, 16), dtype=torch.float32, device="cuda")
    want, want_lse = (t.clone() for t in c.cache.attention(q, cu, 1, observe=True))
    before = c.cache._ws
    stream = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        if side:
            here = torch.cuda.current_stream()
            stream.wait_stream(here)
            c.cache.attention(q, cu, 1, out=out, lse=lse, observe=True, stream=stream)
            here.wait_stream(stream)
        else:
            c.cache.attention(q, cu, 1, out=out, lse=lse, observe=True)
    captured, size = c.cache._ws.data_ptr(), c.cache._ws.numel()
    assert captured == before.data_ptr()
    del before
    c.append([1], [600])
    chunk = tensor(c.rows(600, 16))
    c.cache.attention(chunk, ints([0, 600]), 600, seqs=ints([1]))
    assert c.cache._ws.numel() > size  # replaced
    torch.cuda.synchronize()
    # what the allocator gives out from here on is not the graph's
    others = [torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert all(t.data_ptr() != captured for t in others)
    c.append([1], [40], start=[0])  # back to 40 tokens, other ones
    ref, ref_lse = c.cache.attention(q, cu, 1, observe=True)
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    assert all(bool((t == 0x5A).all()) for t in others)
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
    assert torch.equal(out[0], want[0]) and torch.equal(lse[0], want_lse[0])
    assert c.cache.status() == 0


def test_replaced_workspaces_are_kept_only_for_graphs():
    """Without a capture a replaced workspace goes back to the allocator."""
    c = KvCase(n_seqs=1, K=1, D=64, P=16)
    c.append([0], [100])
    c.cache.attention(tensor(c.rows(1, 4)), ints([0, 1]), 1)
    c.cache.attention(tensor(c.rows(90, 4)), ints([0, 90]), 90)
    assert c.cache._ws_kept == []
