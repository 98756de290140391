"""Calls with an explicit stream: what they make, take and hold belongs to that
stream until its work is done, whatever the caller's own stream does meanwhile."""
import pytest
import torch

from kv_case import KvCase, ints, tensor
from paper_2608_23805_gb300 import api

pytestmark = pytest.mark.gpu
LONG = 400_000_000  # clock cycles that a stream is kept busy: some 200 ms


def cache_of(D=128):
    c = KvCase(n_seqs=1, K=2, D=D, P=16, max_blocks=64, n_blocks=64)
    c.append([0], [600])
    return c


def settle():
    """Nothing under way, and no free memory in the allocator's hands: what is
    freed from here on is what the next allocation of its size takes."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def test_results_do_not_take_memory_that_the_current_stream_still_reads():
    n = 600
    c = KvCase(n_seqs=n, K=2, D=128, P=16, max_blocks=4, n_blocks=4 * n)
    c.append(list(range(n)), [20] * n)
    q, cu = tensor(c.rows(n, 16)), ints(range(n + 1))
    side = torch.cuda.Stream()
    ref, ref_lse = c.cache.attention(q, cu, 1)
    settle()
    # temporaries as large as what the call makes, read late and let go at once
    old = [torch.full_like(ref, 3.0) for _ in range(24)] + [torch.full_like(ref_lse, 3.0) for _ in range(64)]
    torch.cuda.synchronize()
    torch.cuda._sleep(LONG)
    sums = [t.sum(dtype=torch.float32) for t in old]
    sizes, ptrs = [t.numel() for t in old], [t.data_ptr() for t in old]
    del old
    out, lse = c.cache.attention(q, cu, 1, stream=side)
    torch.cuda.synchronize()
    # its kernels may have waited for the busy SM, but nothing orders them with it
    assert out.data_ptr() not in ptrs and lse.data_ptr() not in ptrs
    assert [float(s) for s in sums] == [3.0 * n for n in sizes]
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)


def test_read_back_does_not_take_memory_that_the_current_stream_still_reads():
    c = cache_of()
    cu = ints([0, 600])
    ref = c.cache.read(cu, 600)
    side = torch.cuda.Stream()
    settle()
    old = [torch.full_like(ref[0], 3.0) for _ in range(4)]
    torch.cuda.synchronize()
    torch.cuda._sleep(LONG)
    sums = [t.sum(dtype=torch.float32) for t in old]
    n = old[0].numel()
    del old
    got = c.cache.read(cu, 600, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert [float(s) for s in sums] == [3.0 * n] * 4
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


def test_results_outlive_the_stream_that_made_them():
    """What a call made is read on the caller's stream and let go: its memory is
    not given to the next call on the other stream before that read."""
    c = cache_of()
    q, cu = tensor(c.rows(500, 16)), ints([0, 500])
    q2 = tensor(c.rows(500, 16))
    ref, _ = c.cache.attention(q, cu, 500)
    ref2, _ = c.cache.attention(q2, cu, 500)
    side = torch.cuda.Stream()
    settle()
    out, lse = c.cache.attention(q, cu, 500, stream=side)
    side.synchronize()
    torch.cuda._sleep(LONG)
    late = out.clone()
    del out, lse
    out2, _ = c.cache.attention(q2, cu, 500, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(late, ref) and torch.equal(out2, ref2)


def test_inputs_are_held_until_the_other_stream_has_read_them():
    a, b = cache_of(), cache_of()
    k, v = (tensor(a.rows(400)) for _ in range(2))
    cu = ints([0, 400])
    b.cache.append(k, v, cu)
    side = torch.cuda.Stream()
    settle()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    a.cache.append(k.clone(), v.clone(), cu.clone(), stream=side)
    torch.cuda.current_stream().synchronize()
    over = [torch.zeros_like(k) for _ in range(4)] + [torch.zeros_like(cu) for _ in range(4)]
    torch.cuda.synchronize()
    assert len(over) == 8 and a.cache.status() == 0
    for x, y in zip(a.cache.read(ints([0, 1000]), 1000), b.cache.read(ints([0, 1000]), 1000)):
        assert torch.equal(x, y)


def test_a_cache_let_go_with_work_under_way():
    """Its buffers are not given out before the other stream is done with them."""
    c = KvCase(n_seqs=1, K=2, D=128, P=16, max_blocks=1024, n_blocks=1024)
    k, v, cu = tensor(c.rows(16000)), tensor(c.rows(16000)), ints([0, 16000])
    cache, c.cache = c.cache, None
    side = torch.cuda.Stream()
    size, ptrs = cache.k_codes.shape, [cache.k_codes.data_ptr(), cache.v_codes.data_ptr()]
    torch.full(size, 0x5A, dtype=torch.uint8, device="cuda")  # its kernel is loaded
    settle()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    cache.append(k, v, cu, stream=side)
    del cache
    others = [torch.full(size, 0x5A, dtype=torch.uint8, device="cuda") for _ in range(40)]
    busy = not side.query()
    torch.cuda.synchronize()
    assert busy and not set(ptrs) & {t.data_ptr() for t in others}
    assert all(bool((t == 0x5A).all()) for t in others)


def test_made_on_another_stream():
    """The buffers of a cache made on a stream are that stream's from the start:
    earlier readers of the same memory are not overtaken by its first kernel."""
    make = dict(n_seqs=1, max_blocks=4096, n_blocks=300000, n_kv_heads=1, head_dim=64, block_tokens=16)
    side = torch.cuda.Stream()
    settle()
    old = [torch.full((300000,), 7, dtype=torch.int32, device="cuda") for _ in range(4)]  # as large as free_ids and weight
    torch.cuda.synchronize()
    torch.cuda._sleep(LONG)
    sums = [t.sum() for t in old]
    del old
    cache = api.KvCache(**make, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert [int(s) for s in sums] == [7 * 300000] * 4
    assert int(cache.control[0]) == 300000 and cache.status(side) == 0
