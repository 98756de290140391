"""The cache takes no tensor of another GPU than its own: its kernels would read
addresses that are not theirs.  Tensors here are stand-ins with a device number."""
import math
import types

import pytest
import torch

from paper_2608_23805_gb300 import api


def tensor(shape, dtype, device):
    strides = [math.prod(shape[i + 1:]) for i in range(len(shape))]
    return types.SimpleNamespace(shape=torch.Size(shape), dtype=dtype, is_cuda=device >= 0, get_device=lambda: device, numel=lambda: math.prod(shape),
                                 stride=lambda i=None: tuple(strides) if i is None else strides[i], is_contiguous=lambda: True,
                                 dim=lambda: len(shape), data_ptr=lambda: 4096, device=types.SimpleNamespace(index=device))


@pytest.fixture
def cache():
    c = object.__new__(api.KvCache)
    c.n_seqs, c.K, c.D, c.P, c._device_index = 4, 2, 64, 16, 0
    return c


def ints(n, device=0):
    return tensor((n,), torch.int32, device)


def rows(heads, device=0):
    return tensor((6, heads, 64), torch.bfloat16, device)


@pytest.mark.parametrize("device", [1, -1])
def test_index_vectors(cache, device):
    k, cu = rows(2), ints(4)
    there = ints(3, device)
    for call in (lambda: cache.append(k, k, ints(4, device)), lambda: cache.append(k, k, cu, seqs=there), lambda: cache.append(k, k, cu, start=there),
                 lambda: cache.evict(there, 2), lambda: cache.release(there), lambda: cache.read(ints(4, device), 6),
                 lambda: cache.read(cu, 6, seqs=there), lambda: cache.read(cu, 6, first=there)):
        with pytest.raises(ValueError, match="the cache's device"):
            call()


@pytest.mark.parametrize("device", [1, -1])
def test_attention(cache, device):
    q, cu, lse = rows(4), ints(4), tensor((6, 4), torch.float32, 0)
    for call in (lambda: cache.attention(q, ints(4, device), 2, out=q, lse=lse), lambda: cache.attention(q, cu, 2, seqs=ints(3, device), out=q, lse=lse),
                 lambda: cache.attention(q, cu, 2, out=q, lse=tensor((6, 4), torch.float32, device)),
                 lambda: cache.attention(rows(4, device), cu, 2, out=q, lse=lse), lambda: cache.attention(q, cu, 2, out=rows(4, device), lse=lse)):
        with pytest.raises(ValueError, match="the cache's device"):
            call()


@pytest.mark.parametrize("name", api.KvCache.BUFFERS)
def test_buffers(monkeypatch, name):
    monkeypatch.setattr(api, "_current_device", lambda: 0)
    shapes = {"k_codes": ((8, 2, 16, 64), torch.uint8), "v_codes": ((8, 2, 16, 64), torch.uint8), "k_scale": ((8, 2), torch.float32),
              "v_scale": ((8, 2), torch.float32), "recent": ((4, 2, 2, 32, 64), torch.bfloat16), "table": ((4, 5), torch.int32),
              "seq_state": ((4, 4), torch.int32), "free_ids": ((8,), torch.int32), "control": ((8,), torch.int32), "weight": ((8,), torch.float32)}
    buffers = {n: tensor(shape, dtype, 1 if n == name else 0) for n, (shape, dtype) in shapes.items()}
    with pytest.raises(ValueError, match=name):
        api.KvCache(n_seqs=4, max_blocks=5, n_blocks=8, n_kv_heads=2, head_dim=64, block_tokens=16, buffers=buffers)
