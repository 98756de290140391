"""A small decoder stack on the framework: attention over an 8-bit key-value
cache, then the slot-addressed MoE layer, layer after layer.

    python examples/decode_stack.py [--steps 64] [--keep 12]

Prompts of different lengths go through in one call a layer (chunk form); then
each step adds one token to every sequence (decode form), the weight that each
block of the cache receives is added up, and a sequence over its budget of
``keep`` blocks gives up the ones that mattered least.  The experts are staged
from pinned host memory into a few slots as the layer's router asks for them.
Random weights; the projections are plain matrix products.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_23805_gb300 import api  # noqa: E402
from paper_2608_23805_gb300 import native as N  # noqa: E402


def norm(x):
    return torch.nn.functional.rms_norm(x, x.shape[-1:])


class Stack:
    def __init__(self, *, layers=2, hidden=256, heads=4, kv_heads=2, head_dim=64, experts=16, top_k=2, inter=128,
                 slots=8, seqs=2, max_tokens=512, block_tokens=16, keep=12, seed=0):
        gen = torch.Generator().manual_seed(seed)

        def normal(*shape, std=1.0):
            return torch.randn(shape, generator=gen) * std

        self.layers, self.heads, self.kv_heads, self.head_dim, self.keep = layers, heads, kv_heads, head_dim, keep
        wide = (heads + 2 * kv_heads) * head_dim
        self.w_qkv = [normal(hidden, wide, std=hidden ** -0.5).cuda().bfloat16() for _ in range(layers)]
        self.w_out = [normal(heads * head_dim, hidden, std=hidden ** -0.5).cuda().bfloat16() for _ in range(layers)]
        self.routers = [normal(experts, hidden, std=0.02).cuda() for _ in range(layers)]
        extent = N.lib().msi_extent_bytes(hidden, inter, N.MSI_W_BF16)
        windows = normal(layers * experts, extent // 2, std=0.05).bfloat16().view(torch.uint8).pin_memory()
        self.plan = api.Plan(n_layers=layers, n_experts=experts, top_k=top_k, hidden=hidden, inter=inter, n_slots=slots,
                             host_windows=windows)
        blocks = -(-max_tokens // block_tokens)
        self.caches = [api.KvCache(n_seqs=seqs, max_blocks=blocks, n_blocks=seqs * blocks, n_kv_heads=kv_heads,
                                   head_dim=head_dim, block_tokens=block_tokens) for _ in range(layers)]

    def step(self, x, cu, max_rows, decode, seen=None):
        """x bf16 [rows, hidden]: rows cu[b] .. cu[b+1] are the next tokens of
        sequence b.  seen(layer, q, k, v, out, lse) looks at each attention."""
        H, K, D = self.heads, self.kv_heads, self.head_dim
        for l, cache in enumerate(self.caches):
            qkv = (norm(x) @ self.w_qkv[l]).view(-1, H + 2 * K, D)  # the cache takes the strided parts as they are
            q, k, v = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
            cache.append(k, v, cu)
            out, lse = cache.attention(q, cu, max_rows, observe=decode)
            if seen is not None:
                seen(l, q, k, v, out, lse)
            x = x + out.reshape(-1, H * D) @ self.w_out[l]
            y, _ = self.plan.forward_streamed(l, norm(x), self.routers[l])
            x = x + y
            if decode:
                cache.evict(cu.numel() - 1, keep=self.keep, sinks=1, recent=2)
        return norm(x)

    def status(self):
        return max(c.status() for c in self.caches)


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=64)
    p.add_argument("--keep", type=int, default=12, help="blocks that a sequence keeps")
    a = p.parse_args()
    prompts = (300, 37)
    stack = Stack(keep=a.keep)
    hidden = stack.w_qkv[0].shape[0]
    gen = torch.Generator("cuda").manual_seed(1)
    cu = torch.tensor([0, prompts[0], sum(prompts)], dtype=torch.int32, device="cuda")
    x = torch.randn((sum(prompts), hidden), device="cuda", generator=gen).bfloat16()
    x = stack.step(x, cu, max(prompts), decode=False)[cu[1:].long() - 1]
    one = torch.arange(len(prompts) + 1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        x = stack.step(x, one, 1, decode=True)
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / max(a.steps, 1)
    status, cache = stack.status(), stack.caches[0]
    print("status %d; %.2f ms a step of %d layers" % (status, 1e3 * t, stack.layers))
    for s, (held, at) in enumerate(cache.seq_state[:, :2].tolist()):
        print("sequence %d: %d tokens seen, %d held" % (s, at, held))
    return 0 if status == 0 and bool(torch.isfinite(x.float()).all()) else 1


if __name__ == "__main__":
    sys.exit(main())
