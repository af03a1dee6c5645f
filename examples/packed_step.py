"""Verification steps of a target layer with head norms and a sliding window over a cache in 4 bits, sixteen samples side by side.

    python examples/packed_step.py

Every turn each sample drafts a tree; queries and keys are normed per head and rotated (norm_rope), keys and values go into the packed
cache (packed_append), the tree is attended to through the window (packed_attention).  The longest branch is kept, and pages
that have fallen out of the window, but for the sinks', go back to the pool: a sample's cache stops growing."""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_15148_b200 import binding  # noqa: E402


class PackedLayer:
    """Weights of one layer, its packed cache for `samples` sequences of up to `slots` slots, and the pages that are free."""

    def __init__(self, samples=16, slots=1024, pages=160, page_size=16, hidden=512, heads=8, kv_heads=2, head_dim=64, window=96, sinks=4, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[-1] ** -0.5).to(torch.bfloat16)  # noqa: E731
        self.heads, self.kv_heads, self.head_dim, self.window, self.sinks, self.page_size = heads, kv_heads, head_dim, window, sinks, page_size
        self.w_qkv, self.w_out = w((heads + 2 * kv_heads) * head_dim, hidden), w(hidden, heads * head_dim)
        self.q_gain, self.k_gain = (1 + 0.2 * torch.randn(2, head_dim, generator=g, device="cuda")).to(torch.bfloat16)
        self.freqs = binding.rope_freqs(head_dim, 500000.0)[0].cuda()
        self.scale, self.eps = head_dim ** -0.5, 1e-6
        block = binding.packed_block_bytes(page_size, head_dim)
        k, v = (torch.zeros(pages, kv_heads, block, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.table = torch.full((samples, slots // page_size), -1, dtype=torch.int32)      # kept on the host, copied where it changes
        self.cache = binding.PackedCache(k, v, self.table.cuda(), page_size, head_dim)
        self.free, self.lens = list(range(pages)), torch.zeros(samples, dtype=torch.int32)

    def reserve(self, drafts: int) -> None:
        """Pages for `drafts` more slots of every sample."""
        for b, n in enumerate(self.lens.tolist()):
            for c in range(-(-n // self.page_size), -(-(n + drafts) // self.page_size)):
                if self.table[b, c] < 0:
                    self.table[b, c] = self.free.pop()
        self.cache.block_table.copy_(self.table)

    def release(self) -> None:
        """Pages of which no token to come sees anything go back."""
        for b, n in enumerate(self.lens.tolist()):
            for c in range(-(-self.sinks // self.page_size), max(0, n - self.window + 1) // self.page_size):
                if self.table[b, c] >= 0:
                    self.free.append(int(self.table[b, c]))
                    self.table[b, c] = -1

    def step(self, x, parent, cu):
        """x [M, hidden], the drafted trees (host) -> (hidden states [M, hidden], rotated q, k, v, attention, lse)."""
        pre, end, depth = binding.tree_plan(parent, cu)
        cu = torch.as_tensor(cu, dtype=torch.int32)
        tokens = cu[1:] - cu[:-1]
        M, most, longest = int(cu[-1]), int(tokens.max()), int((self.lens + tokens).max())
        self.reserve(most)
        q, k, v = (t.unflatten(1, (-1, self.head_dim)) for t in (x @ self.w_qkv.T).split([n * self.head_dim for n in (self.heads, self.kv_heads, self.kv_heads)], dim=1))
        positions = (torch.repeat_interleave(self.lens, tokens) + depth).int().cuda()
        pre, end, depth, cu, lens = (t.cuda() for t in (pre, end, depth, cu, self.lens))
        q2, k2, out = torch.empty(M, self.heads, self.head_dim, dtype=x.dtype, device="cuda"), torch.empty_like(k, memory_format=torch.contiguous_format), None
        binding.norm_rope(q, k, positions, self.freqs, self.q_gain, self.k_gain, self.eps, q2, k2)
        binding.packed_append(k2, v, self.cache, lens, cu, most)
        out, lse = torch.empty_like(q2), torch.empty(M, self.heads, device="cuda")
        need = binding.packed_attention_workspace_bytes(self.cache.num_seqs, M, self.heads, self.kv_heads, self.head_dim, most, longest, self.window, self.sinks)
        work = torch.empty(need, dtype=torch.uint8, device="cuda")
        binding.packed_attention(q2, self.cache, lens, cu, pre, end, depth, self.window, self.sinks, most, longest, self.scale, out, lse, work)
        return x + out.flatten(1) @ self.w_out.T, q2, k2, v, out, lse


def main() -> None:
    torch.manual_seed(100)
    layer = PackedLayer()
    samples, line = layer.lens.numel(), 20
    parent = list(range(-1, line - 1)) + [line // 2, line, line + 1]        # a line of 20 and a branch of three from its middle
    for turn in range(24):
        cu = [len(parent) * b for b in range(samples + 1)]
        x = torch.randn(samples * len(parent), layer.w_qkv.shape[1], device="cuda").bfloat16()
        h = layer.step(x, parent * samples, cu)[0]
        layer.lens += line                                                  # the line is kept: its slots are the first behind the cache
        layer.release()
        print(f"turn {turn}: slots {int(layer.lens[0])}, pages held {160 - len(layer.free)}, |h| {h.float().norm(dim=1).mean().item():.2f}")
    if binding.last_device_status() != 0:
        raise SystemExit("the device recorded a condition")


if __name__ == "__main__":
    main()
