"""One verification step of a small target model over a paged cache, from drafted trees to stages.

    python examples/verify_step.py

Every sample holds cached tokens and drafts a tree.  One attention layer (projections by torch.matmul, everything between
them by the library) gives the hidden states of the drafted tokens; the LM head scores them; the scores are ranked against
the calibration buffer; the attention that cached slots received decides what stays when a cache is over its budget."""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_15148_b200 import binding  # noqa: E402


class Target:
    """Weights of the layer and the LM head, and the buffers that a serving loop keeps from step to step."""

    def __init__(self, hidden=512, heads=8, kv_heads=2, head_dim=64, vocab=4000, seed=0, scaling="none"):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[-1] ** -0.5).to(torch.bfloat16)  # noqa: E731
        self.heads, self.kv_heads, self.head_dim, self.vocab = heads, kv_heads, head_dim, vocab
        self.w_qkv, self.w_out = w((heads + 2 * kv_heads) * head_dim, hidden), w(hidden, heads * head_dim)
        self.lm_head = w(vocab, hidden)
        freqs, self.mscale = binding.rope_freqs(head_dim, 500000.0, scaling, 8.0)
        self.freqs = freqs.cuda()
        self.scale = head_dim ** -0.5

    def new_cache(self, samples: int, slots: int, page_size: int = 16) -> binding.PagedCache:
        pages = -(-slots // page_size)
        k, v = (torch.zeros(samples * pages, page_size, self.kv_heads, self.head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        table = torch.randperm(samples * pages).int().view(samples, pages).cuda()
        return binding.PagedCache(k, v, table)

    def attend(self, x, cache, ctx_lens, positions, cu_tokens, pre, end, max_tokens: int, max_len: int):
        """x [M, hidden] -> (hidden states [M, hidden], q, lse); keys and values of the drafted tokens are in the cache after it."""
        M, D = x.shape[0], self.head_dim
        q, k, v = (t.unflatten(1, (-1, D)) for t in (x @ self.w_qkv.T).split([self.heads * D, self.kv_heads * D, self.kv_heads * D], dim=1))
        rotated, out = torch.empty(M, self.heads, D, dtype=x.dtype, device="cuda"), torch.empty(M, self.heads, D, dtype=x.dtype, device="cuda")
        lse = torch.empty(M, self.heads, device="cuda")
        binding.rope_append(q, k, v, positions, self.freqs, cache, ctx_lens, cu_tokens, max_tokens, rotated, mscale=self.mscale)
        need = binding.tree_attention_workspace_bytes(cache.num_seqs, M, self.heads, self.kv_heads, D, max_tokens, max_len)
        work = torch.empty(need, dtype=torch.uint8, device="cuda")
        binding.tree_attention(rotated, cache, ctx_lens, cu_tokens, pre, end, max_tokens, max_len, self.scale, out, lse, work)
        return x + out.flatten(1) @ self.w_out.T, rotated, lse


def verify_step(target: Target, cache, ctx_lens, next_position, x, parent, token_ids, cu_tokens, calib, n: int, alpha: float, weights):
    """Scores the drafted trees of all samples: x [M, hidden] their embeddings, parent and cu_tokens (host) the trees, token_ids
    [M] what each token's hidden state has to predict, calib the sorted calibration buffer with n entries.  Returns the
    scores, stages and what the step computed on the way; the cache holds the drafts behind ctx_lens, `weights` [samples, kv
    heads, slots] grows by the attention that slots received."""
    pre, end, depth = binding.tree_plan(parent, cu_tokens)
    cu_host = torch.as_tensor(cu_tokens, dtype=torch.int32)
    tokens = cu_host[1:] - cu_host[:-1]
    samples, M = tokens.numel(), int(cu_host[-1])
    pre, end, cu = pre.cuda(), end.cuda(), cu_host.cuda()
    positions = (torch.repeat_interleave(next_position.cpu(), tokens) + depth).int().cuda()
    max_tokens, max_len = int(tokens.max()), int((ctx_lens.cpu() + tokens).max())
    hidden, q, lse = target.attend(x, cache, ctx_lens, positions, cu, pre, end, max_tokens, max_len)
    logprob, score = torch.empty(M, device="cuda"), torch.empty(samples, device="cuda")
    work = torch.empty(binding.score_workspace_bytes(M, hidden.shape[1], target.vocab, samples), dtype=torch.uint8, device="cuda")
    binding.score_logprob(hidden, target.lm_head, token_ids, cu, logprob, score, work)
    numer, pvalue = torch.empty(samples, dtype=torch.int32, device="cuda"), torch.empty(samples, device="cuda")
    stage, counts = torch.empty(samples, dtype=torch.uint8, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    binding.rank_classify(score, calib, n, [alpha], numer, pvalue, stage, counts)
    binding.cache_weights(q, cache, lse, ctx_lens, cu, pre, end, max_tokens, max_len, target.scale, weights, weights)
    return {"hidden": hidden, "logprob": logprob, "score": score, "pvalue": pvalue, "stage": stage, "counts": counts, "positions": positions}


def evict(target: Target, cache, lens, weights, budget: int, sinks: int = 4, recent: int = 32, room: int = 256):
    """Cuts every sample's cache to `budget` slots: (new cache with `room` slots to spare, its lengths, its weights)."""
    samples, heads, slots = weights.shape
    kept = torch.empty(samples, heads, budget, dtype=torch.int32, device="cuda")
    counts = torch.empty(samples, dtype=torch.int32, device="cuda")
    binding.cache_select(weights, lens, budget, sinks, recent, kept, counts)
    smaller = target.new_cache(samples, budget + room)
    left = torch.zeros(samples, heads, slots, device="cuda")
    kept_weights = torch.empty(samples, heads, budget, device="cuda")
    binding.cache_gather(cache, kept, counts, smaller, weights, kept_weights)
    left[..., :budget] = kept_weights
    return smaller, counts, left


def main() -> None:
    torch.manual_seed(100)      # (not the seed of the weights: the embeddings would be rows of the LM head)
    target = Target()
    samples, drafts, slots, budget, alpha = 6, 20, 512, 128, 0.25
    cache = target.new_cache(samples, slots)
    lens = torch.zeros(samples, dtype=torch.int32, device="cuda")
    at = torch.zeros(samples, dtype=torch.int32)
    weights = torch.zeros(samples, target.kv_heads, slots, device="cuda")
    calib, n = torch.sort(torch.randn(256, device="cuda") * 0.1 + 8.6)[0], 256
    for turn in range(8):
        # a draft that continues the sample, and a second branch from its middle
        parent = list(range(-1, drafts - 1)) + [drafts // 2] + list(range(drafts, drafts + 4))
        T = len(parent)
        cu = [T * s for s in range(samples + 1)]
        x = torch.randn(samples * T, target.w_qkv.shape[1], device="cuda").bfloat16()
        ids = torch.randint(0, target.vocab, (samples * T,), dtype=torch.int32, device="cuda")
        r = verify_step(target, cache, lens, at, x, parent * samples, ids, cu, calib, n, alpha, weights)
        # the first branch is kept: its slots are the first `drafts` behind the cache
        lens = lens + drafts
        at = at + drafts
        weights[..., int(lens.max()):] = 0
        print(f"turn {turn}: scores {[round(s, 2) for s in r['score'].tolist()]} stages {r['stage'].tolist()} slots {lens.tolist()}")
        if int(lens.max()) > budget:
            cache, lens, weights = evict(target, cache, lens, weights, budget)
            print(f"         caches cut to {lens.tolist()} slots")
    if binding.last_device_status() != 0:
        raise SystemExit("the device recorded a condition")


if __name__ == "__main__":
    main()
