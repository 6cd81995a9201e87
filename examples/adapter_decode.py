"""A layer and an output head over the library's serving operators: a cache of 4 bits with rotated positions, an adapter of its
own for every request, and the log probabilities of what is answered.

    python examples/adapter_decode.py

admits three prompts, then answers greedily.  Each step is the same eight calls: plan the pages, project to queries, keys and
values, add the requests' adapters, rotate and append, attend, project back, project to the vocabulary, take log probabilities.  The host
reads the chosen tokens and counts pages by itself.  Norms, the feed-forward block and further layers are left out.
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_24519_b200 import binding as b  # noqa: E402
from examples.serving_step import GROUP, quantise_w4  # noqa: E402


def rotary_table(positions: int, dim: int, base: float = 10000.0) -> torch.Tensor:
    """positions x dim FP32: cosines, then sines, of position * base^(-2 i / dim), from 64 bits (an angle of a far position has
    more digits than FP32 holds)."""
    step = torch.exp(torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") * (-math.log(base) / dim))
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * step
    return torch.cat([angle.cos(), angle.sin()], 1).float()


class AdapterModel:
    """Weights, adapters, cache and scratch; every buffer is allocated once."""

    def __init__(self, hidden=512, q_heads=8, heads=2, dim=64, page=16, n_pages=64, requests=3, max_pages=16, max_tokens=64, vocabulary=1000,
                 n_adapters=2, rank=16, alternatives=5, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda *s: torch.empty(s, device="cuda").normal_(generator=g)  # noqa: E731
        self.h = b.awe_create(torch.cuda.current_device())
        self.hidden, self.q_heads, self.heads, self.dim, self.page, self.B = hidden, q_heads, heads, dim, page, requests
        self.max_pages, self.max_tokens, self.n_pages, self.vocabulary, self.alternatives = max_pages, max_tokens, n_pages, vocabulary, alternatives
        self.width = (q_heads + 2 * heads) * dim
        self.embedding = draw(vocabulary, hidden).to(torch.bfloat16)

        def weight(N, K):
            codes, scale = quantise_w4(draw(N, K) * K ** -0.5)
            return b.w4_matrix(codes, scale, b.BF16, None, N, K, K, GROUP)

        self.w_qkv, self.w_out, self.w_head = weight(self.width, hidden), weight(hidden, q_heads * dim), weight(vocabulary, hidden)
        bf16 = dict(dtype=torch.bfloat16, device="cuda")
        self.adapters = b.adapters((draw(n_adapters, rank, hidden) * hidden ** -0.5).to(torch.bfloat16), (draw(n_adapters, self.width, rank) * rank ** -0.5).to(torch.bfloat16),
                                   torch.rand(n_adapters, generator=g, device="cuda") + 0.5, b.BF16, n_adapters, rank, self.width, hidden)
        self.turn = b.rotary(rotary_table(max_pages * page, dim), max_pages * page, dim)
        codes = lambda: torch.zeros((n_pages, heads, page, dim // 2), dtype=torch.uint8, device="cuda")  # noqa: E731
        params = lambda: torch.zeros((n_pages, heads, page), dtype=torch.int16, device="cuda")  # noqa: E731
        self.cache = b.kv4_cache(codes(), codes(), params(), params(), n_pages, heads, page, dim)
        i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(device="cuda")
        self.cached, self.table = torch.zeros(requests, **i32), torch.full((requests, max_pages), -1, **i32)
        self.free = torch.arange(n_pages - 1, -1, -1, **i32)
        self.slots, self.positions = torch.empty(max_tokens, dtype=torch.int64, device="cuda"), torch.empty(max_tokens, **i32)
        self.start, self.ctx, self.counts = torch.empty(requests + 1, **i32), torch.empty(requests, **i32), torch.empty(4, **i32)
        self.qkv, self.mixed = torch.empty((max_tokens, self.width), **bf16), torch.empty((max_tokens, q_heads * dim), **bf16)
        self.rows, self.logits = torch.empty((max_tokens, hidden), **bf16), torch.empty((max_tokens, vocabulary), **f32)
        self.entropy, self.top_logprob = torch.empty(max_tokens, **f32), torch.empty((max_tokens, alternatives), **f32)
        self.top_id = torch.empty((max_tokens, alternatives), **i32)
        n = b.awe_kv4_attention_workspace_bytes(self.h, self.cache, max_tokens, q_heads, requests)
        self.workspace = torch.empty(n, dtype=torch.uint8, device="cuda")
        self.lengths = [0] * requests  # the host's own count, for the free list

    def step(self, x: torch.Tensor, new_lengths: list[int], adapter: torch.Tensor):
        """x: the new tokens' rows (request by request), T x hidden BF16; adapter: a number for each request, -1 for none.  Returns the
        most likely next tokens of every row and their log probabilities, T x alternatives."""
        T, h, D = x.shape[0], self.h, self.dim
        assert T == sum(new_lengths) <= self.max_tokens
        new = torch.tensor(new_lengths, dtype=torch.int32).pin_memory().to("cuda", non_blocking=True)
        b.awe_kv_plan(h, self.cached, new, self.B, self.page, self.free, self.free.numel(), self.table, self.max_pages, self.max_pages,
                      self.slots, self.positions, T, self.start, self.ctx, self.counts)
        b.awe_linear_w4(h, self.w_qkv, x, b.BF16, T, x.stride(0), self.qkv, b.BF16, self.width)
        b.awe_linear_adapters(h, self.adapters, x, T, x.stride(0), self.start, adapter, self.B, self.qkv, self.width, self.qkv, b.BF16, self.width)
        keys, values = self.qkv[:, self.q_heads * D:], self.qkv[:, (self.q_heads + self.heads) * D:]
        b.awe_kv4_append(h, self.cache, self.turn, b.BF16, T, self.q_heads, self.qkv, self.width, keys, self.width, values, self.width, self.positions,
                         self.slots, self.qkv, self.width)
        b.awe_kv4_attention(h, self.cache, self.qkv, b.BF16, T, self.q_heads, self.width, self.start, self.ctx, self.B, self.table,
                            self.max_pages, self.max_pages, D ** -0.5, True, 0, self.mixed, self.q_heads * D, None, self.workspace)
        b.awe_linear_w4(h, self.w_out, self.mixed, b.BF16, T, self.q_heads * D, self.rows, b.BF16, self.hidden)
        b.awe_linear_w4(h, self.w_head, self.rows, b.BF16, T, self.hidden, self.logits, b.F32, self.vocabulary)
        b.awe_token_logprobs(h, self.logits, b.F32, T, self.vocabulary, self.vocabulary, 1.0, None, None, self.entropy, None, self.alternatives,
                             self.top_logprob, self.top_id)
        # what the next step starts from
        pages = lambda n: -(-n // self.page)  # noqa: E731
        self.free = self.free[sum(pages(a + n) - pages(a) for a, n in zip(self.lengths, new_lengths)):]
        self.lengths = [a + n for a, n in zip(self.lengths, new_lengths)]
        self.cached.copy_(self.ctx)
        return self.top_id[:T], self.top_logprob[:T]


def main() -> None:
    model = AdapterModel()
    g = torch.Generator(device="cuda").manual_seed(1)
    adapter = torch.tensor([0, -1, 1], dtype=torch.int32, device="cuda")
    prompts = [20, 1, 33]
    tokens = torch.randint(0, model.vocabulary, (sum(prompts),), generator=g, device="cuda")
    ids, logprob = model.step(model.embedding[tokens], prompts, adapter)
    last = torch.tensor(prompts, device="cuda").cumsum(0) - 1
    total = logprob[last, 0].clone()
    for _ in range(10):
        ids, logprob = model.step(model.embedding[ids[last, 0].long()], [1, 1, 1], adapter)
        last = torch.arange(3, device="cuda")
        total += logprob[:, 0]
    torch.cuda.synchronize()
    assert b.awe_last_device_status(model.h) == (0, 0) and bool(torch.isfinite(total).all())
    print(f"answered 11 tokens each after {prompts}: log probabilities {[round(v, 2) for v in total.tolist()]}, "
          f"{b.awe_launch_count(model.h)} kernels launched, {model.free.numel()} pages left")


if __name__ == "__main__":
    main()
