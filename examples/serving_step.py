"""One attention layer of a language model over the library's serving operators: 4-bit projections, a paged
cache of 8-bit keys and values.

    python examples/serving_step.py

admits three prompts, then decodes some tokens.  Each step is the same five calls (plan the pages, project to queries, keys
and values, write the cache, attend, project back); the host never waits for the GPU in between, and counts pages by
itself.  Rotary positions, norms and the rest of a model are left out.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_24519_b200 import binding as b  # noqa: E402

GROUP = 64  # values of k that share a scale


def quantise_w4(w: torch.Tensor):
    """N x K weights -> (codes, scales): per row and group of 64 the largest magnitude becomes 7 (or -7)."""
    N, K = w.shape
    x = w.float().view(N, K // GROUP, GROUP)
    scale = (x.abs().amax(2) / 7).clamp(min=1e-8).to(torch.bfloat16)
    q = (x / scale.float()[..., None]).round().clamp(-8, 7).to(torch.int8).view(N, K)
    return ((q[:, 0::2] & 15) | (q[:, 1::2] << 4)).view(torch.uint8).contiguous(), scale


class AttentionLayer:
    """Weights, cache and scratch of one layer; every buffer is allocated once."""

    def __init__(self, hidden=512, q_heads=8, heads=2, dim=64, page=16, n_pages=64, requests=3, max_pages=16, max_tokens=64, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.h = b.awe_create(torch.cuda.current_device())
        self.hidden, self.q_heads, self.heads, self.dim, self.page, self.B = hidden, q_heads, heads, dim, page, requests
        self.max_pages, self.max_tokens, self.n_pages = max_pages, max_tokens, n_pages
        self.width = (q_heads + 2 * heads) * dim
        self.tensors = []

        def weight(N, K):
            w = torch.empty((N, K), device="cuda").normal_(generator=g) * K ** -0.5
            codes, scale = quantise_w4(w)
            return b.w4_matrix(codes, scale, b.BF16, None, N, K, K, GROUP)

        self.w_qkv, self.w_out = weight(self.width, hidden), weight(hidden, q_heads * dim)
        i8 = dict(dtype=torch.int8, device="cuda")
        self.cache = b.kv_cache(torch.zeros((n_pages, heads, page, dim), **i8), torch.zeros((n_pages, heads, page, dim), **i8),
                                torch.zeros((n_pages, heads), device="cuda"), torch.zeros((n_pages, heads), device="cuda"),
                                n_pages, heads, page, dim)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.cached, self.table = torch.zeros(requests, **i32), torch.full((requests, max_pages), -1, **i32)
        self.free = torch.arange(n_pages - 1, -1, -1, **i32)
        self.slots = torch.empty(max_tokens, dtype=torch.int64, device="cuda")
        self.start, self.ctx, self.counts = torch.empty(requests + 1, **i32), torch.empty(requests, **i32), torch.empty(4, **i32)
        self.qkv = torch.empty((max_tokens, self.width), dtype=torch.bfloat16, device="cuda")
        self.mixed = torch.empty((max_tokens, q_heads * dim), dtype=torch.bfloat16, device="cuda")
        n = b.awe_kv_attention_workspace_bytes(self.h, self.cache, max_tokens, q_heads, requests)
        self.workspace = torch.empty(n, dtype=torch.uint8, device="cuda")
        self.lengths = [0] * requests  # the host's own count, for the free list

    def step(self, x: torch.Tensor, new_lengths: list[int]) -> torch.Tensor:
        """x: the new tokens' rows (request by request), T x hidden BF16.  Returns T x hidden."""
        T, h, D = x.shape[0], self.h, self.dim
        assert T == sum(new_lengths) <= self.max_tokens
        new = torch.tensor(new_lengths, dtype=torch.int32).pin_memory().to("cuda", non_blocking=True)
        b.awe_kv_plan(h, self.cached, new, self.B, self.page, self.free, self.free.numel(), self.table, self.max_pages, self.max_pages,
                      self.slots, None, T, self.start, self.ctx, self.counts)
        b.awe_linear_w4(h, self.w_qkv, x, b.BF16, T, x.stride(0), self.qkv, b.BF16, self.width)
        keys, values = self.qkv[:, self.q_heads * D:], self.qkv[:, (self.q_heads + self.heads) * D:]
        b.awe_kv_write(h, self.cache, keys, values, b.BF16, T, self.width, self.width, self.slots)
        b.awe_kv_attention(h, self.cache, self.qkv, b.BF16, T, self.q_heads, self.width, self.start, self.ctx, self.B, self.table,
                           self.max_pages, self.max_pages, D ** -0.5, True, 0, self.mixed, self.q_heads * D, None, self.workspace)
        y = torch.empty((T, self.hidden), dtype=torch.bfloat16, device="cuda")
        b.awe_linear_w4(h, self.w_out, self.mixed, b.BF16, T, self.q_heads * D, y, b.BF16, self.hidden)
        # what the next step starts from
        pages = lambda n: -(-n // self.page)  # noqa: E731
        taken = sum(pages(a + n) - pages(a) for a, n in zip(self.lengths, new_lengths))
        self.free = self.free[taken:]
        self.lengths = [a + n for a, n in zip(self.lengths, new_lengths)]
        self.cached.copy_(self.ctx)
        return y


def main() -> None:
    layer = AttentionLayer()
    g = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda T: torch.empty((T, layer.hidden), device="cuda").normal_(generator=g).to(torch.bfloat16)  # noqa: E731
    prompts = [20, 1, 33]
    y = layer.step(draw(sum(prompts)), prompts)
    for _ in range(10):
        y = layer.step(draw(3), [1, 1, 1])
    torch.cuda.synchronize()
    assert b.awe_last_device_status(layer.h) == (0, 0) and bool(torch.isfinite(y).all())
    print(f"served {layer.lengths} tokens, {b.awe_launch_count(layer.h)} kernels launched, {layer.free.numel()} pages left")


if __name__ == "__main__":
    main()
