"""One attention layer of a quantised decoder over a paged 4-bit key/value cache.

A batch of requests of different lengths runs its prompts, then single tokens;
requests come and go, their pages taken from and returned to a ring on the GPU.
Per step: the q/k/v projections (logq_linear_grouped), rotary positions, the
step's bookkeeping (logq_kv_plan), the cache write (logq_kv_append), attention
(logq_kv_attention) and the output projection (logq_linear).

    python examples/paged_decode.py [--steps 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_01127_gb300 as logq  # noqa: E402
from paper_2607_01127_gb300 import workloads  # noqa: E402


class Layer:
    """Attention layer with the Llama-3.2-1B shapes: 32 query and 8 kv heads of 64."""
    HEADS, KV_HEADS, DIM = 32, 8, 64

    def __init__(self, requests: int, pages: int = 256, page_size: int = 16, base: float = 1.5, seed: int = 0):
        self.weights = {}
        for i, name in enumerate(("q", "k", "v", "o")):
            n, k = workloads.LLAMA_1B_SHAPES[name]
            w = workloads.weights_torch(n, k, workloads.layer_seed(1, seed, i), device="cuda")
            self.weights[name] = (*logq.logq_quantize(w, 4, base), n, k)
        self.cache = logq.new_kv_cache(pages, page_size, self.KV_HEADS, self.DIM, torch.bfloat16, base)
        self.workspace = logq.new_workspace()
        self.attention_workspace = logq.new_kv_workspace(self.HEADS, self.KV_HEADS, self.DIM)
        self.block_table = torch.full((requests, 32), -1, dtype=torch.int32, device="cuda")
        self.ring = torch.arange(pages, dtype=torch.int32, device="cuda")
        self.ring_state = torch.tensor([0, pages], dtype=torch.int32, device="cuda")

    def rotate(self, x, positions):
        """Rotary position embedding of [tokens, heads, dim]."""
        half = self.DIM // 2
        freq = 1e4 ** (-torch.arange(half, device=x.device) / half)
        angle = positions.clamp(min=0).float()[:, None, None] * freq
        a, b = x.float().chunk(2, -1)
        return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1).to(x.dtype)

    def step(self, x, ctx_len, new_len, max_q: int):
        """x [tokens, hidden] bf16: the requests' new tokens, request after request.  Returns the
        layer's output and (q, attention's output, q_start, kv_len)."""
        tokens, hidden = x.shape
        items = [(c, cb, n, None) for c, cb, n, _ in (self.weights[p] for p in "qkv")]
        q, k, v = logq.logq_linear_grouped(items, x, hidden, torch.bfloat16)
        q_start, kv_len, positions, slots, _ = logq.logq_kv_plan(
            ctx_len, new_len, self.block_table, self.ring, self.ring_state, self.cache.page_size, tokens,
            workspace=self.workspace)
        q = self.rotate(q.view(tokens, self.HEADS, self.DIM), positions)
        k = self.rotate(k.view(tokens, self.KV_HEADS, self.DIM), positions)
        logq.logq_kv_append(self.cache, k, v.view(tokens, self.KV_HEADS, self.DIM), slots)
        out = logq.logq_kv_attention(self.cache, q, q_start, kv_len, self.block_table, max_q=max_q,
                                     workspace=self.attention_workspace)
        codes, cb, n, k_in = self.weights["o"]
        y = logq.logq_linear(codes, cb, out.view(tokens, -1), n, k_in, torch.bfloat16)
        return y, (q, out, q_start, kv_len)


def run(prompts=(40, 3, 117, 64), steps: int = 8, check=None):
    """Prompts, then single tokens; half way the first request ends and another takes its place.
    check(layer, q, out, q_start, kv_len, block_table) is called after every step."""
    layer = Layer(len(prompts))
    hidden = layer.HEADS * layer.DIM
    gen = torch.Generator(device="cuda").manual_seed(0)
    requests, page = len(prompts), layer.cache.page_size
    ctx = torch.zeros(requests, dtype=torch.int32, device="cuda")
    lengths = list(prompts)
    for i in range(steps + 1):
        if i:
            lengths = [1] * requests
        if i == steps // 2 + 1:                            # the first request ends: its pages go back ...
            done = torch.tensor([-1] + [0] * (requests - 1), dtype=torch.int32, device="cuda")
            logq.logq_kv_plan(ctx, done, layer.block_table, layer.ring, layer.ring_state, page, 0, workspace=layer.workspace)
            ctx[0] = 0
            lengths[0] = 25                                # ... and a new prompt takes its place
        new = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        x = torch.randn(sum(lengths), hidden, generator=gen, device="cuda").to(torch.bfloat16)
        y, (q, out, q_start, kv_len) = layer.step(x, ctx, new, max(lengths))
        if check is not None:
            check(layer, q, out, q_start, kv_len, layer.block_table)
        ctx = kv_len.clone()
    status, detail = logq.logq_workspace_status(layer.attention_workspace)
    assert status == logq.LOGQ_OK, (status, detail)
    return y, ctx, layer


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args()
    y, ctx, layer = run(steps=a.steps)
    cache = layer.cache
    used = layer.cache.pages - int(layer.ring_state[1])
    bits = 8 * (cache.k_codes[0].numel() + 2 * cache.k_range[0].numel()) / (cache.heads * cache.page_size * cache.head_dim)
    print(f"cached tokens per request {ctx.tolist()}, {used} of {cache.pages} pages in use, "
          f"{bits:.2f} bits per cached value, output {tuple(y.shape)} rms {float(y.float().square().mean().sqrt()):.3f}")
