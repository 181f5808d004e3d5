"""Decode steps of one attention layer in W4A4: the fused query/key/value
projection and the output projection on MixFP4 weights, each with low-rank
adapters of the requests beside it, the new tokens' keys and values appended to
a paged cache with their rotation, and attention over it.

    python examples/decode_step.py [--batch 32] [--context 2048] [--steps 16] [--cache mixfp4|bf16] [--graph]

One step is

    qkv = linear(x, w_qkv);  mixfp4_lora(x, ..., base=qkv, out=qkv)
    q   = mixfp4_kv_append(k, v, cache, slots, q=q, positions=..., cos_sin=...)
    a   = mixfp4_paged_attention(q, cache, block_table, lengths)
    y   = linear(a, w_o);    mixfp4_lora(a, ..., base=y, out=y)

With --graph the steps are replayed from one CUDA graph; slots, positions and
lengths advance on the GPU between them.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_31035_gb300 import ops  # noqa: E402


class Layer:
    """Weights, adapters and paged cache of one attention layer, and the requests in it."""

    def __init__(self, batch, context, steps, hidden=4096, q_heads=32, kv_heads=8, head_dim=128, page=16, rank=16,
                 adapters=4, cache="mixfp4", seed=0, device="cuda:0"):
        g = torch.Generator(device).manual_seed(seed)

        def randn(*shape, std=1.0):
            return torch.randn(*shape, generator=g, device=device) * std
        self.shape = q_heads, kv_heads, head_dim
        width = (q_heads + 2 * kv_heads) * head_dim
        self.w_qkv = ops.mixfp4_quantize(randn(width, hidden, std=0.02).to(torch.bfloat16))
        self.w_o = ops.mixfp4_quantize(randn(hidden, q_heads * head_dim, std=0.02).to(torch.bfloat16))
        self.lora_qkv, self.lora_o = (
            ops.Adapters(randn(adapters, rank, k, std=k ** -0.5).to(torch.bfloat16),
                         randn(adapters, n, rank, std=0.02).to(torch.bfloat16),
                         torch.full((adapters,), 2.0, device=device))
            for k, n in ((hidden, width), (q_heads * head_dim, hidden)))
        # requests: one new token each, some without an adapter, contexts of different lengths
        self.starts = torch.arange(batch + 1, dtype=torch.int32, device=device)
        self.ids = (torch.arange(batch, device=device) % (adapters + 1) - 1).to(torch.int32)
        lengths = torch.randint(context // 2, context + 1, (batch,), generator=g, device=device)
        pages = -(-(context + steps) // page)
        order = torch.randperm(batch * pages, generator=g, device=device)
        self.table = order.view(batch, pages).to(torch.int32)
        scales = {} if cache == "bf16" else dict(k_ts=torch.full((1,), 24.0 / 2688, device=device),
                                                 v_ts=torch.full((1,), 8.0 / 2688, device=device))
        self.cache = ops.empty_kv_cache(batch * pages, page, kv_heads, head_dim, device, **scales)
        at = torch.arange(context + steps, device=device)
        freq = 500000.0 ** (-torch.arange(0, head_dim, 2, device=device, dtype=torch.float64) / head_dim)
        angle = at[:, None] * freq
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float()
        # the prompts' keys and values, as a prefill leaves them: one append of all their tokens
        for b in range(batch):
            n = int(lengths[b])
            slots = self.slots_of(b, at[:n])
            k, v = randn(n, kv_heads, head_dim), randn(n, kv_heads, head_dim)
            ops.mixfp4_kv_append(k, v, self.cache, slots, positions=at[:n], cos_sin=self.cos_sin)
        self.positions = lengths.clone()          # of the tokens to come
        self.lengths = lengths.to(torch.int32)    # of what the cache holds
        self.x = randn(batch, hidden).to(torch.bfloat16)

    def slots_of(self, rows, positions):
        page = self.cache.page_size
        return self.table[rows, positions // page].long() * page + positions % page

    def step(self, x):
        """The layer's output for one new token of every request, float32 [batch, hidden]."""
        q_heads, kv_heads, d = self.shape
        batch = x.shape[0]
        slots = self.slots_of(torch.arange(batch, device=x.device), self.positions)
        qkv = ops.linear(x, self.w_qkv)
        ops.mixfp4_lora(x, self.lora_qkv, self.starts, self.ids, base=qkv, out=qkv)
        q, k, v = (t.unflatten(1, (-1, d)) for t in qkv.split([q_heads * d, kv_heads * d, kv_heads * d], 1))
        q = ops.mixfp4_kv_append(k, v, self.cache, slots, q=q, positions=self.positions, cos_sin=self.cos_sin)
        self.lengths += 1
        self.positions += 1
        a = ops.mixfp4_paged_attention(q, self.cache, self.table, self.lengths).flatten(1)
        y = ops.linear(a, self.w_o)
        return ops.mixfp4_lora(a, self.lora_o, self.starts, self.ids, base=y, out=y)[0]


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--batch", type=int, default=32)
    p.add_argument("--context", type=int, default=2048)
    p.add_argument("--steps", type=int, default=16)
    p.add_argument("--cache", choices=("mixfp4", "bf16"), default="mixfp4")
    p.add_argument("--graph", action="store_true", help="replay the step from a CUDA graph")
    a = p.parse_args(argv)
    layer = Layer(a.batch, a.context, a.steps + 4, cache=a.cache)
    y = layer.step(layer.x)  # warm-up
    run = lambda: layer.step(layer.x)  # noqa: E731
    if a.graph:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            layer.step(layer.x)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = layer.step(layer.x)
        run = graph.replay
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        r = run()
        y = y if a.graph else r
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / a.steps
    held = int(layer.lengths.sum())
    print(f"{a.batch} requests, {held} tokens in the {a.cache} cache: {t * 1e6:.1f} us a step "
          f"({a.batch / t:.0f} tokens/s of this layer), |y| = {float(y.abs().mean()):.4f}")
    return y


if __name__ == "__main__":
    main()
