"""Speculative decoding steps of one attention layer in W4A4: a tree of drafted
tokens per request is verified at once, what is accepted stays in the paged cache,
and requests may branch.

    python examples/speculative_step.py [--batch 16] [--context 2048] [--drafts 8] [--steps 8] [--cache mixfp4|bf16]
                                        [--softcap 0]

One step is

    qkv = linear(x, w_qkv)                                           # of all drafts
    q   = mixfp4_kv_append(k, v, cache, slots, q=q, positions=..., cos_sin=...)
    a   = mixfp4_tree_attention(q, cache, block_table, lengths, mask=mask)
    y   = linear(a, w_o)
    lengths = mixfp4_kv_accept(cache, block_table, lengths, path, counts)

Slots follow the drafts' order; positions follow the tree: a draft stands behind
its ancestors.  Which drafts are accepted would come from the model's head; here it
is a random path from the root.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_31035_gb300 import ops  # noqa: E402


def random_trees(batch, t, g):
    """Parents int64 [batch, t] (-1: the root's) and ancestor masks int64 [batch, t], on the host."""
    parents = torch.full((batch, t), -1)
    mask = torch.zeros(batch, t, dtype=torch.int64)
    for i in range(t):
        if i:
            parents[:, i] = torch.randint(max(0, i - 4), i, (batch,), generator=g)
            mask[:, i] = mask.gather(1, parents[:, i:i + 1]).squeeze(1)
        mask[:, i] |= (1 << i) if i < 63 else -1 << 63
    return parents, mask


def branch_pages(own, lengths, parents, page):
    """Of children with pages own[i] (int32 [n, width]) and parents' lengths: the page that takes the parent's last one if
    that is filled in part (-1: none is), and the first of the child's columns that are its own."""
    length = lengths[parents.long()].long()
    part = length // page  # the table's width where the parent has filled it
    fresh = own.gather(1, part.clamp(max=own.shape[1] - 1)[:, None]).squeeze(1)
    return torch.where(length % page > 0, fresh, -1).to(torch.int32), part


class Layer:
    """Weights and paged cache of one attention layer, and the requests in it."""

    def __init__(self, batch, context, room, hidden=2048, q_heads=16, kv_heads=4, head_dim=128, page=16, cache="mixfp4",
                 softcap=0.0, seed=0, device="cuda:0"):
        g = torch.Generator(device).manual_seed(seed)

        def randn(*shape, std=1.0):
            return torch.randn(*shape, generator=g, device=device) * std
        self.shape, self.softcap, self.page = (q_heads, kv_heads, head_dim), softcap, page
        self.w_qkv = ops.mixfp4_quantize(randn((q_heads + 2 * kv_heads) * head_dim, hidden, std=0.02).to(torch.bfloat16))
        self.w_o = ops.mixfp4_quantize(randn(hidden, q_heads * head_dim, std=0.02).to(torch.bfloat16))
        width = -(-(context + room) // page)
        scales = {} if cache == "bf16" else dict(k_ts=torch.full((1,), 24.0 / 2688, device=device),
                                                 v_ts=torch.full((1,), 8.0 / 2688, device=device))
        # pages for the requests and for twice as many branches
        self.cache = ops.empty_kv_cache(3 * batch * width, page, kv_heads, head_dim, device, **scales)
        order = torch.randperm(3 * batch * width, generator=g, device=device).to(torch.int32)
        self.table, self.spare = order[:batch * width].view(batch, width).contiguous(), order[batch * width:]
        self.lengths = torch.randint(context // 2, context + 1, (batch,), generator=g, device=device).to(torch.int32)
        at = torch.arange(context + room, device=device)
        freq = 500000.0 ** (-torch.arange(0, head_dim, 2, device=device, dtype=torch.float64) / head_dim)
        self.cos_sin = torch.cat([(at[:, None] * freq).cos(), (at[:, None] * freq).sin()], 1).float()
        for b in range(batch):
            n = int(self.lengths[b])
            k, v = randn(n, kv_heads, head_dim), randn(n, kv_heads, head_dim)
            ops.mixfp4_kv_append(k, v, self.cache, self.slots(b, at[:n]), positions=at[:n], cos_sin=self.cos_sin)

    def slots(self, rows, places):
        return self.table[rows, places // self.page].long() * self.page + places % self.page

    def project(self, x):
        """Queries, keys and values of all drafts, float32 [batch, t, heads, head_dim] each, keys and queries unturned.
        The activations of one call share a scale, so the same draft in another batch may round to other codes."""
        q_heads, kv_heads, d = self.shape
        qkv = ops.linear(x.flatten(0, 1), self.w_qkv).unflatten(0, x.shape[:2])
        return [y.unflatten(2, (-1, d)) for y in qkv.split([q_heads * d, kv_heads * d, kv_heads * d], 2)]

    def attend(self, q, k, v, mask):
        """Attention of all drafts, bfloat16 [batch, t, q_heads, head_dim]; the cache holds their rows from now on."""
        batch, t = q.shape[:2]
        i = torch.arange(t, device=q.device)
        seen = (mask[..., None] >> i) & 1
        first = self.lengths.long()[:, None]
        slots = self.slots(torch.arange(batch, device=q.device)[:, None], first + i).reshape(-1)
        positions = (first + seen.sum(-1) - 1).reshape(-1)  # behind the ancestors; the mask has the draft itself
        q = ops.mixfp4_kv_append(k.flatten(0, 1), v.flatten(0, 1), self.cache, slots, q=q.flatten(0, 1), positions=positions,
                                 cos_sin=self.cos_sin)
        self.lengths += t
        return ops.mixfp4_tree_attention(q.unflatten(0, (batch, t)), self.cache, self.table, self.lengths, mask=mask,
                                         softcap=self.softcap)

    def verify(self, x, mask):
        """The layer's output for all drafts, float32 [batch, t, hidden]."""
        a = self.attend(*self.project(x), mask)
        return ops.linear(a.flatten(2).flatten(0, 1), self.w_o).unflatten(0, x.shape[:2])

    def accept(self, path, t):
        """Of the last t drafts of each request, those on its path stay (int32 [batch, depth], ended by -1)."""
        counts = torch.full_like(self.lengths, t)
        ops.mixfp4_kv_accept(self.cache, self.table, self.lengths, path, counts, out=self.lengths)

    def branch(self, parents):
        """Requests from now on: child i goes on from request parents[i] (int32); full pages are shared, and what comes
        next goes to pages of its own."""
        n, width = parents.numel(), self.table.shape[1]
        if self.spare.numel() < n * width:
            raise ValueError(f"{n} branches want {n * width} pages, {self.spare.numel()} are left")
        own, self.spare = self.spare[:n * width].view(n, width), self.spare[n * width:]
        fresh, part = branch_pages(own, self.lengths, parents, self.page)
        table, self.lengths = ops.mixfp4_kv_fork(self.cache, self.table, self.lengths, parents, fresh)
        later = torch.arange(width, device=table.device) >= part[:, None]
        self.table = torch.where(later, own, table)


def random_path(parents, t, g):
    """A way down from the root of each tree, as many drafts as it has: int32 [batch, t], ended by -1."""
    batch = parents.shape[0]
    path = torch.full((batch, t), -1, dtype=torch.int32)
    for b in range(batch):
        at, k = 0, 0
        while True:
            path[b, k] = at
            k += 1
            children = [i for i in range(at + 1, t) if int(parents[b, i]) == at]
            if not children or torch.rand(1, generator=g) < 0.2:
                break
            at = children[int(torch.randint(len(children), (1,), generator=g))]
    return path


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--batch", type=int, default=16)
    p.add_argument("--context", type=int, default=2048)
    p.add_argument("--drafts", type=int, default=8)
    p.add_argument("--steps", type=int, default=8)
    p.add_argument("--cache", choices=("mixfp4", "bf16"), default="mixfp4")
    p.add_argument("--softcap", type=float, default=0.0)
    a = p.parse_args(argv)
    g = torch.Generator().manual_seed(1)
    layer = Layer(a.batch, a.context, a.steps * a.drafts + a.drafts, cache=a.cache, softcap=a.softcap)
    trees = [random_trees(a.batch, a.drafts, g) for _ in range(a.steps)]
    paths = [random_path(parents, a.drafts, g).to("cuda:0") for parents, _ in trees]
    masks = [mask.to("cuda:0") for _, mask in trees]
    x = torch.randn(a.batch, a.drafts, layer.w_qkv.codes.shape[1] * 2, device="cuda:0").to(torch.bfloat16)
    before = int(layer.lengths.sum())
    torch.cuda.synchronize()
    t = time.perf_counter()
    for mask, path in zip(masks, paths):
        y = layer.verify(x, mask)
        layer.accept(path, a.drafts)
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / a.steps
    kept = int(layer.lengths.sum()) - before
    print(f"{a.batch} requests, {a.drafts} drafts each, {a.cache} cache: {t * 1e6:.1f} us a step, "
          f"{kept / a.steps / a.batch:.2f} tokens kept of each request, |y| = {float(y.abs().mean()):.4f}")
    return y


if __name__ == "__main__":
    main()
