"""Drafted decoding as it is used: append, attention over the trees, acceptance, the next step, a fork.  Each
draft's output is that of decoding its ancestors one token at a time, and the cache afterwards is the one that
decoding the accepted tokens alone leaves."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda:0"


@pytest.fixture(scope="module")
def step():
    spec = importlib.util.spec_from_file_location("speculative_step", os.path.join(ROOT, "examples", "speculative_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def rows(layer, b):
    """Request b's rows of the cache as stored."""
    n = int(layer.lengths[b])
    slots = layer.slots(b, torch.arange(n, device=DEV))
    return [x[slots // layer.page, slots % layer.page] for x in
            (layer.cache.k, layer.cache.v, layer.cache.k_scales, layer.cache.v_scales) if x is not None]


def values(step, layer, b, n):
    """The values of request b's first n tokens, float64 [n, heads, head_dim]."""
    slots = layer.slots(b, torch.arange(n, device=DEV))
    return step.ops.mixfp4_kv_gather(layer.cache, slots, torch.float32)[1].double()


@pytest.mark.parametrize("cache", ["bf16", "mixfp4"])
@pytest.mark.parametrize("t", [1, 7, 64])
def test_trees_are_what_their_branches_give(step, cache, t):
    batch, hidden = 3, 256
    kw = dict(batch=batch, context=200, room=4 * t + 8, hidden=hidden, q_heads=4, kv_heads=2, head_dim=64, cache=cache)
    g = torch.Generator().manual_seed(t)
    layer, chain = step.Layer(**kw), step.Layer(**kw)  # the same requests; one decodes accepted tokens in chains
    one = torch.ones(1, dtype=torch.int64, device=DEV)
    x = torch.randn(batch, t, hidden, generator=g).to(DEV, torch.bfloat16)
    for turn in range(2):
        parents, mask = step.random_trees(batch, t, g)
        path = step.random_path(parents, t, g)
        # projected once: the activations of a call share a scale, so drafts alone would have other keys
        qkv = layer.project(x)
        y = layer.attend(*qkv, mask.to(DEV))
        layer.accept(path.to(DEV), t)
        depth = int((path >= 0).sum(1).max())
        for k in range(depth):  # requests whose path has ended decode a token more, which is taken back
            at = path[:, k].clamp(min=0).long().to(DEV)
            z = chain.attend(*(r[torch.arange(batch, device=DEV), at][:, None].contiguous() for r in qkv), one)
            on = path[:, k] >= 0
            for b in range(batch):
                if on[b]:
                    n = int(chain.lengths[b])
                    v = values(step, chain, b, n)
                    # twice the attention's own bound: sums within 2^-13 (bf16) or 2^-10.5 (MixFP4) of the values' mean
                    # magnitude, at most the largest, with 2^-32 of their sum, and half a step of the result
                    sums = (2.0 ** -13 if cache == "bf16" else 2.0 ** -10.5) * v.abs().amax(0) + 2.0 ** -32 * v.abs().sum(0)
                    sums = sums.repeat_interleave(2, 0)  # two query heads to a key head
                    p, q = z[b, 0].double(), y[b, at[b]].double()
                    assert torch.all((p - q).abs() <= 2 * sums + 2.0 ** -8 * (p.abs() + q.abs())), (turn, b, k)
            chain.lengths -= (~on).to(DEV, torch.int32)
        assert torch.equal(layer.lengths, chain.lengths)
        for b in range(batch):
            for p, q in zip(rows(layer, b), rows(chain, b)):
                assert torch.equal(p, q), (turn, b)


@pytest.mark.parametrize("cache", ["bf16", "mixfp4"])
def test_branches_go_their_own_ways(step, cache):
    layer = step.Layer(3, 100, 64, hidden=256, q_heads=4, kv_heads=2, head_dim=64, cache=cache)
    x = torch.randn(4, 3, 256, generator=torch.Generator().manual_seed(2)).to(DEV, torch.bfloat16)
    mask = torch.tensor([1, 3, 7], device=DEV)
    before = [rows(layer, b) for b in range(3)]
    pool = [p.view(torch.uint8).clone() for p in (layer.cache.k, layer.cache.v)]  # as bytes: pages may hold anything
    table = layer.table.clone()
    parents = torch.tensor([1, 1, 2, 0], dtype=torch.int32, device=DEV)
    layer.branch(parents)
    y = layer.verify(x, mask.expand(4, 3))
    layer.accept(torch.tensor([[0, 1, 2]] * 4, dtype=torch.int32, device=DEV), 3)
    for i, p in enumerate(parents.tolist()):
        for now, then in zip(rows(layer, i), before[p]):
            assert torch.equal(now[:then.shape[0]], then) and now.shape[0] == then.shape[0] + 3
    for now, then in zip((layer.cache.k, layer.cache.v), pool):  # nothing of the parents has changed
        own = table.long().reshape(-1)
        assert torch.equal(now.view(torch.uint8)[own], then[own])
    assert torch.isfinite(y).all()
    assert (rows(layer, 0)[0][-1] != rows(layer, 1)[0][-1]).any()  # two children of one parent, other tokens


def test_example_runs(step, capsys):
    for cache in ("bf16", "mixfp4"):
        step.main(["--batch", "3", "--context", "64", "--drafts", "5", "--steps", "2", "--cache", cache, "--softcap", "30"])
    out = capsys.readouterr().out
    assert "tokens kept" in out and "nan" not in out
