"""The stride of an axis with one element leads nowhere and is not looked at: one token, one sequence, one head, one page
or one token to a page, whatever the strides say."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def ops():
    from paper_2605_31035_gb300 import ops as o
    return o


def randn(*shape, seed=1):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV)


def odd(t):
    """The same tensor with an odd stride on each axis of one element."""
    return t.as_strided(t.shape, [s if n > 1 else 1237 for n, s in zip(t.shape, t.stride())])


def test_append_and_attention_of_one_token():
    o = ops()
    D = 64
    for heads in (1, 2):
        q, k, v = (randn(1, h, D, seed=h + i).to(torch.bfloat16) for i, h in enumerate((4, heads, heads)))
        slot = torch.zeros(1, dtype=torch.int64, device=DEV)
        table, n = (torch.full(s, f, dtype=torch.int32, device=DEV) for s, f in (((1, 1), 0), ((1,), 1)))
        got = []
        for f in (lambda t: t, odd):
            cache = o.empty_kv_cache(1, 16, heads, D, DEV)
            cache.k.zero_(), cache.v.zero_()
            a = o.mixfp4_kv_append(f(k), f(v), cache, f(slot), q=f(q))
            got.append((a, cache.k, cache.v, o.mixfp4_paged_attention(f(q), cache, f(table), f(n))))
        for x, y in zip(*got):
            assert torch.equal(x, y)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("pages,page,heads", [(1, 16, 2), (5, 1, 2), (1, 1, 1), (3, 16, 1)])
def test_cache(fp4, pages, page, heads):
    o = ops()
    D, T = 128, pages * page
    ts = [torch.full((1,), 6.0 / 2688, device=DEV) for _ in range(2)] if fp4 else [None, None]
    k, v = randn(T, heads, D, seed=1), randn(T, heads, D, seed=2)
    slots = torch.arange(T, device=DEV)
    q = randn(2, 4, D, seed=3).to(torch.bfloat16)
    table = torch.arange(pages, dtype=torch.int32, device=DEV).repeat(2, 1)
    n = torch.tensor([T, (T + 1) // 2], dtype=torch.int32, device=DEV)
    got = []
    for f in (lambda t: t, odd):
        c = o.empty_kv_cache(pages, page, heads, D, DEV, *ts)
        # of k alone: the strides of such an axis need not agree either
        parts = [f(c.k), c.v] + ([f(c.k_scales), c.v_scales, *ts] if fp4 else [])
        cache = o.KVCache(*parts)
        o.mixfp4_kv_append(k, v, cache, slots)
        got.append((*o.mixfp4_kv_gather(cache, slots), o.mixfp4_paged_attention(q, cache, table, n)))
    for x, y in zip(*got):
        assert torch.equal(x, y)


def test_adapters_of_one_token():
    o = ops()
    K, N, R = 64, 96, 8
    a, b = (randn(1, *s, seed=i).to(torch.bfloat16) for i, s in enumerate(((R, K), (N, R))))
    ad = o.Adapters(a, b, torch.ones(1, device=DEV))
    x, dy = (randn(1, n, seed=n).to(torch.bfloat16) for n in (K, N))
    base = randn(1, N, seed=5)
    starts, ids = (torch.tensor(t, dtype=torch.int32, device=DEV) for t in ([0, 1], [0]))
    got = []
    for f in (lambda t: t, odd):
        y, u = o.mixfp4_lora(f(x), ad, starts, f(ids), base=f(base))
        got.append((y, u, *o.mixfp4_lora_backward(f(dy), f(x), f(u), ad, starts, f(ids))))
    for p, q in zip(*got):
        assert torch.equal(p, q)
