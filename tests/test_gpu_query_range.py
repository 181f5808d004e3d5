"""Queries whose elements differ by many powers of two inside one row, over keys that are 0 where the row is largest, so that
the small elements make up the scores.

On a MixFP4 cache a row is scaled by a power of two, its largest element M to [2^14, 2^15), and rounded to f16, whose least
step is 2^-24: an element is off by at most half of that, 2^-39 of 2^14 and so of M.  A bf16 number of 8 bits is a multiple of
2^-24 from 2^-17 on, which 2^-31 M or more is after scaling: such elements are exact.  A score is then off by up to
delta = scale 2^-39 M sum_d |k_d| besides what test_gpu_tree_attention.py allows, over the elements below 2^-31 M; each weight
by a factor within exp(2 delta), delta now the largest of all tokens, and the log-sum-exp by delta."""
import os
import sys

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)
import test_gpu_tree_attention as ta  # noqa: E402

pytestmark = pytest.mark.gpu

ops, randn, ints = ta.ops, ta.randn, ta.ints


@pytest.mark.parametrize("power", [20, 30, 33, 35, 37])
@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("t,Hq,D,page", [(1, 2, 64, 16), (4, 4, 128, 16), (40, 8, 128, 24)])
def test_small_elements_beside_a_large_one(fp4, t, Hq, D, page, power):
    o = ops()
    n, Hkv = 300, 2
    cache, table, _, _ = ta.pa.build(fp4, [n], Hkv, D, page, seed=power)
    k, v = randn(n, Hkv, D, seed=1), randn(n, Hkv, D, seed=2)
    k[..., 0] = 0.0
    at = torch.arange(n, device="cuda:0")
    slots = table[0, at // page].long() * page + at % page
    o.mixfp4_kv_append(k, v, cache, slots)
    k, v = (x.double() for x in o.mixfp4_kv_gather(cache, slots, torch.float32))
    assert torch.all(k[..., 0] == 0)
    small = 2.0 ** -power * (randn(1, t, Hq, D, seed=3).abs() * 0.25 + 1.0).clamp(max=1.75)  # [2^-power, 2^(1 - power))
    q = (small * randn(1, t, Hq, D, seed=4).sign()).to(torch.bfloat16)
    q[..., 0] = 1.0
    scale = 2.0 ** (power - 3)
    delta = 0.0
    if fp4 and power > 31:
        delta = scale * 2.0 ** -39 * float(k.abs().sum(-1).max())
        assert delta < 8  # the bound says something
    ref, mag, ls, lim = ta.reference(q[0], k, v, n, t, ta.chain(t), scale, fp4)
    if delta:  # e^(2 delta) - 1 of the weights' share: |out - ref| <= (e^(2 delta) - 1) sum p |v|
        for i in range(t):
            m = n - t + 1 + i
            s = torch.einsum("hgd,nhd->hgn", q[0, i].double().view(Hkv, Hq // Hkv, D), k[:m]) * scale
            A = torch.einsum("hgn,nhd->hgd", s.softmax(-1), v[:m].abs()).reshape(Hq, D)
            mag[i] = mag[i] * 2.718281828 ** (2 * delta) + (2.718281828 ** (2 * delta) - 1) * A
    calls = [lambda: o.mixfp4_tree_attention(q, cache, table, ints([n]), scale=scale, return_lse=True)]
    if t == 1:
        calls.append(lambda: [x[:, None] for x in o.mixfp4_paged_attention(q[:, 0], cache, table, ints([n]), scale=scale,
                                                                          return_lse=True)])
    for call in calls:
        out, lse = call()
        ta.pa.within(out[0], ref, mag)
        assert torch.all((lse[0].double() - ls).abs() <= lim + delta), float((lse[0] - ls).abs().max())
