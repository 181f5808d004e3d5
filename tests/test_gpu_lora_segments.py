"""Starts that break their rule (not decreasing): segments then overlap, and the tokens of an adapter's list may be more
than there are, in sum more than 32 bits count.  Every access stays inside the T tokens, and such a list gives no gradient."""
import os
import sys

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)
import test_gpu_lora as t  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,again,R", [(8, 3, 8), (90, 2, 32), (600, 2, 64)])
def test_overlapping_segments_give_no_gradient(T, again, R):
    o = t.ops()
    K, N = 64, 96
    cuts = [0, T] * again  # segments 0 .. T, T .. 0 (empty), 0 .. T, ...
    ids = [0] * (len(cuts) - 1)
    x, ad, st, ii, _ = t.problem(T, cuts, ids, K, N, R, 2)
    dy = (t.randn(T, N, seed=9) * 1e-3).to(torch.bfloat16)
    _, u = o.mixfp4_lora(x, ad, t.ints([0, T]), t.ints([0]))
    ref = o.mixfp4_lora_backward(dy, x, u, ad, t.ints([0, T]), t.ints([0]))
    _, da, db = o.mixfp4_lora_backward(dy, x, u, ad, st, ii)
    assert torch.all(da == 0) and torch.all(db == 0)
    for got, want in zip(o.mixfp4_lora_backward(dy, x, u, ad, t.ints([0, T, T, T]), t.ints([0, 0, 0])), ref):
        assert torch.equal(got, want)
