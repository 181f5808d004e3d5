"""A sequence with one draft whose own mask bit is off: its row is in the cache and nobody sees it, so whatever it holds
(a row that has not been written yet, say) reaches no result.  Bounds as in test_gpu_tree_attention.py."""
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


def spoil(cache, fp4, page, row, kind, x):
    """Every element of a row's keys or values is x; NaN on a MixFP4 cache, which has no infinities."""
    (getattr(cache, kind + "_scales") if fp4 else getattr(cache, kind))[page, row] = 0x7F if fp4 else x


@pytest.mark.parametrize("x", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("fp4,page,D,layout", [(False, 16, 128, "nhd"), (False, 24, 64, "nhd"), (False, 16, 256, "hnd"),
                                               (False, 16, 48, "nhd"), (True, 16, 128, "nhd"), (True, 32, 64, "hnd"),
                                               (True, 24, 128, "nhd"), (True, 16, 80, "nhd"), (True, 16, 256, "nhd")])
@pytest.mark.parametrize("t,Hq", [(1, 2), (1, 80), (4, 4), (40, 8)])
def test_one_draft_that_does_not_see_itself(fp4, page, D, layout, t, Hq, x):
    """Alone (zeros and -inf), as the first of a page, behind many tokens, under a window, and with another in its batch that
    has all its drafts; its row is spoiled in V, and in K."""
    o = ops()
    lengths = [1, 49, 300, 700, 64 + t]
    counts = [1, 1, 1, 1, t]
    bits = [[0] * t] * 4 + [ta.chain(t) if t > 1 else [0]]
    cache, table, k, v = ta.pa.build(fp4, lengths, 2, D, page, layout, seed=t + D)
    mask = ints([[ta.signed(m) for m in r] for r in bits], torch.int64)
    q = randn(5, t, Hq, D, seed=3).to(torch.bfloat16)
    for kinds in ("v", "kv"):
        for b in range(4):
            at = lengths[b] - 1
            for kind in kinds:
                spoil(cache, fp4, int(table[b, at // page]), at % page, kind, x)
        for window in (0, 100):
            out, lse = o.mixfp4_tree_attention(q, cache, table, ints(lengths), mask=mask, counts=ints(counts), window=window,
                                               return_lse=True)
            assert torch.isfinite(out.float()).all(), (kinds, window)
            ta.check(out, lse, q, k, v, lengths, counts, bits, D ** -0.5, fp4, window=window)
    if t > 1:  # the same without `counts`: one token in the cache is one draft at most
        out, lse = o.mixfp4_tree_attention(q[:1], cache, table[:1], ints(lengths[:1]), mask=mask[:1], return_lse=True)
        assert torch.all(out == 0) and torch.all(lse == -float("inf"))


@pytest.mark.parametrize("fp4", [False, True])
def test_one_draft_that_sees_itself_still_does(fp4):
    """The other side: what the one draft sees does reach its row."""
    o = ops()
    cache, table, k, v = ta.pa.build(fp4, [40], 2, 64, 16, seed=5)
    q = randn(1, 1, 4, 64, seed=3).to(torch.bfloat16)
    spoil(cache, fp4, int(table[0, 39 // 16]), 39 % 16, "v", float("nan"))
    for mask in (None, ints([[1]], torch.int64), ints([[-1]], torch.int64)):
        assert torch.isnan(o.mixfp4_tree_attention(q, cache, table, ints([40]), mask=mask)).all()
