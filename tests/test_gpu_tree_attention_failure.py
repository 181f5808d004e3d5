"""The failure path of the attention of drafted trees, without a fault: the rows of every CTA's first tile are withheld,
each wait ends after its limit, the call reports, and the same call right after is as it was before."""
import os
import sys
import time

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)
import test_gpu_tree_attention as ta  # noqa: E402

pytestmark = pytest.mark.gpu

ops, randn, ints = ta.ops, ta.randn, ta.ints


@pytest.mark.parametrize("lengths", [[40], [700, 3, 129], [9000, 8000], [60] * 90 + [3000]])
@pytest.mark.parametrize("fp4,D,page,t,Hq,Hkv", [
    (False, 128, 16, 5, 8, 2),   # rows by TMA, two CTAs to an SM
    (False, 80, 16, 5, 8, 2),
    (False, 128, 24, 5, 8, 2),   # row by row
    (False, 112, 16, 40, 8, 2),  # two tiles of rows
    (False, 128, 24, 40, 8, 2),
    (True, 128, 16, 5, 8, 2),    # codes by TMA
    (True, 128, 24, 5, 8, 2),    # row by row: places withheld
    (True, 80, 16, 5, 2, 1),     # and scale bytes one by one
    (True, 128, 16, 40, 8, 2),   # two tiles of rows
    (True, 128, 24, 40, 8, 2),
    (True, 96, 16, 5, 8, 2),
])
def test_withheld_rows_are_reported_and_leave_the_device_usable(fp4, D, page, t, Hq, Hkv, lengths):
    o = ops()
    cache, table, k, v = ta.pa.build(fp4, lengths, Hkv, D, page, seed=D)
    q = randn(len(lengths), t, Hq, D, seed=3).to(torch.bfloat16)
    n = ints(lengths)
    want, lse = o.mixfp4_tree_attention(q, cache, table, n, return_lse=True)
    torch.cuda.synchronize()
    at = time.perf_counter()
    bits = o.selftest_tree_attention_missed_rows(q, cache, table, n, limit_ns=5_000_000)
    assert time.perf_counter() - at < 1.0  # a limit for whoever waits, then for those who wait for them
    assert bits != 0
    status = torch.full((1,), 7, dtype=torch.int32, device="cuda:0")
    got, lse2 = o.mixfp4_tree_attention(q, cache, table, n, return_lse=True, status_word=status)
    assert int(status) == 0 and torch.equal(got, want) and torch.equal(lse, lse2)


def test_refusals():
    o = ops()
    cache, table, _, _ = ta.pa.build(False, [20, 20], 2, 128, 16)
    q = randn(2, 3, 4, 128).to(torch.bfloat16)
    good = dict(q=q, cache=cache, block_table=table, lengths=ints([20, 20]))
    for bad in (dict(q=q.float()), dict(q=q[..., :32]), dict(q=q.cpu()), dict(q=q.transpose(0, 1)), dict(cache=3),
                dict(block_table=table.long()), dict(block_table=table[:1]), dict(block_table=table[:, ::2]),
                dict(lengths=ints([20])), dict(lengths=ints([20, 20]).long())):
        with pytest.raises(ValueError):
            o.selftest_tree_attention_missed_rows(**{**good, **bad})
    for limit in (0, 3_000_000_000):
        with pytest.raises(o.MixFP4Error):
            o.selftest_tree_attention_missed_rows(**good, limit_ns=limit)
    small, table, _, _ = ta.pa.build(False, [20, 20], 2, 48, 16)
    with pytest.raises(o.MixFP4Error, match="invalid shape"):
        o.selftest_tree_attention_missed_rows(**{**good, "cache": small, "q": randn(2, 3, 4, 48).to(torch.bfloat16)})
