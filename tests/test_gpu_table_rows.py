"""Block tables whose rows overlap (one row expanded to all sequences, a window sliding over a list of pages): every call that
takes a table refuses them.  Their rows would be read a table's width apart, behind the tensor's end."""
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


@pytest.mark.parametrize("fp4", [False, True])
def test_overlapping_rows_are_refused(fp4):
    o = ops()
    B, Hkv, D = 3, 2, 64
    cache, table, k, v = ta.pa.build(fp4, [40], Hkv, D, 16, seed=1)
    q = randn(B, 4, D, seed=3).to(torch.bfloat16)
    n, i = ints([40] * B), ints([0] * B)
    width = table.shape[1]
    row = table[0].contiguous()
    for bad in (table.expand(B, width), torch.cat([row, row, row]).as_strided((B, width), (1, 1)),
                torch.cat([row, row, row]).as_strided((B, width), (width - 1, 1))):
        for call in (lambda: o.mixfp4_paged_attention(q, cache, bad, n), lambda: o.mixfp4_tree_attention(q[:, None], cache, bad, n),
                     lambda: o.mixfp4_kv_accept(cache, bad, n, i[:, None], i),
                     lambda: o.mixfp4_kv_fork(cache, bad, n, i, i)):
            with pytest.raises(ValueError, match="overlapping rows"):
                call()
    same = table.expand(B, width).contiguous()
    out, lse = o.mixfp4_paged_attention(q, cache, same, n, return_lse=True)
    ta.pa.check(out, lse, q, [40] * B, k.repeat(B, 1, 1), v.repeat(B, 1, 1), D ** -0.5, 0, fp4)
    # one sequence, and tables of one column: any stride of what leads nowhere
    one = o.mixfp4_paged_attention(q[:1], cache, row.as_strided((1, width), (1, 1)), n[:1])
    assert torch.equal(one, o.mixfp4_paged_attention(q[:1], cache, table, n[:1]))
    thin = torch.stack([row[0]] * B)[:, None]
    assert torch.equal(o.mixfp4_paged_attention(q, cache, thin.as_strided((B, 1), (1, 7)), ints([16] * B)),
                       o.mixfp4_paged_attention(q, cache, thin, ints([16] * B)))
    assert torch.all(o.mixfp4_paged_attention(q, cache, same[:, :0], n) == 0)
