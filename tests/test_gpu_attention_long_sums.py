"""Sums over many tokens keep fp32's accuracy where one warp takes a whole long row.

The tensor cores round a chain of sums towards zero, some 2^-25 of the sum for
each link, so a result whose values have a mean would shrink with the chain's length. Here
460 sequences of 65536 to 131072 tokens (they share their pages, as prefixes do)
give every CTA a row's length, some 6000 tiles of 16 tokens, to walk.  The error is looked
at as its mean over results whose bf16 rounding varies: every sequence has
another length, and the second half of the tokens another mean.  23552 results between 1 and 2,
each rounded evenly within 2^-8, average to 2^-8.8 / sqrt(23552) = 2^-16, four times that 2^-14; chains of a few
hundred links add less than 2^-16."""
import os
import sys

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)
import test_attention_paths as paths  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("fp4", [False, True])
def test_mean_of_a_long_row(fp4):
    from paper_2605_31035_gb300 import ops
    n, B, H, D, page = 131072, 460, 4, 128, 64
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert paths.way(fp4, B, H, H, D, "nhd", n, 0, sms)[:2] == (0, 4)
    g = torch.Generator(DEV).manual_seed(1)
    ts = {}
    if fp4:
        ts = {name: torch.full((1,), top / 2688, device=DEV) for name, top in (("k_ts", 6.0), ("v_ts", 4.0))}
    cache = ops.empty_kv_cache(n // page, page, H, D, DEV, **ts)
    slots = torch.arange(n, device=DEV)
    means = 1 + 0.5 * torch.rand(2, H, D, generator=g, device=DEV)
    for i in range(0, n, 16384):
        k, v = (torch.randn(16384, H, D, generator=g, device=DEV) for _ in range(2))
        ops.mixfp4_kv_append(k, 0.3 * v + means[int(i >= n // 2)], cache, slots[i:i + 16384])
    gk, gv = (t.double() for t in ops.mixfp4_kv_gather(cache, slots, torch.float32))
    q = (torch.randn(B, H, D, generator=g, device=DEV) * 0.3).to(torch.bfloat16)
    lengths = n // 2 + torch.arange(B) * (n // 2 - 1) // (B - 1) + 1
    table = torch.arange(n // page, dtype=torch.int32, device=DEV).repeat(B, 1)
    out = ops.mixfp4_paged_attention(q, cache, table, lengths.to(torch.int32).to(DEV))
    errors = []
    for b in range(0, B, 10):
        m = int(lengths[b])
        s = torch.einsum("hd,nhd->hn", q[b].double(), gk[:m]) * D ** -0.5
        ref = torch.einsum("hn,nhd->hd", s.softmax(-1), gv[:m])
        errors.append((out[b].double() - ref) / ref)
    errors = torch.stack(errors)
    assert errors.abs().max() <= 2.0 ** -8
    assert errors.mean().abs() <= 2.0 ** -14, float(errors.mean())
