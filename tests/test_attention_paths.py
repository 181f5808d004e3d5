"""The ways in which mixfp4_paged_attention cuts its work, each by name: a
cluster to a row, one CTA to a row, or equal shares of all rows and a joining
kernel, whose list of cut rows has a place per row or per CTA.  The rule is
restated here from the sizes alone, its constants read from the source, so that
a case says which way it takes and a changed threshold cannot take it off that way
unnoticed.

Bounds of the results as in test_gpu_paged_attention.py."""
import os
import re
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)

SOURCE = open(os.path.join(os.path.dirname(HERE), "paper_2605_31035_gb300", "csrc", "attention.cu")).read()


def constant(name):
    return int(re.search(rf"constexpr int {name} = (\d+);", SOURCE).group(1))


def way(fp4, B, Hq, Hkv, D, layout, table_tokens, window, sms):
    """(CTAs to a row or 0 for shares, key heads of a CTA, a place per row) of a call."""
    dim = 64 if D <= 64 else 128 if D <= 128 else 256
    group = Hq // Hkv
    heads = 8 if group <= 8 else 16 if group <= 16 or D > 128 or -(-group // 16) == -(-group // 24) else 24
    if dim == 256:
        ctas = 2 if fp4 else 1
    else:
        ctas = 2 if heads == 24 else 4 if heads == 8 and not fp4 and dim == 64 else 3
    grid = sms * ctas
    chunks = -(-group // heads)
    together = 1
    if layout != "hnd":  # a token's heads lie together
        for n in (4, 2):
            if together == 1 and Hkv % n == 0 and B * (Hkv // n) * chunks >= grid // 4:
                together = n
    bound = min(window, table_tokens) if window else table_tokens
    single, cluster = B * Hkv * chunks, 0
    for n in (8, 4, 2):
        if not cluster and single * n <= grid and \
                bound <= n * constant("kCtaTokens") * (4 if single * n >= grid // 2 else 1):
            cluster = n
    if not cluster and bound <= constant("kRowTokens"):
        cluster = 1
    if cluster > 1:
        together = 1
    return cluster, together, B * (Hkv // together) * chunks <= grid


WIDE = 6000  # tokens of a table wider than any sequence in it: no cluster, no single CTA to a row
CASES = [
    # B, longest, Hq, Hkv, D, layout, table tokens (0: tight), window, way() of it (None: either)
    (2, 5000, 8, 2, 128, "nhd", WIDE, 0, (0, 1, True)),
    (64, 900, 32, 8, 128, "nhd", WIDE, 0, (0, 4, True)),       # a decode batch of 8 key heads
    (64, 900, 32, 8, 128, "nhd", WIDE, 899, (0, 4, True)),     # a window that the longest sequence passes by a token
    (90, 1300, 32, 8, 128, "nhd", WIDE, 1000, (0, 4, True)),   # windows that start inside pages and tiles
    (160, 1300, 14, 2, 64, "nhd", WIDE, 777, (0, 2, True)),
    (130, 700, 40, 4, 96, "nhd", WIDE, 333, (0, 4, True)),      # ten query heads to a key head
    (80, 700, 24, 6, 80, "nhd", WIDE, 0, (0, 2, True)),
    (700, 150, 16, 4, 128, "nhd", WIDE, 0, (0, 4, False)),     # a place per CTA
    (600, 400, 16, 4, 128, "nhd", WIDE, 300, (0, 4, False)),
    (1500, 20, 8, 2, 64, "nhd", WIDE, 0, (0, 2, False)),       # many sequences to a CTA
    (1500, 20, 3, 1, 64, "nhd", WIDE, 0, (0, 1, False)),
    (100, 600, 32, 8, 128, "hnd", WIDE, 0, (0, 1, False)),
    (100, 600, 32, 8, 128, "hnd", WIDE, 400, (0, 1, False)),
    (100, 600, 24, 8, 48, "hnd", WIDE, 299, (0, 1, False)),
    (90, 400, 16, 8, 256, "nhd", WIDE, 0, (0, 4, None)),       # rows that one CTA of an SM, or two, hold
    (340, 90, 24, 1, 128, "nhd", WIDE, 0, (0, 1, False)),      # 24 query heads to a row
    (340, 90, 48, 2, 64, "nhd", WIDE, 60, (1, 2, False)),         # a window of few tokens: one CTA to a row
    (180, 90, 71, 1, 112, "nhd", WIDE, 0, (0, 1, False)),      # chunks of query heads
    (300, 200, 32, 8, 128, "nhd", 0, 0, (1, 4, False)),
    (20, 300, 16, 2, 128, "nhd", 0, 0, (8, 1, True)),
    (40, 300, 16, 2, 128, "nhd", 0, 0, (4, 1, True)),
    (90, 300, 16, 2, 128, "hnd", 0, 0, (2, 1, True)),
]


def table_tokens(longest, wide, page=16):
    return -(-max(longest, wide) // page) * page


@pytest.mark.parametrize("sms", [148, 152])
def test_cases_take_the_ways_they_are_for(sms):
    ways = set()
    for B, longest, Hq, Hkv, D, layout, wide, window, want in CASES:
        for fp4 in (False, True):
            got = way(fp4, B, Hq, Hkv, D, layout, table_tokens(longest, wide), window, sms)
            ways.add((*got, window > 0, fp4))
            assert got == want or (want[2] is None and got[:2] == want[:2]), (got, want, B, Hq, Hkv, D)
    for fp4 in (False, True):
        for together in (1, 2, 4):
            assert any(w[:2] == (0, together) and w[3] and w[4] is fp4 for w in ways), (together, "window", fp4)
            assert (0, together, False, False, fp4) in ways, (together, "place per CTA", fp4)
            assert any(w[:3] == (0, together, True) and w[4] is fp4 for w in ways), (together, "place per row", fp4)
        assert {w[0] for w in ways if w[4] is fp4} == {0, 1, 2, 4, 8}


@pytest.mark.gpu
@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("B,longest,Hq,Hkv,D,layout,wide,window,want", CASES)
def test_every_way_matches_the_definition(fp4, B, longest, Hq, Hkv, D, layout, wide, window, want):
    import test_gpu_paged_attention as t
    import torch
    g = torch.Generator().manual_seed(B + D + window)
    lengths = torch.randint(0, longest + 1, (B,), generator=g).tolist()
    lengths[0], lengths[B // 2] = longest, longest if B < 3 else 0
    cache, table, k, v = t.build(fp4, lengths, Hkv, D, 16, layout, seed=B)
    table = table[:, :-1]  # build() leaves a column that nobody has
    width = table_tokens(longest, wide) // 16
    if width > table.shape[1]:
        full = torch.full((B, width), -1, dtype=torch.int32, device=t.DEV)
        full[:, :table.shape[1]] = table
        table = full
    assert table.shape[1] == width
    q = (t.randn(B, Hq, D, seed=6) * 1.5).to(torch.bfloat16)
    n = torch.tensor(lengths, dtype=torch.int32, device=t.DEV)
    out, lse = t.ops().mixfp4_paged_attention(q, cache, table, n, window=window, return_lse=True)
    t.check(out, lse, q, lengths, k, v, D ** -0.5, window, fp4)
    again, lse2 = t.ops().mixfp4_paged_attention(q, cache, table, n, window=window, return_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
