"""Attention of drafted tokens over the paged cache against the definition in 64 bits.

Bounds as in test_gpu_paged_attention.py: with A = sum_j p_j |v_j| of the exact
weights p, 2^-13 A on a bf16 cache and 2^-10.5 A on a MixFP4 one, then the rounding to
bf16.  A MixFP4 cache's weights are f16 numbers of 2^7 times 2^(s - m), m at most the
largest score: those below 2^-14 are off by up to 2^-25, half of f16's smallest
step, and their sum is at least 2^7, so that each p_j is off by up to 2^-32 besides:
2^-32 sum_j |v_j| more, which counts where A is next to nothing (a zero of V under all of
the weight).  The log-sum-exp within 2^-17 (1 + top).  top is the largest |score| plus
|bias| of what has a weight of 2^-30 or more: capped scores are within 2^-20 of
themselves and a bias within 2^-23 of itself, so neither widens these."""
import math
import os
import random
import sys

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)
import test_gpu_paged_attention as pa  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
ops, randn = pa.ops, pa.randn


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


def signed(bits):
    return bits - (1 << 64) if bits >= 1 << 63 else bits


def tree(t, seed):
    """Ancestor bits of a random tree whose drafts come after their ancestors."""
    rng = random.Random(seed)
    seen = []
    for i in range(t):
        seen.append(1 << i | (seen[rng.randrange(max(0, i - 5), i)] if i else 0))
    return seen


def chain(t):
    return [(2 << i) - 1 for i in range(t)]


def reference(q, k, v, n, c, bits, scale, fp4, window=0, cap=0.0, slopes=None, skip=None):
    """One sequence's rows [t, H, D] and [t, H] in 64 bits, the bound of each element, and the bound of lse.
    bits: of each draft; skip: tokens on pages outside the cache."""
    t, H, D = q.shape
    Hkv = k.shape[1]
    c = max(0, min(c, t, n))
    first = n - c
    held = k.shape[0]  # tokens within the table
    out = torch.zeros(t, H, D, dtype=torch.float64, device=DEV)
    mag = torch.zeros_like(out)
    lse = torch.full((t, H), -math.inf, dtype=torch.float64, device=DEV)
    lim = torch.zeros_like(lse)
    depth = [bin(bits[i] & ((1 << c) - 1) & ~(1 << i)).count("1") for i in range(c)]
    for i in range(c):
        place = first + depth[i]
        at = ints([j if j < first else first + depth[j - first] for j in range(n)], torch.int64)[:held]
        sees = ints([j < first or bool(bits[i] >> (j - first) & 1) for j in range(n)], torch.bool)[:held]
        if window:
            sees = sees & (place - at < window)
        if skip is not None:
            sees = sees & ~skip
        if not bool(sees.any()):
            continue
        kk, vv = k[sees], v[sees]
        s = torch.einsum("hgd,nhd->hgn", q[i].double().view(Hkv, H // Hkv, D), kk) * scale
        if cap:
            s = cap * torch.tanh(s / cap)
        bias = torch.zeros_like(s)
        if slopes is not None:
            bias = -slopes.double().view(Hkv, H // Hkv, 1) * (place - at[sees])
        x = s + bias
        p = x.softmax(-1)
        out[i] = torch.einsum("hgn,nhd->hgd", p, vv).reshape(H, D)
        mag[i] = (2.0 ** -10.5 if fp4 else 2.0 ** -13) * torch.einsum("hgn,nhd->hgd", p, vv.abs()).reshape(H, D)
        if fp4:
            mag[i] += 2.0 ** -32 * vv.abs().sum(0).repeat_interleave(H // Hkv, 0)
        lse[i] = torch.logsumexp(x, -1).reshape(H)
        top = torch.where(p >= 2.0 ** -30, s.abs() + bias.abs(), 0.0).amax(-1).reshape(H)
        lim[i] = 2.0 ** -17 * (1 + top)
    return out, mag, lse, lim


def check(out, lse, q, k, v, lengths, counts, bits, scale, fp4, skip=None, **kw):
    at = 0
    for b, n in enumerate(lengths):
        ref, mag, ls, lim = reference(q[b], k[at:at + n], v[at:at + n], n, counts[b], bits[b], scale, fp4,
                                      skip=None if skip is None else skip.get(b), **kw)
        at += n
        none = ls == -math.inf
        assert torch.all(out[b][none] == 0) and torch.all(lse[b][none] == -math.inf), b
        pa.within(out[b], ref, mag)
        some = ~none
        assert torch.all((lse[b].double() - ls).abs()[some] <= lim[some]), (b, float((lse[b] - ls).abs()[some].max()))


def run(fp4, lengths, counts, t, Hq, Hkv, D, page, window=0, cap=0.0, bias=False, masks="tree", layout="nhd", wide=0,
        seed=1):
    o = ops()
    cache, table, k, v = pa.build(fp4, lengths, Hkv, D, page, layout, seed=seed)
    if wide:
        full = torch.full((len(lengths), wide), -1, dtype=torch.int32, device=DEV)
        full[:, :table.shape[1]] = table
        table = full
    B = len(lengths)
    q = (randn(B, t, Hq, D, seed=seed + 5) * 1.5).to(torch.bfloat16)
    slopes = None
    if bias:
        slopes = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device=DEV) / Hq).float()
    mask, bits = None, [chain(t)] * B
    if masks == "tree":
        bits = [tree(t, seed * 100 + b) for b in range(B)]
        mask = ints([[signed(m) for m in r] for r in bits], torch.int64)
    elif masks == "shared":
        bits = [tree(t, seed)] * B
        mask = ints([signed(m) for m in bits[0]], torch.int64)
    elif masks == "any":  # no tree: drafts see later ones, not always themselves, some nothing; bits behind the drafts set
        rng = random.Random(seed)
        bits = [[rng.getrandbits(64) if i % 3 else 0 for i in range(t)] for _ in range(B)]
        mask = ints([[signed(m) for m in r] for r in bits], torch.int64)
    n = ints(lengths)
    kw = dict(mask=mask, counts=None if counts is None else ints(counts), window=window, softcap=cap, slopes=slopes)
    out, lse = o.mixfp4_tree_attention(q, cache, table, n, return_lse=True, **kw)
    check(out, lse, q, k, v, lengths, [t] * B if counts is None else counts, bits, D ** -0.5, fp4, window=window,
          cap=cap, slopes=slopes)
    again, lse2 = o.mixfp4_tree_attention(q, cache, table, n, return_lse=True, **kw)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


CASES = [
    # lengths, counts, t, Hq, Hkv, D, page, options
    ([1], None, 1, 1, 1, 16, 1, dict(masks="chain")),
    ([1, 0, 15, 16, 17, 63, 64, 65], None, 1, 8, 2, 128, 16, dict(masks="chain", cap=30.0)),
    ([127, 128, 129, 255, 256, 257, 8, 0], None, 8, 8, 2, 128, 16, {}),
    ([700], [5], 7, 32, 8, 128, 16, dict(layout="hnd")),
    ([129, 3000, 0, 13, 5], [13, 1, 3, 13, 0], 13, 14, 2, 64, 48, dict(layout="kv", cap=30.0)),
    ([513, 64], None, 64, 24, 1, 128, 64, {}),                 # more rows than one pass over the cache takes
    ([77, 333, 40], [40, 33, 3], 40, 6, 6, 48, 3, dict(layout="hnd", masks="shared")),
    ([250, 1111], None, 5, 16, 16, 80, 16, dict(bias=True)),
    ([100, 900, 64], None, 33, 8, 1, 256, 32, {}),
    ([50], None, 3, 40, 2, 192, 16, dict(layout="kv", bias=True, cap=50.0)),
    ([200, 31], None, 9, 71, 1, 64, 16, {}),
    ([300, 9], None, 9, 2, 1, 32, 7, dict(masks="any")),
    ([300, 70], [64, 33], 64, 4, 2, 128, 16, dict(masks="any", window=40)),
    ([5000, 10, 100], None, 6, 9, 3, 96, 16, dict(window=7)),  # windows that start and end inside pages
    ([5000, 10, 100], None, 17, 12, 4, 128, 32, dict(window=1000, layout="hnd")),
    ([40, 3], None, 2, 2, 2, 64, 16, dict(window=1)),
    ([9000, 4100], None, 16, 8, 2, 128, 16, dict(bias=True)),
    ([2100], None, 32, 16, 2, 112, 16, dict(cap=5.0, window=900)),
]


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_matches_the_definition(fp4, case):
    lengths, counts, t, Hq, Hkv, D, page, kw = CASES[case]
    run(fp4, lengths, counts, t, Hq, Hkv, D, page, seed=case + 3, **kw)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("rows", [1, 8, 31, 32, 33, 64, 65, 127, 128, 129, 200, 256, 257])
def test_every_number_of_rows(fp4, rows):
    """Rows (drafts times query heads) to a key head, around the numbers where the kernel changes its way."""
    t = next(k for k in (64, 50, 43, 40, 33, 32, 31, 13, 1) if rows % k == 0)
    run(fp4, [700, 3, 129], [t, min(3, t), t], t, 2 * (rows // t), 2, 64, 16, seed=rows)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("Hkv,D,page,layout", [(8, 128, 16, "nhd"), (8, 128, 128, "hnd"), (1, 128, 64, "nhd"),
                                               (3, 128, 32, "kv"), (4, 64, 16, "nhd"), (4, 64, 256, "hnd"), (8, 32, 16, "nhd"),
                                               (2, 32, 48, "hnd"), (1, 256, 16, "nhd"), (3, 256, 128, "hnd"),
                                               (2, 96, 64, "hnd"), (5, 160, 16, "nhd"), (2, 64, 24, "nhd")])
def test_layouts(fp4, Hkv, D, page, layout):
    """Rows and scale bytes as the copies of each way into shared memory find them: whole pages, parts, heads together or
    apart, pages that are not a multiple of 16."""
    run(fp4, [300, 1000, 5, 129], None, 5, 2 * Hkv, Hkv, D, page, layout=layout, window=0, seed=D + page)
    run(fp4, [300, 1000, 5, 129], [5, 2, 5, 1], 5, 2 * Hkv, Hkv, D, page, layout=layout, window=150, seed=D + page + 1)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("B,longest,t,D,Hq,Hkv", [(3, 9000, 24, 128, 8, 2), (3, 9000, 8, 128, 8, 2), (3, 9000, 16, 128, 8, 2),
                                                  (20, 3000, 24, 128, 32, 8), (3, 9000, 64, 128, 8, 2),
                                                  (5, 2000, 7, 256, 4, 1), (30, 500, 3, 64, 8, 2)])
def test_same_results_every_time(fp4, B, longest, t, D, Hq, Hkv):
    """No result depends on which warp, copy or product comes first."""
    o = ops()
    g = random.Random(B)
    lengths = [g.randint(1, longest) for _ in range(B)]
    counts = [g.randint(0, t) for _ in range(B)]
    cache, table, _, _ = pa.build(fp4, lengths, Hkv, D, 16, seed=B)
    q = (randn(B, t, Hq, D, seed=5) * 1.5).to(torch.bfloat16)
    mask = ints([signed(m) for m in tree(t, B)], torch.int64)
    first, lse = o.mixfp4_tree_attention(q, cache, table, ints(lengths), mask=mask, counts=ints(counts), return_lse=True)
    for _ in range(40):
        out, l2 = o.mixfp4_tree_attention(q, cache, table, ints(lengths), mask=mask, counts=ints(counts), return_lse=True)
        assert torch.equal(out, first) and torch.equal(l2, lse)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("t,n,B", [(2, 140000, 20), (33, 150000, 10)])
def test_parts_of_many_tiles(fp4, t, n, B):
    """Parts of rows of more than 8192 tokens to a CTA, whose sums are set aside on the way; page numbers are in
    any order."""
    o = ops()
    D, page, Hq = 64, 16, 4
    pages = B * (n // page)
    g = torch.Generator(DEV).manual_seed(t)
    if fp4:
        parts = [torch.randint(0, 256, (pages, page, 1, D // 2), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
        parts += [torch.randint(0x30, 0x38, (pages, page, 1, D // 16), generator=g, device=DEV, dtype=torch.uint8)
                  for _ in range(2)]
        one = torch.ones(1, device=DEV)
        cache = o.KVCache(*parts, one * 0.25, one)
    else:
        cache = o.KVCache(*(torch.randn(pages, page, 1, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2)))
    table = torch.randperm(pages, generator=g, device=DEV).to(torch.int32).view(B, -1)
    q = (randn(B, t, Hq, D, seed=5) * 1.5).to(torch.bfloat16)
    out, lse = o.mixfp4_tree_attention(q, cache, table, ints([n] * B), return_lse=True)
    for b in (0, B // 2, B - 1):
        slots = (table[b].long()[:, None] * page + torch.arange(page, device=DEV)).reshape(-1)
        k, v = (x.double() for x in o.mixfp4_kv_gather(cache, slots, torch.float32))
        for i in (0, t - 1):
            m = n - t + 1 + i
            s = torch.einsum("hd,nd->hn", q[b, i].double(), k[:m, 0]) * D ** -0.5
            p = s.softmax(-1)
            A = p @ v[:m, 0].abs()
            bound = 2.0 ** -10.5 * A + 2.0 ** -32 * v[:m, 0].abs().sum(0) if fp4 else 2.0 ** -13 * A
            pa.within(out[b, i], p @ v[:m, 0], bound)
            assert torch.all((lse[b, i].double() - torch.logsumexp(s, -1)).abs() <= 2.0 ** -17 * (1 + s.abs().amax(-1)))


@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("fp4", [False, True])
def test_pages_far_into_the_pool(fp4, page):
    """Pages more than 2^32 bytes behind the first, by TMA and row by row, and moved there."""
    o = ops()
    Hkv, D, Hq, t, n = 4, 128, 8, 5, 900
    row = D // 2 if fp4 else 2 * D
    pages = (2 ** 32 + 2 ** 26) // (page * Hkv * row)
    ts = dict(k_ts=torch.full((1,), 0.25, device=DEV), v_ts=torch.full((1,), 1.0, device=DEV)) if fp4 else {}
    cache = o.empty_kv_cache(pages, page, Hkv, D, DEV, **ts)
    held = -(-n // page) + 1
    far = pages - 1 - torch.randperm(2 * held, device=DEV).to(torch.int32)
    table = far[:held].view(1, -1)
    at = torch.arange(n, device=DEV)
    slots = table[0, at // page].long() * page + at % page
    o.mixfp4_kv_append(randn(n, Hkv, D, seed=1), randn(n, Hkv, D, seed=2), cache, slots)
    q = (randn(1, t, Hq, D, seed=5) * 1.5).to(torch.bfloat16)

    def look(table, n):
        at = torch.arange(n, device=DEV)
        rows = o.mixfp4_kv_gather(cache, table[0, at // page].long() * page + at % page, torch.float32)
        k, v = (x.double() for x in rows)
        out, lse = o.mixfp4_tree_attention(q, cache, table, ints([n]), return_lse=True)
        check(out, lse, q, k, v, [n], [t], [chain(t)], D ** -0.5, fp4)
        return out
    first = look(table, n)
    o.mixfp4_kv_copy_pages(cache, far[:held], far[held:])
    assert torch.equal(look(far[held:].view(1, -1), n), first)
    path = ints([[0, 2, 3, -1]])
    before = [x.clone() for x in o.mixfp4_kv_gather(cache, slots, torch.float32)]
    length = o.mixfp4_kv_accept(cache, table, ints([n]), path, ints([t]))
    assert length.tolist() == [n - t + 3]
    after = o.mixfp4_kv_gather(cache, slots, torch.float32)
    kept = [*range(n - t), n - t, n - t + 2, n - t + 3]
    assert all(torch.equal(y[:n - t + 3], x[kept]) for x, y in zip(before, after))
    tables, lengths = o.mixfp4_kv_fork(cache, table, length, ints([0, 0]), torch.stack([far[held], ints([-1])[0]]))
    assert lengths.tolist() == length.tolist() * 2
    assert torch.equal(look(tables[:1].contiguous(), n - t + 3), look(tables[1:].contiguous(), n - t + 3))


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("B,longest,t,D", [(1, 30000, 3, 64), (3, 9000, 24, 128), (150, 300, 2, 64), (700, 40, 1, 128),
                                           (1500, 20, 3, 16)])
def test_many_shares(fp4, B, longest, t, D):
    """Sequences cut over many CTAs, many sequences to a CTA, more sequences than a CTA has threads."""
    g = random.Random(B)
    lengths = [g.randint(0, longest) for _ in range(B)]
    lengths[0] = longest
    run(fp4, lengths, [g.randint(0, t) for _ in range(B)], t, 8, 2, D, 16, masks="shared", seed=B,
        wide=longest // 16 + 70)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_scores_that_grow_or_shrink_along_the_sequence(fp4, cap):
    """The running maximum moves at every tile, or never after the first."""
    o = ops()
    H, D, n, t = 2, 128, 4000, 3
    for sign in (1.0, -1.0):
        cache, table, _, _ = pa.build(fp4, [n], H, D, 16, seed=3)
        k = torch.zeros(n, H, D, device=DEV)
        k[:, :, 0] = torch.linspace(-8.0, 8.0, n, device=DEV)[:, None] * sign
        v = randn(n, H, D, seed=11)
        slots = (table[0, :n // 16].long()[:, None] * 16 + torch.arange(16, device=DEV)).reshape(-1)
        o.mixfp4_kv_append(k, v, cache, slots)
        gk, gv = (x.double() for x in o.mixfp4_kv_gather(cache, slots, torch.float32))
        q = torch.zeros(1, t, 4, D, dtype=torch.bfloat16, device=DEV)
        q[..., 0] = ints([1.0, 30.0, 90.0, 0.0], torch.bfloat16)
        out, lse = o.mixfp4_tree_attention(q, cache, table, ints([n]), softcap=cap, return_lse=True)
        check(out, lse, q, gk, gv, [n], [t], [chain(t)], D ** -0.5, fp4, cap=cap)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_steep_slopes(fp4, sign):
    """A bias of many powers of two over the sequence, for near and (slopes below zero) for far tokens."""
    o = ops()
    lengths, t = [1500, 90], 4
    cache, table, k, v = pa.build(fp4, lengths, 2, 64, 16, seed=3)
    q = randn(2, t, 4, 64, seed=4).to(torch.bfloat16)
    slopes = sign * torch.tensor([4.0, 0.5, 0.0, 0.01], device=DEV)
    out, lse = o.mixfp4_tree_attention(q, cache, table, ints(lengths), slopes=slopes, return_lse=True)
    check(out, lse, q, k, v, lengths, [t, t], [chain(t)] * 2, 0.125, fp4, slopes=slopes)


@pytest.mark.parametrize("fp4", [False, True])
def test_large_and_tiny_queries(fp4):
    """Rows whose queries differ by many powers of two, and rows of zeros."""
    o = ops()
    n, t = 200, 6
    cache, table, k, v = pa.build(fp4, [n], 1, 64, 16, seed=8)
    size = torch.tensor([1.0, 2.0 ** -60, 2.0 ** 60, 0.0, 2.0 ** -120, 1e-3], device=DEV)
    q = (randn(1, t, 2, 64, seed=9) * size[:, None, None]).to(torch.bfloat16)
    for rows, scale in (([0, 1, 3, 4, 5], 0.125), ([2], 0.125 * 2.0 ** -60)):
        out, lse = o.mixfp4_tree_attention(q, cache, table, ints([n]), scale=scale, return_lse=True)
        ref, mag, ls, lim = reference(q[0], k, v, n, t, chain(t), scale, fp4)
        pa.within(out[0][rows], ref[rows], mag[rows])
        assert torch.all((lse[0].double() - ls).abs()[rows] <= lim[rows])


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("t,Hq", [(4, 2), (9, 8), (24, 8), (60, 8)])
def test_what_is_not_seen_does_not_reach_a_row(fp4, t, Hq):
    """A draft whose key and value are NaN and infinite spoils the rows that see it and no others; so does a certain
    token that some rows' windows still hold."""
    o = ops()
    n, D, Hkv, window = 400, 64, 2, 100
    cache, table, k, v = pa.build(fp4, [n], Hkv, D, 16, seed=t)
    bits = tree(t, 7)
    depth = [bin(m).count("1") - 1 for m in bits]
    q = randn(1, t, Hq, D, seed=3).to(torch.bfloat16)
    first = n - t
    spoiled = {first + t // 2}
    clean, clean_lse = o.mixfp4_tree_attention(q, cache, table, ints([n]), mask=ints([bits], torch.int64),
                                               window=window, return_lse=True)
    edge = first + 1 - window  # seen by drafts of depth 0 alone
    for token, kinds in ((first + t // 2, ("k", "v")), (edge, ("v",)), (first + t - 1, ("v",))):
        at = int(table[0, token // 16]), token % 16
        kept = []
        for kind in kinds:
            x = getattr(cache, kind + "_scales" if fp4 else kind)
            kept.append((x, x[at].clone()))
            x[at] = 0x7F if fp4 else float("inf" if kind == "v" else "nan")
        sees = [bool(bits[i] >> (token - first) & 1) if token >= first else first + depth[i] - token < window
                for i in range(t)]
        assert any(sees) and not all(sees) or t == 4 or token == first + t - 1
        out, lse = o.mixfp4_tree_attention(q, cache, table, ints([n]), mask=ints([bits], torch.int64), window=window,
                                           return_lse=True)
        for i in range(t):
            if sees[i]:
                assert not torch.isfinite(out[0, i]).any(), (token, i)
            else:
                assert torch.isfinite(out[0, i].float()).all(), (token, i)
                torch.testing.assert_close(out[0, i], clean[0, i], rtol=2.0 ** -7, atol=2.0 ** -9)
                torch.testing.assert_close(lse[0, i], clean_lse[0, i], rtol=2.0 ** -18, atol=2.0 ** -18)
        for x, y in kept:
            x[at] = y


@pytest.mark.parametrize("n,t,Hq", [(40, 3, 4), (300, 40, 4), (3000, 9, 32)])
def test_infinite_and_nan_scores(n, t, Hq):
    """A score of NaN makes out and lse NaN, one of +inf out NaN and lse +inf, one of -inf has no weight; an infinite
    element of V makes its dimension infinite."""
    o = ops()
    D, Hkv = 64, 2
    cache, table, k, v = pa.build(False, [n], Hkv, D, 16, seed=5)
    q = (randn(1, t, Hq, D, seed=6) * 0.2).to(torch.bfloat16)
    q[..., 0] = 0.0
    G = Hq // Hkv
    q[0, 0, 0, 0], q[0, 1, 0, 0], q[0, 2, G, 0] = 1.0, -1.0, float("nan")  # heads of key head 0, 0 and 1
    at = int(table[0, 0]), 3
    cache.k[at][0, 0] = float("inf")
    k[3, 0, 0] = math.inf
    q[0, :, :G, 0][q[0, :, :G, 0] == 0] = 1e-30  # 0 * inf would be NaN: these see +inf as well
    out, lse = o.mixfp4_tree_attention(q, cache, table, ints([n]), return_lse=True)
    assert torch.isnan(out[0, 0, 0]).all() and lse[0, 0, 0] == math.inf
    assert torch.isnan(out[0, 2, G]).all() and torch.isnan(lse[0, 2, G])
    ref, mag, ls, lim = reference(q[0], k, v, n, t, chain(t), D ** -0.5, False)
    pa.within(out[0, 1, 0], ref[1, 0], mag[1, 0])
    assert (lse[0, 1, 0] - ls[1, 0]).abs() <= 2.0 ** -17 * 20
    # infinite values: seen by every row, dimensions 0 (+inf), 1 (-inf) and 2 (both signs)
    cache, table, k, v = pa.build(False, [n], Hkv, D, 16, seed=5)
    q = (randn(1, t, Hq, D, seed=6) * 0.2).to(torch.bfloat16)
    for token, dim, x in ((1, 0, math.inf), (n - t, 1, -math.inf), (1, 2, math.inf), (n - t, 2, -math.inf)):
        cache.v[int(table[0, token // 16]), token % 16, 1, dim] = x
    out = o.mixfp4_tree_attention(q, cache, table, ints([n]))
    assert torch.all(out[0, :, G:, 0] == math.inf) and torch.all(out[0, :, G:, 1] == -math.inf)
    assert torch.isnan(out[0, :, G:, 2]).all()
    assert torch.isfinite(out[0, :, G:, 3:].float()).all() and torch.isfinite(out[0, :, :G].float()).all()


@pytest.mark.parametrize("fp4", [False, True])
def test_pages_outside_the_cache_are_not_seen(fp4):
    o = ops()
    lengths, t = [100, 40, 16], 5
    cache, table, k, v = pa.build(fp4, lengths, 2, 64, 16, seed=2)
    table[0, 3], table[1, 0], table[2, 0] = -1, cache.pages, -7
    table[0, 6] = 2 ** 31 - 1  # four drafts of five are gone too
    q = randn(3, t, 4, 64, seed=5).to(torch.bfloat16)
    gone = {b: torch.zeros(n, dtype=torch.bool, device=DEV) for b, n in enumerate(lengths)}
    gone[0][48:64] = gone[0][96:] = True
    gone[1][:16] = True
    gone[2][:] = True
    out, lse = o.mixfp4_tree_attention(q, cache, table, ints(lengths), return_lse=True)
    check(out, lse, q, k, v, lengths, [t] * 3, [chain(t)] * 3, 0.125, fp4, skip=gone)


def test_lengths_and_counts_outside_their_ranges():
    """Negative lengths see nothing, one past the table's pages ends with them; counts are cut to 0 .. min(t, n)."""
    o = ops()
    t = 4
    cache, table, k, v = pa.build(False, [32, 32, 2], 2, 64, 16, seed=2)
    q = randn(3, t, 4, 64, seed=5).to(torch.bfloat16)
    out, lse = o.mixfp4_tree_attention(q, cache, table[:, :2], ints([-5, 34, 2]), counts=ints([2, 9, 100]),
                                       return_lse=True)
    assert torch.all(out[0] == 0) and torch.all(lse[0] == -math.inf)
    # 34 tokens with 4 drafts of which the table holds two; then 2 tokens, both drafts
    ref, mag, ls, lim = reference(q[1], k[32:64], v[32:64], 34, t, chain(t), 0.125, False)
    pa.within(out[1], ref, mag)
    assert torch.all((lse[1].double() - ls).abs() <= lim)
    check(out[2:], lse[2:], q[2:], k[64:], v[64:], [2], [2], [chain(t)], 0.125, False)
    out = o.mixfp4_tree_attention(q, cache, table, ints([32, 32, 2]), counts=ints([-1, 0, 0]))
    assert torch.all(out == 0)
    none = o.mixfp4_tree_attention(q, cache, table[:, :0], ints([3, 3, 3]))
    assert torch.all(none == 0)
    assert o.mixfp4_tree_attention(q[:0], cache, table[:0], ints([])).shape == (0, t, 4, 64)
    assert o.mixfp4_tree_attention(q[:, :0], cache, table, ints([32, 32, 2])).shape == (3, 0, 4, 64)


@pytest.mark.parametrize("fp4", [False, True])
def test_one_draft_is_one_token_attention(fp4):
    o = ops()
    lengths = [700, 0, 33, 2000]
    cache, table, k, v = pa.build(fp4, lengths, 2, 128, 16, seed=4)
    q = randn(4, 8, 128, seed=5).to(torch.bfloat16)
    for window in (0, 50):
        one, l1 = o.mixfp4_paged_attention(q, cache, table, ints(lengths), window=window, return_lse=True)
        two, l2 = o.mixfp4_tree_attention(q[:, None], cache, table, ints(lengths), window=window, return_lse=True)
        bound = 2.0 ** (-10.5 if fp4 else -13) * 2 * v.abs().max()
        assert torch.all((one.float() - two[:, 0].float()).abs() <= bound + 2.0 ** -8 * one.float().abs())
        fin = torch.isfinite(l1)
        assert torch.equal(fin, torch.isfinite(l2[:, 0]))
        assert torch.all((l1 - l2[:, 0]).abs()[fin] <= 2.0 ** -16 * 20)


@pytest.mark.parametrize("fp4", [False, True])
def test_strides_workspace_and_stream(fp4):
    o = ops()
    lengths, t, H, D = [300, 5, 1000], 5, 8, 128
    cache, table, k, v = pa.build(fp4, lengths, 2, D, 16, seed=4)
    n = ints(lengths)
    fused = randn(t, 3, 3, H, D + 8, seed=5).to(torch.bfloat16)
    q = fused[:, 1, :, :, :D].transpose(0, 1)  # drafts outermost
    bits = [tree(t, b) for b in range(3)]
    mask = ints(bits, torch.int64)
    ref, lse = o.mixfp4_tree_attention(q.contiguous(), cache, table, n, mask=mask, return_lse=True)
    check(ref, lse, q, k, v, lengths, [t] * 3, bits, D ** -0.5, fp4)
    need = o.tree_attention_workspace_bytes(cache, 3, t, H)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)
    wide = torch.full((3, table.shape[1] + 5), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    broad = torch.zeros(3, t + 2, dtype=torch.int64, device=DEV)
    broad[:, :t] = mask
    side = torch.cuda.Stream()
    got, glse = torch.empty_like(ref), torch.empty_like(lse)
    torch.cuda.synchronize()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    o.mixfp4_tree_attention(q, cache, wide[:, :table.shape[1]], n, mask=broad[:, :t], out=got, lse=glse, workspace=ws,
                            stream=side)
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
    other, olse = o.mixfp4_tree_attention(q, cache, table, n, mask=mask, return_lse=True, stream=side)
    side.synchronize()
    assert torch.equal(got, ref) and torch.equal(glse, lse)
    assert torch.equal(other, ref) and torch.equal(olse, lse)
    # one sequence: strides of the axis that leads nowhere may be anything
    one = q[2:].as_strided((1, t, H, D), (3, *q.stride()[1:]), q[2:].storage_offset())
    got = o.mixfp4_tree_attention(one, cache, table[2:], n[2:], mask=mask[2:])
    torch.testing.assert_close(got, ref[2:], rtol=2.0 ** -7, atol=2.0 ** -9)
    with pytest.raises(o.MixFP4Error, match="invalid shape"):
        o.mixfp4_tree_attention(q, cache, table, n, workspace=ws[:need - 1])
    status = torch.full((1,), 7, dtype=torch.int32, device=DEV)
    got = o.mixfp4_tree_attention(q, cache, table, n, mask=mask, status_word=status)
    assert torch.equal(got, ref) and int(status) == 0


def test_two_calls_at_once():
    """Two streams, each with its own workspace, over one cache."""
    o = ops()
    lengths, t = [3000, 1000], 6
    cache, table, k, v = pa.build(False, lengths, 2, 128, 16, seed=4)
    n = ints(lengths)
    qs = [randn(2, t, 8, 128, seed=i).to(torch.bfloat16) for i in range(2)]
    want = [o.mixfp4_tree_attention(q, cache, table, n) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            got[i].append(o.mixfp4_tree_attention(qs[i], cache, table, n, stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


def test_in_a_cuda_graph():
    """Lengths, counts, masks and rows may change between replays; two graphs may share a workspace in turn."""
    o = ops()
    t = 6
    cache, table, k, v = pa.build(False, [640, 64], 2, 64, 16, seed=4)
    q = randn(2, t, 4, 64, seed=5).to(torch.bfloat16)
    n, c, mask = ints([10, 64]), ints([6, 6]), ints([tree(t, 1)] * 2, torch.int64)
    ws = torch.empty(o.tree_attention_workspace_bytes(cache, 2, t, 4), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o.mixfp4_tree_attention(q, cache, table, n, mask=mask, counts=c)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for cap in (0.0, 3.0):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(o.mixfp4_tree_attention(q, cache, table, n, mask=mask, counts=c, softcap=cap, workspace=ws))
    for lengths, counts, seed in (([10, 64], [6, 6], 1), ([0, 1], [0, 1], 2), ([640, 33], [6, 2], 3)):
        n.copy_(ints(lengths))
        c.copy_(ints(counts))
        mask.copy_(ints([tree(t, seed), tree(t, seed + 9)], torch.int64))
        for g in graphs:
            g.replay()
        for out, cap in zip(outs, (0.0, 3.0)):
            assert torch.equal(out, o.mixfp4_tree_attention(q, cache, table, n, mask=mask, counts=c, softcap=cap))


def test_refusals():
    o = ops()
    cache, table, _, _ = pa.build(False, [20, 20], 2, 64, 16)
    t = 3
    q = randn(2, t, 4, 64).to(torch.bfloat16)
    n = ints([20, 20])
    mask = ints([[1, 3, 7]] * 2, torch.int64)
    good = dict(q=q, cache=cache, block_table=table, lengths=n, mask=mask)
    o.mixfp4_tree_attention(**good)
    for bad in (dict(q=q.float()), dict(q=q[:, :, :3]), dict(q=q[..., :32]), dict(q=q[0]), dict(q=q.cpu()), dict(cache=3),
                dict(q=q[:, :1].expand(2, 65, 4, 64)), dict(block_table=table.long()), dict(block_table=table[:1]),
                dict(block_table=table.cpu()), dict(block_table=table[:, ::2]), dict(lengths=n.long()),
                dict(lengths=n[:1]), dict(window=-1), dict(out=q[:1]), dict(out=q.float()), dict(mask=mask.int()),
                dict(mask=mask[:1]), dict(mask=mask[:, :2]), dict(mask=mask.cpu()), dict(mask=mask[0, :2]),
                dict(counts=n.long()), dict(counts=n[:1]), dict(softcap=-1.0), dict(softcap=float("nan")),
                dict(softcap=1e7), dict(softcap=1e-7), dict(slopes=torch.zeros(3, device=DEV)),
                dict(slopes=torch.zeros(4)), dict(slopes=torch.zeros(4, device=DEV, dtype=torch.float64)),
                dict(lse=torch.empty(2, 3, device=DEV)), dict(workspace=torch.empty(1 << 22, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            o.mixfp4_tree_attention(**{**good, **bad})
    with pytest.raises(o.MixFP4Error, match="misaligned"):
        o.mixfp4_tree_attention(**{**good, "q": randn(2, t, 4, 68).to(torch.bfloat16)[..., 4:]})
