"""Attention of one new token per sequence over the paged cache against the
definition in 64 bits.

Bounds, with A = sum_j p_j |v_j| of the exact weights p: scores are fp32 sums
of exact products, below 2^7 in magnitude here, which with the exponential's
argument leaves the weights within 2^-14 of p, numerator and denominator
together 2^-13 A; on a MixFP4 cache a weight is rounded to f16 besides (2^-11),
in all 2^-10.5 A.  The result is the bf16 rounding of a value within that bound
of the exact one: rounding keeps order, so it lies between the roundings of the
bound's two ends.  The log-sum-exp is within 2^-17 (1 + max |s|)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def ops():
    from paper_2605_31035_gb300 import ops as o
    return o


def randn(*shape, seed=1):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV)


def build(fp4, lengths, Hkv, D, page, layout="nhd", seed=1, spare=2):
    """A cache with random rows at the sequences' slots and NaN (bf16) or NaN scale bytes (MixFP4) everywhere else,
    and the block table, whose unused entries lead nowhere."""
    o = ops()
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    width = max(need + [1]) + 1
    table = torch.full((len(lengths), width), 2 ** 31 - 1, dtype=torch.int32)
    rows, slots = [], []
    for b, n in enumerate(lengths):
        mine, order = order[:need[b]], order[need[b]:]
        table[b, :need[b]] = torch.tensor(mine, dtype=torch.int32)
        slots += [mine[j // page] * page + j % page for j in range(n)]
    T = sum(lengths)
    k, v = randn(T, Hkv, D, seed=seed), randn(T, Hkv, D, seed=seed + 1)
    k[..., :max(1, D // 40)] *= 5.0

    def alloc(n, dtype):
        fill = 0x7F if dtype is torch.uint8 else float("nan")
        if layout == "kv":
            t = torch.full((pages, 2, page, Hkv, n), fill, dtype=dtype, device=DEV)
            return t[:, 0], t[:, 1]
        shape = (2, pages, Hkv, page, n) if layout == "hnd" else (2, pages, page, Hkv, n)
        t = torch.full(shape, fill, dtype=dtype, device=DEV)
        return (t[0].transpose(1, 2), t[1].transpose(1, 2)) if layout == "hnd" else (t[0], t[1])
    if fp4:
        ts = [torch.tensor([c / 2688], dtype=torch.float32, device=DEV) for c in (20.0, 5.0)]
        cache = o.KVCache(*alloc(D // 2, torch.uint8), *alloc(D // 16, torch.uint8), *ts)
    else:
        cache = o.KVCache(*alloc(D, torch.bfloat16))
    if T:
        at = torch.tensor(slots, device=DEV)
        o.mixfp4_kv_append(k, v, cache, at)
        gk, gv = o.mixfp4_kv_gather(cache, at, torch.float32)  # the rows as stored
    else:
        gk = gv = torch.empty(0, Hkv, D, device=DEV)
    return cache, table.to(DEV), gk.double(), gv.double()


def within(out, ref, bound):
    """out is the bf16 rounding of something within `bound` of ref (64-bit)."""
    lo, hi = (t.float().to(torch.bfloat16) for t in (ref - bound, ref + bound))
    assert torch.all((lo <= out) & (out <= hi)), float(((out.double() - ref).abs() - bound).max())


def check(out, lse, q, lengths, k, v, scale, window, fp4, skip=None):
    B, H, D = q.shape
    Hkv = k.shape[1]
    at = 0
    for b, n in enumerate(lengths):
        lo = max(0, n - window) if window else 0
        kb, vb = k[at + lo:at + n], v[at + lo:at + n]
        if skip is not None and b in skip:
            kb, vb = kb[~skip[b]], vb[~skip[b]]
        at += n
        if kb.shape[0] == 0:
            assert torch.all(out[b] == 0) and torch.all(lse[b] == -math.inf), b
            continue
        s = torch.einsum("hgd,nhd->hgn", q[b].double().view(Hkv, H // Hkv, D), kb) * scale
        assert s.abs().max() < 128 / 1.45
        p = s.softmax(-1)
        ref = torch.einsum("hgn,nhd->hgd", p, vb).reshape(H, D)
        mag = torch.einsum("hgn,nhd->hgd", p, vb.abs()).reshape(H, D)
        within(out[b], ref, (2.0 ** -10.5 if fp4 else 2.0 ** -13) * mag)
        ls = torch.logsumexp(s, -1).reshape(H)
        top = s.abs().amax(-1).reshape(H)
        assert torch.all((lse[b].double() - ls).abs() <= 2.0 ** -17 * (1 + top)), b


CASES = [
    # fp4, lengths, Hq, Hkv, D, page, window, layout
    (False, [1], 1, 1, 16, 1, 0, "nhd"),
    (False, [1, 0, 15, 16, 17, 63, 64, 65], 8, 2, 128, 16, 0, "nhd"),
    (False, [700], 32, 8, 128, 16, 0, "hnd"),
    (False, [129, 3000, 0, 1], 14, 2, 64, 48, 0, "kv"),
    (False, [513, 64], 24, 1, 128, 64, 0, "nhd"),         # more query heads to a key head than one pass takes
    (False, [77, 333], 6, 6, 48, 3, 0, "hnd"),
    (False, [250, 1111], 16, 16, 80, 16, 0, "nhd"),
    (False, [100, 900], 8, 1, 256, 32, 0, "nhd"),
    (False, [50], 40, 2, 192, 16, 0, "kv"),
    (False, [200, 31], 71, 1, 64, 16, 0, "nhd"),
    (False, [200, 31], 32, 1, 128, 16, 0, "nhd"),
    (False, [5000, 10, 100], 9, 3, 96, 16, 7, "nhd"),     # windows that start and end inside pages
    (False, [5000, 10, 100], 12, 4, 128, 32, 1000, "hnd"),
    (False, [40, 3], 2, 2, 64, 16, 1, "nhd"),
    (True, [1], 1, 1, 16, 1, 0, "nhd"),
    (True, [1, 0, 15, 16, 17, 63, 64, 65], 8, 2, 128, 16, 0, "nhd"),
    (True, [700, 2100], 32, 8, 128, 16, 0, "hnd"),
    (True, [129, 3000, 0, 1], 14, 2, 64, 48, 0, "kv"),
    (True, [513, 64], 24, 1, 128, 64, 0, "nhd"),
    (True, [77, 333], 6, 6, 48, 3, 0, "hnd"),
    (True, [250, 1111], 16, 16, 80, 16, 0, "nhd"),
    (True, [100, 900], 8, 1, 256, 32, 0, "nhd"),
    (True, [100, 900], 20, 1, 256, 32, 50, "nhd"),
    (True, [50], 40, 2, 192, 16, 0, "kv"),
    (True, [200, 31], 71, 1, 64, 16, 0, "nhd"),
    (True, [200, 31], 18, 1, 112, 16, 0, "nhd"),
    (True, [5000, 10, 100], 9, 3, 96, 16, 7, "nhd"),
]


@pytest.mark.parametrize("fp4,lengths,Hq,Hkv,D,page,window,layout", CASES)
def test_matches_the_definition(fp4, lengths, Hq, Hkv, D, page, window, layout):
    o = ops()
    cache, table, k, v = build(fp4, lengths, Hkv, D, page, layout, seed=sum(lengths) + D)
    q = (randn(len(lengths), Hq, D, seed=5) * 1.5).to(torch.bfloat16)
    n = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    scale = D ** -0.5
    out, lse = o.mixfp4_paged_attention(q, cache, table, n, window=window, return_lse=True)
    check(out, lse, q, lengths, k, v, scale, window, fp4)
    again, lse2 = o.mixfp4_paged_attention(q, cache, table, n, window=window, return_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    # a table with room for long sequences: the rows are then cut over the device, not over a cluster
    wide = torch.full((len(lengths), 6000 // page + 9), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    out, lse = o.mixfp4_paged_attention(q, cache, wide, n, window=window if window < 3000 else 0, return_lse=True)
    check(out, lse, q, lengths, k, v, scale, window, fp4)
    if window:  # a window below 4096 would bound them again: the same sequences as their last tokens alone
        out, lse = o.mixfp4_paged_attention(q, cache, wide, n, return_lse=True)
        check(out, lse, q, lengths, k, v, scale, 0, fp4)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("B,longest", [(1, 40000), (3, 20000), (200, 300), (1500, 20)])
def test_many_shares(fp4, B, longest):
    """Sequences cut over many CTAs, many sequences to a CTA, and more sequences than a CTA has threads."""
    o = ops()
    g = torch.Generator().manual_seed(B)
    lengths = torch.randint(0, longest + 1, (B,), generator=g).tolist()
    lengths[0] = longest
    cache, table, k, v = build(fp4, lengths, 2, 64, 16, seed=B)
    q = (randn(B, 8, 64, seed=6) * 1.5).to(torch.bfloat16)
    out, lse = o.mixfp4_paged_attention(q, cache, table, torch.tensor(lengths, dtype=torch.int32, device=DEV),
                                        return_lse=True)
    check(out, lse, q, lengths, k, v, 0.125, 0, fp4)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (16, 2, 256), (24, 1, 64), (6, 3, 80), (48, 1, 32)])
@pytest.mark.parametrize("B,longest,window", [(1, 300, 0), (7, 250, 50), (12, 1000, 0), (40, 100, 0), (60, 130, 50),
                                              (150, 240, 0), (500, 33, 0)])
def test_rows_of_bounded_length(fp4, Hq, Hkv, D, B, longest, window):
    """A cluster of 8, 4 or 2 CTAs to a row, one CTA, or shares of all, as the number of rows and the table allow."""
    o = ops()
    g = torch.Generator().manual_seed(B + D)
    lengths = [int(torch.randint(0, longest + 1, (1,), generator=g)) for _ in range(B)]
    lengths[0], lengths[B // 2] = longest, 0 if B > 1 else longest
    cache, table, k, v = build(fp4, lengths, Hkv, D, 16, "nhd" if B % 2 else "hnd", seed=B)
    q = (randn(B, Hq, D, seed=5) * 1.5).to(torch.bfloat16)
    lens = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    out, lse = o.mixfp4_paged_attention(q, cache, table, lens, window=window, return_lse=True)
    check(out, lse, q, lengths, k, v, D ** -0.5, window, fp4)


@pytest.mark.parametrize("fp4", [False, True])
def test_scores_that_grow_or_shrink_along_the_sequence(fp4):
    """The running maximum moves at every tile, or never after the first."""
    o = ops()
    H, D, n = 2, 128, 4000
    for sign in (1.0, -1.0):
        cache, table, _, _ = build(fp4, [n], H, D, 16, seed=3)
        k = torch.zeros(n, H, D, device=DEV)
        k[:, :, 0] = torch.linspace(-8.0, 8.0, n, device=DEV)[:, None] * sign
        v = randn(n, H, D, seed=11)
        slots = (table[0, :n // 16].long()[:, None] * 16 + torch.arange(16, device=DEV)).reshape(-1)
        o.mixfp4_kv_append(k, v, cache, slots)
        gk, gv = (t.double() for t in o.mixfp4_kv_gather(cache, slots, torch.float32))
        q = torch.zeros(1, 4, D, dtype=torch.bfloat16, device=DEV)
        q[:, :, 0] = torch.tensor([1.0, 30.0, 90.0, 0.0], device=DEV)
        out, lse = o.mixfp4_paged_attention(q, cache, table, torch.tensor([n], dtype=torch.int32, device=DEV),
                                            return_lse=True)
        check(out, lse, q, [n], gk, gv, D ** -0.5, 0, fp4)


@pytest.mark.parametrize("fp4", [False, True])
def test_large_and_tiny_queries(fp4):
    """Heads whose queries differ by many powers of two, and a head of zeros."""
    o = ops()
    H, D, n = 1, 64, 100
    cache, table, k, v = build(fp4, [n], H, D, 16, seed=8)
    q = randn(1, 6, D, seed=9)
    q *= torch.tensor([1.0, 2.0 ** -60, 2.0 ** 60, 0.0, 2.0 ** -120, 1e-3], device=DEV)[None, :, None]
    q = q.to(torch.bfloat16)
    n_ = torch.tensor([n], dtype=torch.int32, device=DEV)
    for rows, scale in (([0, 1, 3, 4, 5], 0.125), ([2], 0.125 * 2.0 ** -60)):
        out, lse = o.mixfp4_paged_attention(q, cache, table, n_, scale=scale, return_lse=True)
        check(out[:, rows], lse[:, rows], q[:, rows], [n], k, v, scale, 0, fp4)


@pytest.mark.parametrize("fp4", [False, True])
def test_pages_outside_the_cache_are_not_seen(fp4):
    o = ops()
    lengths = [100, 40, 16]
    cache, table, k, v = build(fp4, lengths, 2, 64, 16, seed=2)
    table[0, 3], table[1, 0] = -1, cache.pages
    table[2, 0] = -7
    q = randn(3, 4, 64, seed=5).to(torch.bfloat16)
    gone = {b: torch.zeros(n, dtype=torch.bool, device=DEV) for b, n in enumerate(lengths)}
    gone[0][48:64] = True
    gone[1][:16] = True
    gone[2][:] = True
    out, lse = o.mixfp4_paged_attention(q, cache, table, torch.tensor(lengths, dtype=torch.int32, device=DEV),
                                        return_lse=True)
    check(out, lse, q, lengths, k, v, 0.125, 0, fp4, skip=gone)


def test_lengths_outside_the_table():
    """Negative lengths see nothing; one past the table's pages ends with them."""
    o = ops()
    cache, table, k, v = build(False, [32, 32], 2, 64, 16, seed=2)
    q = randn(2, 4, 64, seed=5).to(torch.bfloat16)
    out, lse = o.mixfp4_paged_attention(q, cache, table[:, :2], torch.tensor([-5, 1000], dtype=torch.int32, device=DEV),
                                        return_lse=True)
    check(out, lse, q, [0, 32], k[32:], v[32:], 0.125, 0, False)
    none = o.mixfp4_paged_attention(q, cache, table[:, :0], torch.tensor([3, 3], dtype=torch.int32, device=DEV))
    assert torch.all(none == 0)
    assert o.mixfp4_paged_attention(q[:0], cache, table[:0], torch.empty(0, dtype=torch.int32, device=DEV)).shape[0] == 0


def test_strides_workspace_and_stream():
    o = ops()
    lengths = [300, 5, 1000]
    cache, table, k, v = build(False, lengths, 2, 128, 16, seed=4)
    n = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    fused = randn(3, 3, 8, 128 + 8, seed=5).to(torch.bfloat16)
    q = fused[:, 1, :, :128]
    ref, lse = o.mixfp4_paged_attention(q.contiguous(), cache, table, n, return_lse=True)
    check(ref, lse, q, lengths, k, v, 128 ** -0.5, 0, False)
    need = o.paged_attention_workspace_bytes(cache, 3, 8)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)
    wide = torch.full((3, table.shape[1] + 5), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, glse = torch.empty_like(ref), torch.empty_like(lse)
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    o.mixfp4_paged_attention(q, cache, wide[:, :table.shape[1]], n, out=got, lse=glse, workspace=ws, stream=side)
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
    side.synchronize()
    assert torch.equal(got, ref) and torch.equal(glse, lse)
    with pytest.raises(o.MixFP4Error, match="invalid shape"):
        o.mixfp4_paged_attention(q, cache, table, n, workspace=ws[:-1])


def test_in_a_cuda_graph():
    """Lengths and rows may change between replays."""
    o = ops()
    cache, table, k, v = build(False, [64, 64], 2, 64, 16, seed=4)
    q = randn(2, 4, 64, seed=5).to(torch.bfloat16)
    n = torch.tensor([10, 64], dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o.mixfp4_paged_attention(q, cache, table, n)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = o.mixfp4_paged_attention(q, cache, table, n)
    for lengths in ([10, 64], [0, 1], [64, 33]):
        n.copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        assert torch.equal(out, o.mixfp4_paged_attention(q, cache, table, n))


def test_refusals():
    o = ops()
    cache, table, _, _ = build(False, [20, 20], 2, 64, 16)
    q = randn(2, 4, 64).to(torch.bfloat16)
    n = torch.tensor([20, 20], dtype=torch.int32, device=DEV)
    good = dict(q=q, cache=cache, block_table=table, lengths=n)
    for bad in (dict(q=q.float()), dict(q=q[:, :3]), dict(q=q[..., :32]), dict(q=q[0]), dict(q=q.cpu()), dict(cache=3),
                dict(block_table=table.long()), dict(block_table=table[:1]), dict(block_table=table.cpu()),
                dict(block_table=table[:, ::2]), dict(lengths=n.long()), dict(lengths=n[:1]), dict(window=-1),
                dict(out=q[:1]), dict(out=q.float()), dict(lse=torch.empty(2, 3, device=DEV)),
                dict(workspace=torch.empty(1 << 22, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            o.mixfp4_paged_attention(**{**good, **bad})
    with pytest.raises(o.MixFP4Error, match="misaligned"):
        o.mixfp4_paged_attention(**{**good, "q": randn(2, 4, 68).to(torch.bfloat16)[..., 4:]})
