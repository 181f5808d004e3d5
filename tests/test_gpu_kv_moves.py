"""Rows and pages moved within the paged cache (accepted drafts, forks, copies):
bit for bit what indexing gives, and nothing else in the cache changes."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def ops():
    from paper_2605_31035_gb300 import ops as o
    return o


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


def fill(pages, page, H, D, fp4, layout, seed):
    """A cache of random bits in one of the layouts."""
    g = torch.Generator(DEV).manual_seed(seed)

    def alloc(n):
        if layout == "kv":
            t = torch.randint(0, 256, (pages, 2, page, H, n), generator=g, device=DEV, dtype=torch.uint8)
            return t[:, 0], t[:, 1]
        if layout == "padded":  # room behind a row, a token and a page
            t = torch.randint(0, 256, (2, pages, page + 1, H + 1, n + 32), generator=g, device=DEV, dtype=torch.uint8)
            return t[0, :, :page, :H, :n], t[1, :, :page, :H, :n]
        shape = (2, pages, H, page, n) if layout == "hnd" else (2, pages, page, H, n)
        t = torch.randint(0, 256, shape, generator=g, device=DEV, dtype=torch.uint8)
        return (t[0].transpose(1, 2), t[1].transpose(1, 2)) if layout == "hnd" else (t[0], t[1])
    o = ops()
    if fp4:
        ts = torch.ones(1, device=DEV)
        return o.KVCache(*alloc(D // 2), *alloc(D // 16), ts, ts)
    return o.KVCache(*(x.view(torch.bfloat16) for x in alloc(D * 2)))


def arrays(cache):
    return [x if x.dtype is torch.uint8 else x.view(torch.int16)
            for x in (cache.k, cache.v, cache.k_scales, cache.v_scales) if x is not None]


def table_of(lengths, page, pages, seed, width=None):
    order = list(range(pages))
    random.Random(seed).shuffle(order)
    width = width or max([-(-n // page) for n in lengths] + [1])
    table, at = [], 0
    for n in lengths:
        need = -(-n // page)
        table.append(order[at:at + need] + [-1] * (width - need))
        at += need
    assert at <= pages
    return table, order[at:]


SHAPES = [  # page, heads, head_dim, layout
    (16, 8, 128, "nhd"), (16, 8, 128, "hnd"), (64, 2, 64, "kv"), (1, 1, 16, "nhd"), (3, 6, 48, "hnd"), (16, 3, 80, "kv"),
    (48, 2, 256, "nhd"), (7, 5, 32, "padded"), (32, 1, 192, "padded"), (128, 4, 112, "nhd"), (16, 33, 128, "nhd"),
    (1, 3, 64, "hnd"), (5, 1, 16, "hnd"),
]


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("page,H,D,layout", SHAPES)
@pytest.mark.parametrize("n", [0, 1, 37])
def test_copy_pages(fp4, page, H, D, layout, n):
    cache = fill(3 * n + 5, page, H, D, fp4, layout, seed=n + D)
    order = list(range(cache.pages))
    random.Random(n).shuffle(order)
    src, dst = order[:n], order[n:2 * n]
    if n > 8:
        src[1] = src[0]                     # one page to two places
        dst[2] = src[2]                     # its own copy
        src[3], dst[4] = -1, cache.pages    # left out
        src[5], dst[6] = 2 ** 31 - 1, -2 ** 31
    want = [x.clone() for x in arrays(cache)]
    for s, d in zip(src, dst):
        if 0 <= s < cache.pages and 0 <= d < cache.pages:
            for w, x in zip(want, arrays(cache)):
                w[d] = x[s]
    ops().mixfp4_kv_copy_pages(cache, ints(src), ints(dst))
    for w, x in zip(want, arrays(cache)):
        assert torch.equal(w, x)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("page,H,D,layout", SHAPES)
def test_accept(fp4, page, H, D, layout):
    """Paths of every kind: in order, with sources among the places written, out of order, twice the same draft, ending
    early; sequences without drafts, without tokens; counts past the length."""
    o = ops()
    rng = random.Random(D + page)
    lengths = [70, 0, 64, 5, 100, 33, 90, 12, 81]
    counts = [64, 0, 64, 9, 40, 0, 64, 12, 63]
    depth = 64
    paths = [sorted(rng.sample(range(64), 20)), [0, 1], list(range(64)), [1, 3], rng.sample(range(40), 40), [0],
             [63] * 10 + [0, 5, 63, 2], [2, 12, 3], [3, 1, 0, -1, 2]]
    paths = [p + [-1] * (depth - len(p)) for p in paths]
    pages = sum(-(-n // page) for n in lengths) + 3
    cache = fill(pages, page, H, D, fp4, layout, seed=page)
    table, _ = table_of(lengths, page, pages, seed=D)
    before = [x.clone() for x in arrays(cache)]
    want = [x.clone() for x in before]
    new = []
    for b, (n, c) in enumerate(zip(lengths, counts)):
        c = min(c, n)
        k = 0
        while k < depth and 0 <= paths[b][k] < c:
            s, d = n - c + paths[b][k], n - c + k
            for w, x in zip(want, before):
                w[table[b][d // page], d % page] = x[table[b][s // page], s % page]
            k += 1
        new.append(n - c + k)
    n = ints(lengths)
    got = o.mixfp4_kv_accept(cache, ints(table), n, ints(paths), ints(counts))
    assert got.tolist() == new and n.tolist() == lengths
    for w, x in zip(want, arrays(cache)):
        assert torch.equal(w, x)


def test_accept_in_place_and_outside():
    """lengths changed in place by every CTA's reckoning alike; places on pages outside the cache or behind the table stay
    and give nothing; a path of no entries."""
    o = ops()
    cache = fill(40, 4, 33, 128, False, "nhd", seed=1)
    table = [[0, 1, -1, 3], [4, 5, 6, 40], [7, 8, 9, 10]]
    lengths, counts = [16, 16, 20], [12, 12, 12]
    paths = [[1, 5, 8, 9], [9, 10, 3, 4], [2, 7, 8, 9]]
    before = [x.clone() for x in arrays(cache)]
    want = [x.clone() for x in before]
    for b in range(3):
        for k, j in enumerate(paths[b]):
            s, d = lengths[b] - counts[b] + j, lengths[b] - counts[b] + k
            if s < 16 and d < 16 and 0 <= table[b][s // 4] < 40 and 0 <= table[b][d // 4] < 40:
                for w, x in zip(want, before):
                    w[table[b][d // 4], d % 4] = x[table[b][s // 4], s % 4]
    n = ints(lengths)
    got = o.mixfp4_kv_accept(cache, ints(table), n, ints(paths), ints(counts), out=n)
    assert got.data_ptr() == n.data_ptr() and n.tolist() == [8, 8, 12]
    for w, x in zip(want, arrays(cache)):
        assert torch.equal(w, x)
    n = ints(lengths)
    assert o.mixfp4_kv_accept(cache, ints(table), n, ints(paths)[:, :0], ints(counts)).tolist() == [4, 4, 8]
    assert o.mixfp4_kv_accept(cache, ints(table)[:0], n[:0], ints(paths)[:0], n[:0]).numel() == 0
    for w, x in zip(want, arrays(cache)):
        assert torch.equal(w, x)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("page,H,D,layout", SHAPES)
def test_fork(fp4, page, H, D, layout):
    o = ops()
    lengths = [3 * page, 2 * page + max(1, page // 2), 1, 0, page - 1 if page > 1 else 2, 5 * page + page // 3]
    parents = [1, 1, 0, 5, 5, -1, 2, 6, 3, 4, 1, 2]
    pages = sum(-(-n // page) for n in lengths) + len(parents) + 2
    cache = fill(pages, page, H, D, fp4, layout, seed=page + 1)
    table, spare = table_of(lengths, page, pages, seed=D, width=8)
    fresh = [spare[i] for i in range(len(parents))]
    fresh[1], fresh[4] = -1, cache.pages
    want = [x.clone() for x in arrays(cache)]
    want_table, want_n = [], []
    for p, f in zip(parents, fresh):
        if not 0 <= p < len(lengths):
            want_table.append([-1] * 8)
            want_n.append(0)
            continue
        row, part = list(table[p]), lengths[p] % page
        if part and 0 <= f < cache.pages:
            for w, x in zip(want, arrays(cache)):
                w[f, :part] = x[row[lengths[p] // page], :part]
            row[lengths[p] // page] = f
        want_table.append(row)
        want_n.append(lengths[p])
    got, n = o.mixfp4_kv_fork(cache, ints(table), ints(lengths), ints(parents), ints(fresh))
    assert got.tolist() == want_table and n.tolist() == want_n
    for w, x in zip(want, arrays(cache)):
        assert torch.equal(w, x)


def test_fork_outside():
    """A last page outside the cache is not copied, a length past the table has no last page, negative ones are 0."""
    o = ops()
    cache = fill(20, 4, 2, 64, False, "nhd", seed=1)
    before = [x.clone() for x in arrays(cache)]
    table = [[0, -1, 2], [3, 4, 5], [6, 7, 8]]
    got, n = o.mixfp4_kv_fork(cache, ints(table), ints([6, 13, -3]), ints([0, 1, 2]), ints([10, 11, 12]))
    assert got.tolist() == [[0, 10, 2], [3, 4, 5], [6, 7, 8]] and n.tolist() == [6, 13, 0]
    for w, x in zip(before, arrays(cache)):
        assert torch.equal(w, x)
    got, n = o.mixfp4_kv_fork(cache, ints(table)[:, :0], ints([6, 13, -3]), ints([0, 1]), ints([10, 11]))
    assert got.shape == (2, 0) and n.tolist() == [6, 13]
    assert o.mixfp4_kv_fork(cache, ints(table), ints([6, 13, -3]), ints([]), ints([]))[0].shape == (0, 3)


def test_streams_and_graphs():
    """On another stream than the current one, and captured: what changes between replays is read anew."""
    o = ops()
    cache = fill(64, 16, 4, 128, True, "nhd", seed=2)
    src, dst = ints([1, 2, 3]), ints([11, 12, 13])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    o.mixfp4_kv_copy_pages(cache, src, dst, stream=side)
    table, n = o.mixfp4_kv_fork(cache, ints([[0, 1]]), ints([20]), ints([0, 0]), ints([20, 21]), stream=side)
    out = o.mixfp4_kv_accept(cache, table, n, ints([[1], [2]]), ints([3, 3]), stream=side)
    side.synchronize()
    assert torch.equal(cache.k[11:14], cache.k[1:4]) and table.tolist() == [[0, 20], [0, 21]]
    # 20 tokens with 3 drafts at 17, 18 and 19: child 0 keeps the second one, child 1 the third
    assert out.tolist() == [18, 18]
    for child, row in ((20, 2), (21, 3)):
        assert torch.equal(cache.v[child, 1], cache.v[1, row]) and torch.equal(cache.k_scales[child, 1], cache.k_scales[1, row])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o.mixfp4_kv_copy_pages(cache, src, dst)
    src.copy_(ints([5, 6, 7]))
    graph.replay()
    assert torch.equal(cache.k[11:14], cache.k[5:8]) and torch.equal(cache.v_scales[11:14], cache.v_scales[5:8])


def test_refusals():
    o = ops()
    cache = fill(20, 4, 2, 64, False, "nhd", seed=1)
    table, n, c, path = ints([[0, 1], [2, 3]]), ints([8, 8]), ints([2, 2]), ints([[0], [1]])
    good = dict(cache=cache, block_table=table, lengths=n, path=path, counts=c)
    for bad in (dict(cache=None), dict(block_table=table.long()), dict(block_table=table[:1]), dict(lengths=n.long()),
                dict(lengths=n.cpu()), dict(path=path.long()), dict(path=path[:1]), dict(path=path[:, :1].expand(2, 65)),
                dict(path=path[:1].expand(2, 1)[:, [0, 0]].t()), dict(counts=c[:1]), dict(counts=c.long()),
                dict(out=n.long()), dict(out=n[:1])):
        with pytest.raises(ValueError):
            o.mixfp4_kv_accept(**{**good, **bad})
    for out in (c, path[:, 0].reshape(2)):
        if out.data_ptr() == path.data_ptr() or out is c:
            with pytest.raises(o.MixFP4Error, match="argument"):
                o.mixfp4_kv_accept(**{**good, "out": out})
    good = dict(cache=cache, block_table=table, lengths=n, parents=ints([0]), fresh=ints([9]))
    for bad in (dict(cache=None), dict(block_table=table[0]), dict(block_table=table[:1]), dict(lengths=n.float()),
                dict(parents=ints([0]).long()), dict(fresh=ints([9, 8])), dict(fresh=ints([9]).cpu()),
                dict(out=(ints([[0]]), ints([0]))), dict(out=(ints([[0, 0]]), ints([0, 0])))):
        with pytest.raises(ValueError):
            o.mixfp4_kv_fork(**{**good, **bad})
    for out in ((table[1:], ints([0])), (ints([[0, 0]]), n[:1])):
        with pytest.raises(o.MixFP4Error, match="argument"):
            o.mixfp4_kv_fork(**{**good, "out": out})
    for bad in (dict(src=ints([1]).long()), dict(src=ints([1]).cpu()), dict(src=ints([[1]])), dict(dst=ints([1, 2])),
                dict(cache=7)):
        with pytest.raises(ValueError):
            o.mixfp4_kv_copy_pages(**{**dict(cache=cache, src=ints([1]), dst=ints([2])), **bad})
