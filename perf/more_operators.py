"""Performance cases of the operators for drafted tokens and shared pages: what is measured.

They stand beside the paged cache's append, gather and one-token attention:

* ``tree``    attention of up to 64 drafted tokens per sequence, a tree by its
  ancestor masks, over the paged cache (bf16 or MixFP4); one token a sequence is
  its smallest form.  Scores may be capped by a tanh and get a bias that
  grows with distance, and a sliding window may bound what is seen.
* ``accept``  the accepted drafts' rows move to the places behind the prefix.
* ``fork``    sequences branch: tables and lengths of the children, and a page of
  their own for the last, partly filled page.
* ``copy``    pages copied within a pool (what compacting it does).

With ``own`` false, ``run`` computes the same in elementary torch operations in
32 bits; ``exact`` restates the definitions in 64 bits.
"""
import functools
import math
import random

import torch

own = False

DEV = "cuda:0"

# ---------------------------------------------------------------------- cases


def listed():
    return [
        # One new token of one sequence under capped scores, a short context: the smallest call, where latency is all.
        dict(name="tree_1x700_cap", op="tree", B=1, t=1, longest=700, even=True, Hq=32, Hkv=8, D=128, page=16,
             window=0, cap=50.0, bias=False, chain=True, fp4=False, hnd=False, mix=1),
        # A decode batch of ragged contexts up to 8192 tokens, trees of 8 drafts (8B heads).
        dict(name="tree_64x8192_8", op="tree", B=64, t=8, longest=8192, even=False, Hq=32, Hkv=8, D=128, page=16,
             window=0, cap=0.0, bias=False, chain=False, fp4=False, hnd=False, mix=2),
        # The same on a MixFP4 cache.
        dict(name="tree_64x8192_8_fp4", op="tree", B=64, t=8, longest=8192, even=False, Hq=32, Hkv=8, D=128, page=16,
             window=0, cap=0.0, bias=False, chain=False, fp4=True, hnd=False, mix=3),
        # Wide trees over long contexts (70B heads): arithmetic, not the cache, takes the time.
        dict(name="tree_8x16384_64", op="tree", B=8, t=64, longest=16384, even=False, Hq=64, Hkv=8, D=128, page=64,
             window=0, cap=0.0, bias=False, chain=False, fp4=False, hnd=True, mix=4),
        # Two very long contexts on a MixFP4 cache, a chain of 4 drafts, bias by distance: the cache's length is split.
        dict(name="tree_2x131072_bias_fp4", op="tree", B=2, t=4, longest=131072, even=True, Hq=32, Hkv=8, D=128,
             page=64, window=0, cap=0.0, bias=True, chain=True, fp4=True, hnd=True, mix=5),
        # Seven query heads to a key head, narrow heads, a window, capped scores, trees of 13 or fewer, empty sequences.
        dict(name="tree_33_window_cap", op="tree", B=33, t=13, longest=3333, even=False, Hq=14, Hkv=2, D=64, page=32,
             window=1000, cap=30.0, bias=False, chain=False, fp4=False, hnd=False, mix=6),
        # A decode batch whose trees have been verified.
        dict(name="accept_8", op="accept", B=8, t=16, longest=100, Hkv=8, D=128, page=16, hnd=False, mix=7),
        # A large batch of wide trees.
        dict(name="accept_256", op="accept", B=256, t=64, longest=100, Hkv=8, D=128, page=16, hnd=True, mix=8),
        # One prompt in four beams.
        dict(name="fork_4", op="fork", B=1, n=4, longest=1000, Hkv=8, D=128, page=16, fp4=False, hnd=False, mix=9),
        # A large batch goes on in two branches each, MixFP4 cache with large pages; the copied rows are read back.
        dict(name="fork_512_fp4", op="fork", B=256, n=512, longest=2000, Hkv=8, D=128, page=64, fp4=True, hnd=False,
             mix=10),
        # A few pages move.
        dict(name="copy_5", op="copy", n=5, pages=64, Hkv=8, D=128, page=16, hnd=False, mix=11),
        # A pool is compacted: 4099 pages (268 MB) move to its beginning.
        dict(name="copy_4099", op="copy", n=4099, pages=9000, Hkv=8, D=128, page=16, hnd=False, mix=12),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# (query heads, key heads, head dimension): grouped, multi-head and multi-query forms, wide and odd ones
_HEADS = [(32, 8, 128), (64, 8, 128), (32, 32, 128), (14, 2, 64), (28, 4, 128), (16, 2, 256), (8, 1, 256), (24, 1, 128),
          (12, 4, 96), (16, 16, 80), (40, 8, 128), (9, 3, 64), (6, 6, 48)]


def draw(rng):
    op = rng.choice(["tree"] * 6 + ["accept", "fork", "copy"])
    Hq, Hkv, D = rng.choice(_HEADS)
    page, hnd, mix = rng.choice([16, 16, 32, 64, 48, 128]), rng.random() < 0.4, rng.randrange(20, 1 << 20)
    if op == "tree":
        B, longest, t = _log(rng, 1, 256), _log(rng, 1, 131072), _log(rng, 1, 64)
        while B * longest * Hkv * D > 64 * 8192 * 8 * 128 or B * longest * t * Hq * D > 8 * 16384 * 64 * 64 * 128 / 2:
            if rng.random() < 0.5:
                B = max(1, B // 2)
            else:
                longest = max(1, longest * 2 // 3)
        return dict(op=op, B=B, t=t, longest=max(longest, t), even=rng.random() < 0.3, Hq=Hq, Hkv=Hkv, D=D, page=page,
                    window=rng.choice([0, 0, 0, _log(rng, 1, 4096)]), cap=rng.choice([0.0, 0.0, 0.0, 30.0, 50.0]),
                    bias=rng.random() < 0.25, chain=rng.random() < 0.25, fp4=rng.random() < 0.5, hnd=hnd, mix=mix)
    if op == "accept":
        B, t = _log(rng, 1, 256), _log(rng, 1, 64)
        while B * (100 + t) * Hkv * D > 256 * 164 * 8 * 128:
            B = max(1, B // 2)
        return dict(op=op, B=B, t=t, longest=_log(rng, 1, 100), Hkv=Hkv, D=D, page=page, hnd=hnd, mix=mix)
    if op == "fork":
        B, n, longest = _log(rng, 1, 256), _log(rng, 1, 512), _log(rng, 1, 2000)
        while n * page * Hkv * D > 512 * 64 * 8 * 128:
            n = max(1, n // 2)
        while B * longest * Hkv * D > 256 * 2000 * 8 * 128:
            longest = max(1, longest // 2)
        return dict(op=op, B=B, n=n, longest=longest, Hkv=Hkv, D=D, page=page, fp4=rng.random() < 0.5, hnd=hnd, mix=mix)
    n = _log(rng, 1, 4096)
    while n * page * Hkv * D > 4096 * 16 * 8 * 128:
        n = max(1, n // 2)
    return dict(op=op, n=n, pages=2 * n + rng.randrange(1, 1 + n), Hkv=Hkv, D=D, page=page, hnd=hnd, mix=mix)


def _lengths(case):
    """Tokens in the cache of each sequence, the drafted ones included, and how many those are."""
    B, t, longest = case["B"], case["t"], case["longest"]
    if case.get("even"):
        return [longest] * B, [t] * B
    rng = random.Random(case["mix"])
    n = [rng.randint(1, max(1, longest - t)) + t for _ in range(B)]
    c = [rng.randint(1, t) if rng.random() < 0.3 else t for _ in range(B)]
    n[rng.randrange(B)] = max(longest, t)
    if B >= 16:
        i = rng.randrange(B)
        n[i] = c[i] = 0  # a slot of the batch without a request
    return n, c


def _tree(case, b):
    """Ancestors of each draft of sequence b, itself included, as bits."""
    t = case["t"]
    if case["chain"]:
        return [(2 << i) - 1 for i in range(t)]
    rng = random.Random(case["mix"] * 4099 + b)
    seen = []
    for i in range(t):
        seen.append(1 << i | (seen[rng.randrange(max(0, i - 6), i)] if i else 0))
    return seen


def _paths(case):
    """Accepted drafts of each sequence: the first ones as drafted, then others behind the places they all go to."""
    n, c = _lengths(case)
    paths = []
    for b, count in enumerate(c):
        rng = random.Random(case["mix"] * 5003 + b)
        a = rng.randint(1, max(1, min(count, 12))) if count else 0
        first = rng.randint(max(0, 2 * a - count), a)
        paths.append(list(range(first)) + sorted(rng.sample(range(a, count), a - first)))
    return n, c, paths


def _fork(case):
    """Lengths of the sequences and, of each child, its parent and whether it gets a page of its own."""
    rng = random.Random(case["mix"])
    n = [rng.randint(1, case["longest"]) for _ in range(case["B"])]
    n[rng.randrange(case["B"])] = case["longest"]
    parents = [i % case["B"] if rng.random() < 0.8 else rng.randrange(case["B"]) for i in range(case["n"])]
    return n, parents


def work(case):
    if case["op"] == "tree":
        n, c = _lengths(case)
        row = case["D"] * 9 / 16 if case["fp4"] else case["D"] * 2
        read = flops = 0
        for a, k in zip(n, c):
            seen = min(a, case["window"] + k) if case["window"] else a
            read += seen
            flops += 4 * min(seen, case["window"] or seen) * k * case["Hq"] * case["D"]
        return {"bytes": read * (case["Hkv"] * row * 2 + 4 / case["page"]) +
                case["B"] * case["t"] * (case["Hq"] * (case["D"] * 4 + 4) + 8), "flops": flops}
    row = case["Hkv"] * case["D"] * 2 * 2
    if case["op"] == "accept":
        moved = sum(sum(i != k for k, i in enumerate(p)) for p in _paths(case)[2])
        return {"bytes": 2 * moved * row + case["B"] * 4 * (case["t"] + 3), "flops": 0}
    if case["op"] == "fork":
        n, parents = _fork(case)
        rows = sum(n[p] % case["page"] for p in parents)
        table = case["n"] * -(-case["longest"] // case["page"]) * 8
        if case["fp4"]:  # copied, then read back and returned in bf16
            return {"bytes": rows * row * 9 / 32 * 3 + rows * row + table, "flops": 0}
        return {"bytes": 2 * rows * row + table, "flops": 0}
    return {"bytes": 2 * case["n"] * case["page"] * row + 8 * case["n"], "flops": 0}


# --------------------------------------------------------------------- inputs


def _gen(seed, which):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + which)
    return g


@functools.lru_cache(maxsize=None)
def _t(v):
    """A constant (number or tuple) on the GPU, made once."""
    return torch.tensor(v, dtype=torch.float32, device=DEV)


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


def _paged(rows, hnd):
    """Rows [pages, page, heads, n] stored in that order or, with hnd, head by head within a page."""
    return rows.transpose(1, 2).contiguous().transpose(1, 2) if hnd else rows.contiguous()


def _cache(case, pages, seed):
    """A cache of `pages` pages: keys with a few strong channels, values without.  A MixFP4 cache holds codes of both
    books in random order and block scales that make their rows as large as the bf16 cache's."""
    page, H, D, hnd = case["page"], case["Hkv"], case["D"], case["hnd"]
    c = {}
    for which, name in ((11, "k"), (12, "v")):
        g = _gen(seed, which)
        gain = torch.ones(H, D, device=DEV)
        if name == "k":
            gain[torch.rand(H, D, generator=g, device=DEV) < 0.03] = 6.0
        if case.get("fp4"):
            codes = torch.randint(0, 256, (pages, page, H, D // 2), generator=g, device=DEV, dtype=torch.uint8)
            # E4M3 bytes of 2^(e - 7) (1 + f / 8) around the block's gain, the book in the sign bit
            top = gain.view(H, D // 16, 16).amax(-1)
            f = torch.randint(0, 8, (pages, page, H, D // 16), generator=g, device=DEV, dtype=torch.uint8)
            book = torch.randint(0, 2, f.shape, generator=g, device=DEV, dtype=torch.uint8)
            e = (10.0 + torch.log2(top).floor()).to(torch.uint8)
            scales = book << 7 | e << 3 | f
            c[name], c[name + "s"] = _paged(codes, hnd), _paged(scales, hnd)
            c[name + "t"] = _t((0.036,))
        else:
            x = torch.empty(pages, page, H, D, dtype=torch.bfloat16, device=DEV)
            step = max(1, (1 << 26) // (page * H * D))
            for i in range(0, pages, step):
                x[i:i + step] = torch.randn(x[i:i + step].shape, generator=g, device=DEV) * gain
            c[name] = _paged(x, hnd)
    return c


def _tables(n, page, g, width=None):
    """Pages of sequences of n[b] tokens in a shuffled pool: table (-1 behind a sequence's pages) and pool size."""
    need = _ints([-(-k // page) for k in n], torch.int64)
    total = int(sum(-(-k // page) for k in n))
    pool = torch.randperm(total + 1, generator=g, device=DEV).to(torch.int32)
    ends = need.cumsum(0)
    i = torch.arange(width or max(1, -(-max(n) // page)), device=DEV)
    at = (ends - need)[:, None] + i
    return torch.where(at < ends[:, None], pool[at.clamp(max=total)], -1), total + 1


def _signed(bits):
    return bits - (1 << 64) if bits >= 1 << 63 else bits


def _inputs(case, seed):
    g = _gen(seed, 2)
    page = case["page"]
    if case["op"] == "tree":
        n, c = _lengths(case)
        table, pages = _tables(n, page, g)
        q = (torch.randn(case["B"], case["t"], case["Hq"], case["D"], generator=g, device=DEV) * 1.5)
        mask = None
        if not case["chain"]:
            mask = _ints([[_signed(m) for m in _tree(case, b)] for b in range(case["B"])], torch.int64)
        slopes = None
        if case["bias"]:
            slopes = torch.exp2(-8.0 * torch.arange(1, case["Hq"] + 1, device=DEV) / case["Hq"]).float()
        return dict(q=q.to(torch.bfloat16), table=table, n=_ints(n), counts=_ints(c), mask=mask, slopes=slopes,
                    pages=pages, scale=case["D"] ** -0.5)
    if case["op"] == "accept":
        n, c, paths = _paths(case)
        table, pages = _tables(n, page, g)
        path = _ints([p + [-1] * (case["t"] - len(p)) for p in paths])
        return dict(table=table, n=_ints(n), counts=_ints(c), path=path, pages=pages)
    if case["op"] == "fork":
        n, parents = _fork(case)
        table, pages = _tables(n, page, g)
        fresh = [pages + i if n[p] % page else -1 for i, p in enumerate(parents)]
        st = dict(table=table, n=_ints(n), parents=_ints(parents), fresh=_ints(fresh), pages=pages + len(parents))
        st["slots"] = _ints([f * page + j for f, p in zip(fresh, parents) for j in range(n[p] % page)], torch.int64)
        return st
    order = torch.randperm(case["pages"], generator=g, device=DEV).to(torch.int32)
    return dict(src=order[:case["n"]].contiguous(), dst=order[case["n"]:2 * case["n"]].contiguous(),
                pages=case["pages"])


def prepare(case, seed):
    st = _inputs(case, seed)
    st["cache"] = _cache(case, st["pages"], seed)
    st["case"] = case
    if own:  # the handle that a user's program keeps
        from paper_2605_31035_gb300 import ops
        c = st["cache"]
        st["kv"] = ops.KVCache(c["k"], c["v"], c.get("ks"), c.get("vs"), c.get("kt"), c.get("vt"))
    return st


# ------------------------------------------------------------------------ run


def run(st):
    case = st["case"]
    if own:
        return _run_own(case, st)
    return {"tree": _tree_plain, "accept": _accept_plain, "fork": _fork_plain, "copy": _copy_plain}[case["op"]](case, st)


def _run_own(case, st):
    from paper_2605_31035_gb300 import ops
    kv, c = st["kv"], st["cache"]
    if case["op"] == "tree":
        return ops.mixfp4_tree_attention(st["q"], kv, st["table"], st["n"], mask=st["mask"], counts=st["counts"],
                                         scale=st["scale"], window=case["window"], softcap=case["cap"],
                                         slopes=st["slopes"], return_lse=True)
    if case["op"] == "accept":
        return ops.mixfp4_kv_accept(kv, st["table"], st["n"], st["path"], st["counts"]), c["k"], c["v"]
    if case["op"] == "fork":
        table, n = ops.mixfp4_kv_fork(kv, st["table"], st["n"], st["parents"], st["fresh"])
        return (table, n, *_fork_rows(case, st, lambda: ops.mixfp4_kv_gather(kv, st["slots"])))
    ops.mixfp4_kv_copy_pages(kv, st["src"], st["dst"])
    return c["k"], c["v"]


def _fork_rows(case, st, gather):
    """What a fork is followed by here: of a bf16 cache the cache itself, of a MixFP4 one the copied rows as values."""
    return gather() if case["fp4"] else (st["cache"]["k"], st["cache"]["v"])


_BOOKS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0,
          0.0, 1.0, 2.0, 3.0, 4.0, 5.0, 6.0, 7.0, -0.0, -1.0, -2.0, -3.0, -4.0, -5.0, -6.0, -7.0)


def _values(codes, scales, ts):
    """MixFP4 rows in fp32."""
    nib = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).unflatten(-1, (-1, 16)) + (scales >> 7)[..., None] * 16
    s8 = (scales & 127).view(torch.float8_e4m3fn).float()
    return (_t(_BOOKS)[nib.int()] * (s8 * ts)[..., None]).flatten(-2)


def _rows(c, name, pages, fp4):
    """The cache's rows of these pages in fp32."""
    return _values(c[name][pages], c[name + "s"][pages], c[name + "t"]) if fp4 else c[name][pages].float()


def _seen(case, st, L):
    """Of each draft, which of L cached tokens it sees [B, t, L], and their distance from it."""
    B, t = case["B"], case["t"]
    i = torch.arange(t, device=DEV)
    mask = st["mask"] if st["mask"] is not None else _ints([_signed((2 << k) - 1) for k in range(t)], torch.int64)
    bits = ((mask[..., None] >> i) & 1).bool().expand(B, t, t)
    depth = (bits & (i != i[:, None])).sum(-1)  # [B, t]
    n, c = st["n"].long()[:, None], st["counts"].long()[:, None]
    pos = torch.arange(L, device=DEV)
    draft = pos - (n - c)  # [B, L]: which draft a token is
    is_draft = (draft >= 0) & (pos < n)
    at = draft.clamp(0, t - 1)
    seen = torch.where(is_draft[:, None], bits.gather(2, at[:, None].expand(B, t, L)), (draft < 0)[:, None])
    place = torch.where(is_draft, n - c + depth.gather(1, at), pos)  # a draft stands behind its ancestors
    far = (n - c + depth)[..., None] - place[:, None]
    if case["window"]:
        seen = seen & (far < case["window"])
    return seen & (i < c)[..., None], far


def _tree_plain(case, st):
    B, t, Hq, Hkv, D = (case[k] for k in ("B", "t", "Hq", "Hkv", "D"))
    G = Hq // Hkv
    pages = st["table"].clamp(min=0).long()
    k = _rows(st["cache"], "k", pages, case["fp4"]).flatten(1, 2).transpose(1, 2)  # [B, Hkv, L, D]
    v = _rows(st["cache"], "v", pages, case["fp4"]).flatten(1, 2).transpose(1, 2)
    L = k.shape[2]
    seen, far = _seen(case, st, L)
    q = st["q"].float().view(B, t, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * t, D)
    s = torch.matmul(q, k.transpose(2, 3)).view(B, Hkv, G, t, L).mul_(st["scale"])
    if case["cap"]:
        s = torch.tanh(s / case["cap"]) * case["cap"]
    if case["bias"]:
        s = s - st["slopes"].view(Hkv, G, 1, 1) * far.float()[:, None, None]
    s = s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(m > -math.inf, m, torch.zeros_like(m))).exp_()
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, G * t, L), v).view(B, Hkv, G, t, D) / torch.where(z > 0, z, torch.ones_like(z))
    lse = (m + torch.log(z)).squeeze(-1)
    return (o.permute(0, 3, 1, 2, 4).reshape(B, t, Hq, D).to(torch.bfloat16),
            lse.permute(0, 3, 1, 2).reshape(B, t, Hq))


def _accept_plain(case, st):
    page, path = case["page"], st["path"]
    good = (path >= 0) & (path < st["counts"][:, None])
    good = good.int().cumprod(1).bool()  # the path ends at its first entry that is no draft
    first = (st["n"] - st["counts"]).long()[:, None]
    k = torch.arange(path.shape[1], device=DEV)
    src, dst = first + path.clamp(min=0), first + k
    b = torch.arange(case["B"], device=DEV)[:, None].expand_as(src)

    def slot(pos):
        last = st["table"].shape[1] * page - 1
        return st["table"].long()[b, pos.clamp(max=last) // page] * page + pos % page
    s, d = slot(src)[good], slot(dst)[good]
    for x in (st["cache"]["k"], st["cache"]["v"]):
        x[d // page, d % page] = x[s // page, s % page]
    return (first.squeeze(1) + good.sum(1)).int(), st["cache"]["k"], st["cache"]["v"]


def _fork_plain(case, st):
    page, c = case["page"], st["cache"]
    p = st["parents"].long()
    n, table = st["n"][p], st["table"][p]
    part = (n % page)[:, None]
    last = (n // page).long().clamp(max=table.shape[1] - 1)[:, None]
    own_page = (st["fresh"] >= 0)[:, None] & (part > 0)
    old = table.gather(1, last)
    table = table.scatter(1, last, torch.where(own_page, st["fresh"][:, None], old))
    j = torch.arange(page, device=DEV)
    use = own_page & (j < part)
    src, dst = old.long().expand_as(use)[use], st["fresh"].long()[:, None].expand_as(use)[use]
    at = j.expand_as(use)[use]
    for name in ("k", "v", "ks", "vs"):
        if name in c:
            c[name][dst, at] = c[name][src, at]

    def gather():
        s = st["slots"]
        return tuple(_values(c[x][s // page, s % page], c[x + "s"][s // page, s % page], c[x + "t"]).to(torch.bfloat16)
                     for x in ("k", "v"))
    return (table, n, *_fork_rows(case, st, gather))


def _copy_plain(case, st):
    c, src, dst = st["cache"], st["src"].long(), st["dst"].long()
    for name in ("k", "v"):
        c[name][dst] = c[name][src]
    return c["k"], c["v"]


# ---------------------------------------------------------------------- exact


def exact(case, seed):
    if case["op"] == "tree":
        return _tree_exact(case, seed)
    t = _inputs(case, seed)
    c = _cache(case, t["pages"], seed)
    return {"accept": _accept_exact, "fork": _fork_exact, "copy": _copy_exact}[case["op"]](case, t, c)


def _rows64(c, name, fp4):
    """Rows in 64 bits (a MixFP4 value is sign * codebook value * block scale * tensor scale)."""
    x = c[name]
    if not fp4:
        return x.double()
    sc = c[name + "s"]
    e, f = ((sc & 127) >> 3).double(), (sc & 7).double()
    s8 = torch.where(e > 0, torch.exp2(e - 7) * (1 + f / 8), f * 2.0 ** -9).repeat_interleave(16, -1)
    one = (sc >> 7).repeat_interleave(16, -1).bool()
    nib = torch.stack([x & 15, x >> 4], -1).flatten(-2)
    p = (nib & 7).double()
    e2, m2 = torch.floor(p / 2), p % 2
    mag = torch.where(one, p, torch.where(e2 > 0, torch.exp2(e2 - 1) * (1 + m2 / 2), m2 / 2))
    return torch.where(nib > 7, -mag, mag) * s8 * c[name + "t"].double()


def _tree_exact(case, seed):
    x = _inputs(case, seed)
    c = _cache(case, x["pages"], seed)
    t, Hq, D, page = (case[k] for k in ("t", "Hq", "D", "page"))
    G = Hq // case["Hkv"]
    out = torch.zeros(case["B"], t, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.full((case["B"], t, Hq), -math.inf, dtype=torch.float64, device=DEV)
    for b, (n, count) in enumerate(zip(*_lengths(case))):
        if n == 0:
            continue
        tree = _tree(case, b)[:count]
        above = [[i != j and bool(tree[i] >> j & 1) for j in range(count)] for i in range(count)]
        depth = torch.tensor([sum(r) for r in above], device=DEV)
        first = n - count
        place = torch.cat([torch.arange(first, device=DEV), first + depth])
        far = (first + depth)[:, None] - place
        sees = torch.ones(count, n, dtype=torch.bool, device=DEV)
        sees[:, first:] = torch.tensor(above, device=DEV) | torch.eye(count, dtype=torch.bool, device=DEV)
        if case["window"]:
            sees &= far < case["window"]
        pages = x["table"][b, :-(-n // page)].long()
        for h in range(case["Hkv"]):
            part = {k: (v[pages][:, :, h] if v.dim() == 4 else v) for k, v in c.items()}
            k = _rows64(part, "k", case["fp4"]).flatten(0, 1)[:n]
            v = _rows64(part, "v", case["fp4"]).flatten(0, 1)[:n]
            for g in range(h * G, (h + 1) * G):
                s = x["q"][b, :count, g].double() @ k.T * x["scale"]
                if case["cap"]:
                    s = case["cap"] * torch.tanh(s / case["cap"])
                if case["bias"]:
                    s = s - x["slopes"][g].double() * far
                s = torch.where(sees, s, -math.inf)
                lse[b, :count, g] = torch.logsumexp(s, 1)
                out[b, :count, g] = torch.softmax(s, 1) @ v
    return out, lse


def _accept_exact(case, x, c):
    page = case["page"]
    n, counts, paths = _paths(case)
    table = x["table"].tolist()
    moves = []
    for b, path in enumerate(paths):
        first = n[b] - counts[b]
        at = [table[b][i // page] * page + i % page if n[b] else 0 for i in range(first, n[b])]
        moves += [(at[j], at[k]) for k, j in enumerate(path)]
    src, dst = (_ints([m[i] for m in moves], torch.int64) for i in range(2))
    got = [torch.tensor([n[b] - counts[b] + len(p) for b, p in enumerate(paths)], dtype=torch.int32, device=DEV)]
    for name in ("k", "v"):
        y = c[name].clone()
        y[dst // page, dst % page] = c[name][src // page, src % page]
        got.append(y.double())
    return tuple(got)


def _fork_exact(case, x, c):
    page = case["page"]
    n, parents = _fork(case)
    table, fresh = x["table"].tolist(), x["fresh"].tolist()
    rows, moves = [], []
    for p, f in zip(parents, fresh):
        r = list(table[p])
        if f >= 0:
            i = n[p] // page
            moves += [(r[i] * page + j, f * page + j) for j in range(n[p] % page)]
            r[i] = f
        rows.append(r)
    got = [_ints(rows), _ints([n[p] for p in parents])]
    src, dst = (_ints([m[i] for m in moves], torch.int64) for i in range(2))
    for name in ("k", "v"):
        if case["fp4"]:
            part = {k: (v[src // page, src % page] if v.dim() == 4 else v) for k, v in c.items()}
            got.append(_rows64(part, name, True))
        else:
            y = c[name].clone()
            y[dst // page, dst % page] = c[name][src // page, src % page]
            got.append(y.double())
    return tuple(got)


def _copy_exact(case, x, c):
    got = []
    for name in ("k", "v"):
        y = c[name].clone()
        for i in range(0, case["n"], 512):
            y[x["dst"][i:i + 512].long()] = c[name][x["src"][i:i + 512].long()]
        got.append(y.double())
    return tuple(got)
