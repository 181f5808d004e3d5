"""Performance cases of the decode-time and adapter operators: what is measured.

Three groups of calls stand beside the W4A4 linear layer of this package:

* ``append``  keys and values of new tokens go into a paged cache (bf16, or
  MixFP4 codes and scales), queries and keys rotated to their positions on the
  way.  On a MixFP4 cache the pass also reads the appended rows back as values
  (``mixfp4_kv_gather``, what a chunked prefill does with them).
* ``attend``  attention of one new token per sequence over the paged cache.
* ``lora``    low-rank adapters of many requests at once beside a shared
  projection, forward; with ``train`` the forward and the backward pass
  (gradients of the input and of both adapter matrices).

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
        # One new token of one sequence (8B heads), projections in fp32 as the linear layer returns them: the
        # smallest call, where latency is all.
        dict(name="append_1", op="append", T=1, Hq=32, Hkv=8, D=128, rot=128, inter=False, x32=True, fp4=False,
             page=16, hnd=False, skip=0),
        # A decode batch (70B heads) into a MixFP4 cache.
        dict(name="append_64_fp4", op="append", T=64, Hq=64, Hkv=8, D=128, rot=128, inter=False, x32=True, fp4=True,
             page=16, hnd=False, skip=0),
        # A prefill of odd length into a MixFP4 cache, a few padding tokens without a slot.
        dict(name="append_8111_fp4", op="append", T=8111, Hq=32, Hkv=8, D=128, rot=128, inter=False, x32=True,
             fp4=True, page=64, hnd=False, skip=5),
        # One sequence, a short context: latency.
        dict(name="attend_1x700", op="attend", B=1, longest=700, even=True, Hq=32, Hkv=8, D=128, page=16, window=0,
             fp4=False, hnd=False, mix=1),
        # A decode batch of ragged contexts up to 8192 tokens (8B heads).
        dict(name="attend_64x8192", op="attend", B=64, longest=8192, even=False, Hq=32, Hkv=8, D=128, page=16,
             window=0, fp4=False, hnd=False, mix=2),
        # Two sequences of a very long context (70B heads): the cache's length has to be split.
        dict(name="attend_2x131072", op="attend", B=2, longest=131072, even=True, Hq=64, Hkv=8, D=128, page=64,
             window=0, fp4=False, hnd=True, mix=3),
        # The ragged decode batch on a MixFP4 cache.
        dict(name="attend_64x8192_fp4", op="attend", B=64, longest=8192, even=False, Hq=32, Hkv=8, D=128, page=16,
             window=0, fp4=True, hnd=False, mix=4),
        # Seven query heads to a key head, narrow heads, a sliding window, odd lengths, empty sequences.
        dict(name="attend_33_window", op="attend", B=33, longest=3333, even=False, Hq=14, Hkv=2, D=64, page=32,
             window=1000, fp4=False, hnd=False, mix=5),
        # A decode batch in which every token has an adapter of its own request.
        dict(name="lora_decode_32", op="lora", T=32, S=32, K=4096, N=4096, R=16, L=16, train=False, mix=6),
        # A ragged prefill of a dozen requests through the MLP gate.
        dict(name="lora_prefill_2999", op="lora", T=2999, S=12, K=4096, N=14336, R=32, L=8, train=False, mix=7),
        # A small training step of several adapters at once, uneven lengths.
        dict(name="lora_train_333", op="lora", T=333, S=7, K=1024, N=1040, R=8, L=5, train=True, mix=8),
        # A training step of 4096 tokens on the attention projection, four adapters of rank 64.
        dict(name="lora_train_4096", op="lora", T=4096, S=8, K=4096, N=4096, R=64, L=4, train=True, mix=9),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# (query heads, key heads, head dimension): grouped, multi-head and multi-query forms, wide and odd ones
_HEADS = [(32, 8, 128), (64, 8, 128), (32, 32, 128), (14, 2, 64), (28, 4, 128), (16, 2, 256), (8, 1, 256), (24, 1, 128),
          (12, 4, 96), (16, 16, 80), (40, 8, 128), (9, 3, 64), (6, 6, 48)]


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "attend", "attend", "lora", "lora", "lora"])
    if op == "append":
        Hq, Hkv, D = rng.choice(_HEADS)
        T = _log(rng, 1, 8000)
        while T * (Hq + 2 * Hkv) * D > 8000 * 48 * 128:
            T = max(1, T // 2)
        return dict(op=op, T=T, Hq=Hq, Hkv=Hkv, D=D, rot=rng.choice([D, D, D, D // 2 // 8 * 8, 0]),
                    inter=rng.random() < 0.3, x32=rng.random() < 0.6, fp4=rng.random() < 0.5,
                    page=rng.choice([16, 16, 32, 64, 48, 128]), hnd=rng.random() < 0.4,
                    skip=rng.choice([0, 0, T // 7]))
    if op == "attend":
        Hq, Hkv, D = rng.choice(_HEADS)
        B, longest = _log(rng, 1, 256), _log(rng, 1, 131072)
        while B * longest * Hkv * D > 64 * 8192 * 8 * 128 or B * longest * Hq > 2 * 131072 * 64:
            if rng.random() < 0.5:
                B = max(1, B // 2)
            else:
                longest = max(1, longest * 2 // 3)
        return dict(op=op, B=B, longest=longest, even=rng.random() < 0.3, Hq=Hq, Hkv=Hkv, D=D,
                    page=rng.choice([16, 16, 32, 64, 48, 128]), window=rng.choice([0, 0, 0, _log(rng, 1, 4096)]),
                    fp4=rng.random() < 0.5, hnd=rng.random() < 0.4, mix=rng.randrange(10, 1 << 20))
    train = rng.random() < 0.4
    T, K, N = _log(rng, 1, 4096), _log(rng, 16, 896) * 16, _log(rng, 16, 896) * 16
    R, L = rng.choice([8, 16, 16, 24, 32, 64, 64, 128]), _log(rng, 1, 64)
    while L * R > 1024:
        L //= 2
    while T * (K + N) * (3 if train else 1) * L * R > 4096 * 8192 * 3 * 256 or \
            T * (K + 2 * N) * (3 if train else 1) > 4096 * 12288 * 3:
        T = max(1, T // 2)
    if not train:
        N = max(1, N - rng.choice([0, 0, 1, 6]))
    S = rng.choice([1, min(T, 3), min(T, _log(rng, 1, 64)), T if T <= 256 else min(T, 16)])
    return dict(op=op, T=T, S=S, K=K, N=N, R=R, L=L, train=train, mix=rng.randrange(10, 1 << 20))


def _lengths(case):
    """Tokens in the cache of each sequence, the new one included."""
    B, longest = case["B"], case["longest"]
    if case["even"]:
        return [longest] * B
    rng = random.Random(case["mix"])
    n = [rng.randint(1, longest) for _ in range(B)]
    n[rng.randrange(B)] = longest
    if B >= 16:
        n[rng.randrange(B)] = 0  # a slot of the batch without a request
    return n


def _segments(case):
    """Starts [S + 1] of the requests' tokens and each request's adapter (-1: none)."""
    T, S, L = case["T"], case["S"], case["L"]
    rng = random.Random(case["mix"])
    cuts = list(range(T + 1)) if S == T else [0] + sorted(rng.randint(0, T) for _ in range(S - 1)) + [T]
    return cuts, [rng.randrange(L) if S < 4 or rng.random() < 0.9 else -1 for _ in range(S)]


def work(case):
    if case["op"] == "append":
        T, Hq, Hkv, D = (case[k] for k in ("T", "Hq", "Hkv", "D"))
        x = T * (Hq + 2 * Hkv) * D * (4 if case["x32"] else 2) + T * (16 + 4 * case["rot"])
        kv = T * Hkv * D * 2
        if case["fp4"]:  # written as codes and scales, read again, returned in bf16
            return {"bytes": x + T * Hq * D * 2 + 2 * kv * 9 // 16 + kv * 2, "flops": 0}
        return {"bytes": x + T * Hq * D * 2 + kv * 2, "flops": 0}
    if case["op"] == "attend":
        n = sum(min(k, case["window"]) if case["window"] else k for k in _lengths(case))
        row = case["D"] * 9 / 16 if case["fp4"] else case["D"] * 2
        return {"bytes": n * (case["Hkv"] * row * 2 + 4 / case["page"]) + case["B"] * case["Hq"] * (case["D"] * 4 + 4),
                "flops": 4 * n * case["Hq"] * case["D"]}
    T, K, N, R, L = (case[k] for k in ("T", "K", "N", "R", "L"))
    cuts, ids = _segments(case)
    n = sum(cuts[i + 1] - cuts[i] for i in range(len(ids)) if ids[i] >= 0)
    used = len({ids[i] for i in range(len(ids)) if ids[i] >= 0 and cuts[i + 1] > cuts[i]})
    b = 2 * n * K + 8 * T * N + used * 2 * R * (K + N) + 4 * n * R
    f = 2 * n * R * (K + N)
    if case["train"]:
        # x and dy once, the base of dx read and dx written, both gradients written
        b += 2 * n * (K + N) + 8 * T * K + used * 2 * R * (K + N) + 4 * n * R + L * 4 * R * (K + N)
        f *= 3
    return {"bytes": b, "flops": f}


# --------------------------------------------------------------------- inputs


def _gen(seed, which):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + which)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_E1M2 = (0.0, 1.0, 2.0, 3.0, 4.0, 5.0, 6.0, 7.0)


@functools.lru_cache(maxsize=None)
def _t(v):
    """A constant (number or tuple) on the GPU, made once."""
    return torch.tensor(v, dtype=torch.float32, device=DEV)


def _payload(m, book):
    """Nearest position in `book`, a tie to the even one, saturating."""
    i = torch.zeros_like(m, dtype=torch.uint8)
    for j in range(1, 8):
        mid = (book[j - 1] + book[j]) / 2
        i += (m >= mid) if j % 2 == 0 else (m > mid)
    return i


def _algorithm1(x, s32):
    """Algorithm 1 on fp32 [..., D] with a given tensor scale: payloads, block scales and E1M2 flags.  The error
    sums of a block are fma chains over its even and odd elements (the fma through 64 bits)."""
    a = (x.abs() / s32).unflatten(-1, (-1, 16))
    B = a.amax(-1)
    got = []
    for div, book in ((6.0, _E2M1), (7.0, _E1M2)):
        s8 = (B / _t(div)).clamp(max=448.0).to(torch.float8_e4m3fn).float()
        p = _payload(torch.where(s8[..., None] > 0, a / s8[..., None], torch.zeros_like(a)), book)
        d = (_t(book)[p.long()] * s8[..., None] - a).unflatten(-1, (8, 2))
        S = torch.zeros_like(d[..., 0, :])
        for i in range(8):
            S = (S.double() + d[..., i, :].double().square()).float()
        got.append((S.sum(-1), p, s8))
    (S2, p2, s2), (S1, p1, s1) = got
    one = ~(S2 < S1)
    return torch.where(one[..., None], p1, p2), torch.where(one, s1, s2), one


def _pack(x, s32):
    """Codes [..., D / 2] and scale bytes [..., D / 16] of fp32 values."""
    codes = torch.empty(*x.shape[:-1], x.shape[-1] // 2, dtype=torch.uint8, device=DEV)
    scales = torch.empty(*x.shape[:-1], x.shape[-1] // 16, dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 26) * x.shape[0] // max(1, x.numel()))
    for i in range(0, x.shape[0], step):
        c = x[i:i + step].float()
        p, s8, one = _algorithm1(c, s32)
        p = p.flatten(-2) | (torch.signbit(c).to(torch.uint8) << 3)
        codes[i:i + step] = p[..., 0::2] | (p[..., 1::2] << 4)
        scales[i:i + step] = s8.to(torch.float8_e4m3fn).view(torch.uint8) | (one.to(torch.uint8) << 7)
    return codes, scales


def _paged(rows, hnd):
    """Rows [pages, page, heads, n] stored in that order or, with hnd, head by head within a page."""
    return rows.transpose(1, 2).contiguous().transpose(1, 2) if hnd else rows.contiguous()


def _cache(case, pages, seed, fill):
    """A cache of `pages` pages: keys with a few strong channels, values without; or empty (zeros)."""
    page, H, D = case["page"], case["Hkv"], case["D"]
    c = {}
    for which, name in ((11, "k"), (12, "v")):
        g = _gen(seed, which)
        if fill:
            x = torch.empty(pages, page, H, D, dtype=torch.bfloat16, device=DEV)
            gain = torch.ones(H, D, device=DEV)
            if name == "k":
                gain[torch.rand(H, D, generator=g, device=DEV) < 0.03] = 6.0
            step = max(1, (1 << 26) // (page * H * D))
            for i in range(0, pages, step):
                x[i:i + step] = _randn(g, *x[i:i + step].shape) * gain
        else:
            x = torch.zeros(pages, page, H, D, dtype=torch.bfloat16, device=DEV)
        if case["fp4"]:
            ts = _t((40.0 / 2688.0 if name == "k" else 8.0 / 2688.0,))
            codes, scales = _pack(x, ts) if fill else (torch.zeros_like(x[..., ::2], dtype=torch.uint8),
                                                      torch.zeros_like(x[..., ::16], dtype=torch.uint8))
            c[name], c[name + "s"], c[name + "t"] = _paged(codes, case["hnd"]), _paged(scales, case["hnd"]), ts
        else:
            c[name] = _paged(x, case["hnd"])
    return c


def _own_cache(c):
    from paper_2605_31035_gb300 import ops
    return ops.KVCache(c["k"], c["v"], c.get("ks"), c.get("vs"), c.get("kt"), c.get("vt"))


_POSITIONS = 16384


def _cos_sin(rot):
    f = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / max(rot, 1))
    a = torch.arange(_POSITIONS, dtype=torch.float64, device=DEV)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _append_inputs(case, seed):
    T, Hq, Hkv, D, page = (case[k] for k in ("T", "Hq", "Hkv", "D", "page"))
    g = _gen(seed, 1)
    x = _randn(g, T, (Hq + 2 * Hkv) * D)  # the fused projection's output
    x = x if case["x32"] else x.to(torch.bfloat16)
    q, k, v = (p.unflatten(1, (-1, D)) for p in x.split([Hq * D, Hkv * D, Hkv * D], dim=1))
    # page 0 is never handed out; a prefill fills pages in turn, its pages are anywhere in the pool
    pages = 2 + -(-T // page)
    order = 1 + torch.randperm(pages - 1, generator=g, device=DEV)
    t = torch.arange(T, device=DEV)
    slots = order[t // page] * page + t % page
    if case["skip"]:
        slots[torch.randperm(T, generator=g, device=DEV)[:case["skip"]]] = -1
    pos = torch.randint(0, _POSITIONS - T, (1,), generator=g, device=DEV) + t
    return dict(q=q, k=k, v=v, slots=slots, pos=pos, cs=_cos_sin(case["rot"]) if case["rot"] else None,
                pages=pages)


def _attend_inputs(case, seed):
    B, page = case["B"], case["page"]
    g = _gen(seed, 2)
    n = _lengths(case)
    need = [-(-k // page) for k in n]
    pool = torch.randperm(sum(need) + 1, generator=g, device=DEV).to(torch.int32)
    ends = torch.tensor(need, device=DEV).cumsum(0)
    i = torch.arange(max(need + [1]), device=DEV)
    at = (ends - torch.tensor(need, device=DEV))[:, None] + i
    table = torch.where(at < ends[:, None], pool[at.clamp(max=pool.numel() - 1)], -1)
    q = (_randn(g, B, case["Hq"], case["D"]) * 1.5).to(torch.bfloat16)
    return dict(q=q, table=table, n=torch.tensor(n, dtype=torch.int32, device=DEV), pages=pool.numel(),
                scale=case["D"] ** -0.5)


def _lora_inputs(case, seed):
    T, K, N, R, L = (case[k] for k in ("T", "K", "N", "R", "L"))
    g = _gen(seed, 3)
    cuts, ids = _segments(case)
    gain = torch.where(torch.rand(K, generator=g, device=DEV) < 0.01, 10.0, 1.0)
    t = dict(x=(_randn(g, T, K) * gain).to(torch.bfloat16), base=_randn(g, T, N),
             a=(_randn(g, L, R, K) * K ** -0.5).to(torch.bfloat16), b=(_randn(g, L, N, R) * 0.05).to(torch.bfloat16),
             scaling=torch.rand(L, generator=g, device=DEV) + 0.5,
             starts=torch.tensor(cuts, dtype=torch.int32, device=DEV),
             ids=torch.tensor(ids, dtype=torch.int32, device=DEV))
    if case["train"]:
        t.update(dy=(_randn(g, T, N) * 1e-3).to(torch.bfloat16), dx=_randn(g, T, K) * 1e-3)
    return t


def prepare(case, seed):
    if case["op"] == "append":
        st = _append_inputs(case, seed)
        st["cache"] = _cache(case, st["pages"], seed, fill=False)
    elif case["op"] == "attend":
        st = _attend_inputs(case, seed)
        st["cache"] = _cache(case, st["pages"], seed, fill=True)
    else:
        st = _lora_inputs(case, seed)
    st["case"] = case
    if own:  # the handles that a user's program keeps
        from paper_2605_31035_gb300 import ops
        if "cache" in st:
            st["kv"] = _own_cache(st["cache"])
        else:
            st["adapters"] = ops.Adapters(st["a"], st["b"], st["scaling"])
    return st


# ------------------------------------------------------------------------ run


def run(st):
    case = st["case"]
    if own:
        return _run_own(case, st)
    return {"append": _append_plain, "attend": _attend_plain, "lora": _lora_plain}[case["op"]](case, st)


def _run_own(case, st):
    from paper_2605_31035_gb300 import ops
    if case["op"] == "append":
        q = ops.mixfp4_kv_append(st["k"], st["v"], st["kv"], st["slots"], q=st["q"], positions=st["pos"],
                                 cos_sin=st["cs"], interleaved=case["inter"])
        if case["fp4"]:
            return (q, *ops.mixfp4_kv_gather(st["kv"], st["slots"]))
        return q, st["cache"]["k"], st["cache"]["v"]
    if case["op"] == "attend":
        return ops.mixfp4_paged_attention(st["q"], st["kv"], st["table"], st["n"], scale=st["scale"],
                                          window=case["window"], return_lse=True)
    y, u = ops.mixfp4_lora(st["x"], st["adapters"], st["starts"], st["ids"], base=st["base"])
    if not case["train"]:
        return y
    dx, da, db = ops.mixfp4_lora_backward(st["dy"], st["x"], u, st["adapters"], st["starts"], st["ids"],
                                          base=st["dx"])
    return y, dx, da, db


def _rotated(x, cs, rot, inter):
    """The first `rot` dimensions turned by the tokens' angles, pairs (i, i + rot / 2) or (2i, 2i + 1)."""
    if not rot:
        return x
    c, s = cs[:, None, :rot // 2], cs[:, None, rot // 2:]
    r, rest = x[..., :rot], x[..., rot:]
    if inter:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([r, rest], -1)


def _append_plain(case, st):
    c, slots, page = st["cache"], st["slots"], case["page"]
    cs = st["cs"][st["pos"]] if case["rot"] else None
    q = _rotated(st["q"].float(), cs, case["rot"], case["inter"]).to(torch.bfloat16)
    k, v = _rotated(st["k"].float(), cs, case["rot"], case["inter"]), st["v"].float()
    has = (slots >= 0)[:, None, None]
    if case["fp4"]:
        got = []
        for x, ts in ((k, c["kt"]), (v, c["vt"])):
            p, s8, one = _algorithm1(x, ts)
            p = p.long()
            m = torch.where(one[..., None], _t(_E1M2)[p], _t(_E2M1)[p]) * s8[..., None] * ts
            m = torch.where(torch.signbit(x), -m.flatten(-2), m.flatten(-2))
            got.append(torch.where(has, m, torch.zeros_like(m)).to(torch.bfloat16))
        return q, got[0], got[1]
    at = slots.clamp(min=0)
    for x, y in ((k, c["k"]), (v, c["v"])):  # a token without a slot gives slot 0, which nobody owns, its own value
        y[at // page, at % page] = torch.where(has, x.to(torch.bfloat16), y[at // page, at % page])
    return q, c["k"], c["v"]


def _values(c, name, pages, fp4):
    """The cache's rows of these pages in fp32."""
    if not fp4:
        return c[name][pages].float()
    codes, scales = c[name][pages], c[name + "s"][pages]
    book = _t(_E2M1 + tuple(-x for x in _E2M1) + _E1M2 + tuple(-x for x in _E1M2))
    kind = (scales >> 7)[..., None] * 16
    nib = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).unflatten(-1, (-1, 16)) + kind
    s8 = (scales & 127).view(torch.float8_e4m3fn).float() * c[name + "t"]
    return (book[nib.int()] * s8[..., None]).flatten(-2)


def _attend_plain(case, st):
    B, Hq, Hkv, D = case["B"], case["Hq"], case["Hkv"], case["D"]
    pages = st["table"].clamp(min=0).long()
    k = _values(st["cache"], "k", pages, case["fp4"]).flatten(1, 2).transpose(1, 2)  # [B, Hkv, L, D]
    v = _values(st["cache"], "v", pages, case["fp4"]).flatten(1, 2).transpose(1, 2)
    q = st["q"].float().view(B, Hkv, Hq // Hkv, D)
    pos = torch.arange(k.shape[2], device=DEV)
    n = st["n"][:, None]
    seen = pos < n
    if case["window"]:
        seen &= pos >= n - case["window"]
    s = torch.matmul(q, k.transpose(2, 3)) * st["scale"]
    s = torch.where(seen[:, None, None], s, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -math.inf, m, torch.zeros_like(m)))
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(z > 0, z, torch.ones_like(z))
    return o.reshape(B, Hq, D).to(torch.bfloat16), (m + torch.log(z)).reshape(B, Hq)


def _owners(st, T, dtype=torch.float32):
    """[T, L, 1]: one where the token's request has that adapter."""
    n = (st["starts"][1:] - st["starts"][:-1]).long()
    ids = torch.repeat_interleave(st["ids"], n, output_size=T)
    return (ids[:, None] == torch.arange(st["a"].shape[0], device=DEV)).to(dtype)[..., None]


def _lora_plain(case, st):
    T, N = case["T"], case["N"]
    L, R, K = st["a"].shape
    x, a, b = st["x"].float(), st["a"].float().reshape(L * R, K), st["b"].float().transpose(1, 2).reshape(L * R, N)
    mine = _owners(st, T)
    scaled = mine * st["scaling"][:, None]
    u = (x @ a.T).view(T, L, R)
    us = (u * scaled).view(T, L * R)
    y = st["base"] + us @ b
    if not case["train"]:
        return y
    dy = st["dy"].float()
    vs = ((dy @ b.T).view(T, L, R) * scaled).view(T, L * R)
    dx = st["dx"] + vs @ a
    return y, dx, (vs.T @ x).view(L, R, K), (dy.T @ us).view(N, L, R).transpose(0, 1).contiguous()


# ---------------------------------------------------------------------- exact


def exact(case, seed):
    return {"append": _append_exact, "attend": _attend_exact, "lora": _lora_exact}[case["op"]](case, seed)


def _turn(x, pos, rot, inter, cs):
    """The rotation as a product of complex numbers, in 64 bits, with the table's angles."""
    x = x.double()
    if not rot:
        return x
    w = torch.complex(*cs[pos].double().chunk(2, 1))[:, None]
    r = x[..., :rot]
    z = torch.view_as_complex(r.unflatten(-1, (-1, 2))) if inter else torch.complex(*r.chunk(2, -1))
    z = torch.view_as_real(z * w)
    return torch.cat([z.flatten(-2) if inter else torch.cat([z[..., 0], z[..., 1]], -1), x[..., rot:]], -1)


def _nearest(x, ts):
    """The MixFP4 values of 64-bit numbers: the fp32 steps of Algorithm 1 whose roundings define the codes (quotient
    by the tensor scale, block scale, quotient by the block scale), all else in 64 bits."""
    mag = x.abs().float()
    a = (mag / ts).reshape(-1, 16)
    top = a.max(1).values
    best = None
    for book in (_E2M1, _E1M2):
        w = (top / book[-1]).clamp(max=448.0).to(torch.float8_e4m3fn).float()
        m = torch.nan_to_num(a / w[:, None], nan=0.0, posinf=0.0)
        values = torch.tensor(book, dtype=torch.float64, device=DEV)
        hi = torch.bucketize(m.double(), values).clamp(1, 7)
        up, down = values[hi] - m, m - values[hi - 1]
        q = values[torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)] * w[:, None].double()
        e = (q - a).square().sum(1, keepdim=True)
        best = (e, q) if best is None else (None, torch.where(best[0] < e, best[1], q))
    return torch.where(torch.signbit(x), -1.0, 1.0) * best[1].reshape(x.shape) * ts.double()


def _append_exact(case, seed):
    t = _append_inputs(case, seed)
    c = _cache(case, t["pages"], seed, fill=False)
    turn = (t["pos"], case["rot"], case["inter"], t["cs"])
    q, k, v = _turn(t["q"], *turn), _turn(t["k"], *turn), t["v"].double()
    has = t["slots"] >= 0
    if case["fp4"]:
        return (q, *(torch.where(has[:, None, None], _nearest(x, ts), 0.0) for x, ts in ((k, c["kt"]), (v, c["vt"]))))
    out = [q]
    at = t["slots"][has]
    for x, y in ((k, c["k"]), (v, c["v"])):
        y = y.double()
        y[at // case["page"], at % case["page"]] = x[has]
        out.append(y)
    return tuple(out)


def _attend_exact(case, seed):
    t = _attend_inputs(case, seed)
    c = _cache(case, t["pages"], seed, fill=True)
    G, D = case["Hq"] // case["Hkv"], case["D"]
    out = torch.zeros(case["B"], case["Hq"], D, dtype=torch.float64, device=DEV)
    lse = torch.full((case["B"], case["Hq"]), -math.inf, dtype=torch.float64, device=DEV)
    for i, n in enumerate(_lengths(case)):
        lo = max(0, n - case["window"]) if case["window"] else 0
        if n == 0:
            continue
        pages = t["table"][i, :-(-n // case["page"])].long()
        for h in range(case["Hkv"]):
            part = {x: (y[pages][:, :, h:h + 1] if y.dim() == 4 else y) for x, y in c.items()}
            whole = torch.arange(pages.numel(), device=DEV)
            k = _rows64(part, "k", whole, case["fp4"])[lo:n]
            v = _rows64(part, "v", whole, case["fp4"])[lo:n]
            s = t["q"][i, h * G:(h + 1) * G].double() @ k.T * t["scale"]
            lse[i, h * G:(h + 1) * G] = torch.logsumexp(s, 1)
            out[i, h * G:(h + 1) * G] = torch.softmax(s, 1) @ v
    return out, lse


def _rows64(c, name, pages, fp4):
    """One head's rows in 64 bits (a MixFP4 value is sign * codebook value * block scale * tensor scale)."""
    x = c[name].reshape(-1, c[name].shape[-1])
    if not fp4:
        return x.double()
    sc = c[name + "s"].reshape(-1, c[name + "s"].shape[-1])
    e, f = ((sc & 127) >> 3).double(), (sc & 7).double()
    s8 = torch.where(e > 0, torch.exp2(e - 7) * (1 + f / 8), f * 2.0 ** -9).repeat_interleave(16, 1)
    one = (sc >> 7).repeat_interleave(16, 1).bool()
    nib = torch.stack([x & 15, x >> 4], 2).reshape(x.shape[0], -1)
    p = (nib & 7).double()
    e2, m2 = torch.floor(p / 2), p % 2
    mag = torch.where(one, p, torch.where(e2 > 0, torch.exp2(e2 - 1) * (1 + m2 / 2), m2 / 2))
    return torch.where(nib > 7, -mag, mag) * s8 * c[name + "t"].double()


def _lora_exact(case, seed):
    t = _lora_inputs(case, seed)
    cuts, ids = _segments(case)
    y = t["base"].double()
    dx = t["dx"].double() if case["train"] else None
    da, db = torch.zeros_like(t["a"], dtype=torch.float64), torch.zeros_like(t["b"], dtype=torch.float64)
    for i, j in enumerate(ids):
        rows = slice(cuts[i], cuts[i + 1])
        if j < 0:
            continue
        x, a, b, s = t["x"][rows].double(), t["a"][j].double(), t["b"][j].double(), t["scaling"][j].double()
        u = x @ a.T
        y[rows] += s * (u @ b.T)
        if case["train"]:
            dy = t["dy"][rows].double()
            w = s * (dy @ b)
            dx[rows] += w @ a
            da[j] += w.T @ x
            db[j] += s * (dy.T @ u)
    return (y, dx, da, db) if case["train"] else y
