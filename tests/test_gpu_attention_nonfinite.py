"""Infinities and NaN in what mixfp4_paged_attention sees: the results are those
of the definition in 64 bits, NaN for NaN and sign for sign.

A score of NaN makes a head's result and log-sum-exp NaN; one of +inf the result NaN and
the log-sum-exp +inf; one of -inf has weight 0.  An infinite element of V
makes its dimension infinite, two of different signs NaN.  Only a sequence that
sees nothing has a log-sum-exp of -inf here.  What stays finite keeps the bounds of
test_gpu_paged_attention.py; every weight here is above 2^-100 of the largest."""
import math
import os
import sys

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)
import test_gpu_paged_attention as t  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
D, Hkv, Hq = 128, 2, 8

# lengths and the table's tokens (0: as many as the longest): a cluster of 8, 4 or 2 CTAs to a row, a CTA to a row,
# whole rows in shares, and rows cut over many shares
WAYS = {
    "cluster of 8": ([300, 7, 0], 0),
    "cluster of 4": ([300, 7, 0, 100] * 10, 0),
    "cluster of 2": ([300, 7, 0, 100] * 25, 0),
    "CTA": ([200, 7, 0, 100] * 80, 0),
    "shares": ([90, 7, 0, 60] * 100, 6000),
    "cut rows": ([20000, 7, 0], 0),
}


def attend(way, fp4, spoil):
    """`spoil(q, cache, slots of sequence 0)` puts in what is not finite; then result and definition are compared."""
    lengths, wide = WAYS[way]
    cache, table, _, _ = t.build(fp4, lengths, Hkv, D, 16, seed=5)
    table = table[:, :-1]
    if wide:
        full = torch.full((len(lengths), wide // 16), -1, dtype=torch.int32, device=DEV)
        full[:, :table.shape[1]] = table
        table = full
    q = t.randn(len(lengths), Hq, D, seed=6).to(torch.bfloat16)
    slots = []
    for b, n in enumerate(lengths):
        j = torch.arange(n, device=DEV)
        slots.append(table[b, j // 16].long() * 16 + j % 16)
    spoil(q, cache, slots[0])
    out, lse = t.ops().mixfp4_paged_attention(q, cache, table, torch.tensor(lengths, dtype=torch.int32, device=DEV),
                                              return_lse=True)
    k, v = (x.double() for x in t.ops().mixfp4_kv_gather(cache, torch.cat(slots), torch.float32))
    t.check(out[1:], lse[1:], q[1:], lengths[1:], k[lengths[0]:], v[lengths[0]:], D ** -0.5, 0, fp4)
    k, v = k[:lengths[0]], v[:lengths[0]]
    s = torch.einsum("hgd,nhd->hgn", q[0].double().view(Hkv, Hq // Hkv, D), k) * D ** -0.5
    p = s.softmax(-1)
    ref = torch.einsum("hgn,nhd->hgd", p, v).reshape(Hq, D)
    mag = torch.einsum("hgn,nhd->hgd", p, v.abs()).reshape(Hq, D)
    ls = torch.logsumexp(s, -1).reshape(Hq)
    for got, want in ((out[0], ref), (lse[0], ls)):
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(got.isposinf(), want.isposinf()) and torch.equal(got.isneginf(), want.isneginf())
    fine = ref.isfinite()
    t.within(out[0][fine], ref[fine], (2.0 ** -10.5 if fp4 else 2.0 ** -13) * mag[fine])
    fine = ls.isfinite()
    top = torch.where(s.isfinite(), s, 0.0).abs().amax(-1).reshape(Hq)
    assert torch.all((lse[0].double() - ls).abs()[fine] <= 2.0 ** -17 * (1 + top)[fine])
    return ref, ls


def put(cache, slot, name, head, d, value):
    getattr(cache, name)[slot // 16, slot % 16, head, d] = value


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("way", WAYS)
def test_queries(way, fp4):
    def spoil(q, cache, slots):
        q[0, 1, 5] = math.nan
        q[0, 3, 9] = math.inf
        q[0, 6, 70] = -math.inf
    ref, ls = attend(way, fp4, spoil)
    assert ls[1].isnan() and not ls[3].isfinite() and not ls[6].isfinite() and ls[[0, 2, 4, 5, 7]].isfinite().all()


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_keys(way, value):
    def spoil(q, cache, slots):
        put(cache, slots[len(slots) // 2], "k", 0, 17, value)
        put(cache, slots[-1], "k", 0, 17, value)
    ref, ls = attend(way, False, spoil)
    assert ls[4:].isfinite().all() and (value != value) == bool(ls[:4].isnan().all())


@pytest.mark.parametrize("way", WAYS)
def test_an_infinite_and_a_nan_score(way):
    def spoil(q, cache, slots):
        q[0, :4] = 1.0
        put(cache, slots[0], "k", 0, 3, math.inf)
        put(cache, slots[-1], "k", 0, 3, math.nan)
        q[0, 4:] = 1.0
        put(cache, slots[0], "k", 1, 3, math.inf)
    ref, ls = attend(way, False, spoil)
    assert ls[:4].isnan().all() and ls[4:].isposinf().all() and ref.isnan().all()


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("name", ["k", "v"])
def test_scale_bytes(way, name):
    """A MixFP4 row whose scale byte is NaN."""
    def spoil(q, cache, slots):
        put(cache, slots[len(slots) // 3], name + "_scales", 1, 2, 0x7F)
    attend(way, True, spoil)


@pytest.mark.parametrize("way", WAYS)
def test_values(way):
    def spoil(q, cache, slots):
        j = len(slots) // 2
        put(cache, slots[0], "v", 0, 0, math.inf)
        put(cache, slots[j], "v", 0, 64, -math.inf)
        put(cache, slots[-1], "v", 1, 127, math.inf)
        put(cache, slots[j], "v", 1, 3, math.inf)
        put(cache, slots[j + 1], "v", 1, 3, -math.inf)
        put(cache, slots[1], "v", 1, 50, math.nan)
    ref, ls = attend(way, False, spoil)
    assert ls.isfinite().all() and ref[:4, 0].isposinf().all() and ref[:4, 64].isneginf().all()
    assert ref[4:, 127].isposinf().all() and ref[4:, [3, 50]].isnan().all() and int((~ref.isfinite()).sum()) == 4 * 5
