"""The paged key-value cache on the GPU: appending with the position rotation
against the definition (bf16 rows bit for bit against the fp32 formula, MixFP4
rows bit for bit against the oracle's Algorithm 1 on the fp32 rows), and
reading rows back."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def ops():
    from paper_2605_31035_gb300 import ops as o
    return o


def rotated(x, cs, inter):
    """The rotation of fp32 rows [T, H, D], products and sums rounded one by one."""
    rot = cs.shape[1]
    c, s = cs[:, None, :rot // 2], cs[:, None, rot // 2:]
    y = x.clone()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    p, q = a * c - b * s, b * c + a * s
    if inter:
        y[..., 0:rot:2], y[..., 1:rot:2] = p, q
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = p, q
    return y


def angles(rows, rot, seed=3):
    a = torch.rand(rows, rot // 2, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * 6.283
    return torch.cat([a.cos(), a.sin()], 1).float().to(DEV)


def randn(*shape, seed=1):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV)


def make_cache(fp4, pages, page, H, D, layout="nhd", poison=True):
    """A cache full of values that no test expects; layouts: token by token, head by head, k and v in one buffer."""
    def one(n, dtype, count=2):
        shape = {"nhd": (count, pages, page, H, n), "hnd": (count, pages, H, page, n), "kv": (pages, count, page, H, n)}
        t = torch.full(shape[layout], 0x7E if dtype is torch.uint8 else float("nan"), dtype=dtype, device=DEV)
        if layout == "hnd":
            return t[0].transpose(1, 2), t[1].transpose(1, 2)
        return (t[:, 0], t[:, 1]) if layout == "kv" else (t[0], t[1])
    if not fp4:
        return ops().KVCache(*one(D, torch.bfloat16))
    ts = [torch.tensor([v], dtype=torch.float32, device=DEV) for v in (7.0 / 2688, 5.0 / 2688)]
    return ops().KVCache(*one(D // 2, torch.uint8), *one(D // 16, torch.uint8), *ts)


CASES = [
    # fp4, T, Hq, Hkv, D, rot, inter, fp32 input, page, layout
    (False, 1, 32, 8, 128, 128, False, True, 16, "nhd"),
    (False, 37, 8, 2, 128, 64, False, False, 16, "hnd"),
    (False, 5, 4, 4, 64, 0, False, True, 1, "nhd"),
    (False, 19, 6, 6, 48, 24, False, True, 48, "kv"),
    (False, 19, 6, 3, 80, 40, True, False, 3, "nhd"),
    (False, 9, 3, 1, 256, 254, False, True, 16, "kv"),
    (False, 9, 3, 1, 16, 16, True, True, 16, "nhd"),
    (True, 1, 32, 8, 128, 128, False, True, 16, "nhd"),
    (True, 37, 8, 2, 128, 64, False, False, 16, "hnd"),
    (True, 21, 4, 2, 64, 64, True, True, 7, "nhd"),
    (True, 19, 6, 6, 48, 24, False, True, 48, "hnd"),
    (True, 11, 2, 2, 80, 0, False, False, 16, "kv"),
    (True, 9, 8, 1, 256, 96, False, True, 64, "nhd"),
    (True, 300, 4, 4, 96, 96, False, True, 32, "nhd"),
]


@pytest.mark.parametrize("fp4,T,Hq,Hkv,D,rot,inter,f32,page,layout", CASES)
def test_append_matches_the_definition(oracle, fp4, T, Hq, Hkv, D, rot, inter, f32, page, layout):
    o = ops()
    pages = -(-T // page) + 3
    cache = make_cache(fp4, pages, page, Hkv, D, layout)
    # a fused projection's rows with padding behind them
    x = randn(T, (Hq + 2 * Hkv) * D + 32, seed=T + D)
    x = x if f32 else x.to(torch.bfloat16)
    q, k, v = (p.unflatten(1, (-1, D)) for p in x[:, :-32].split([Hq * D, Hkv * D, Hkv * D], 1))
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(T))[:T].to(DEV)
    if T > 4:
        slots[1], slots[3] = -1, pages * page  # kept nowhere
    cs = angles(50 + T, rot) if rot else None
    pos = torch.randint(0, 50 + T, (T,), generator=torch.Generator().manual_seed(T + 1)).to(DEV)
    before = [t.clone() for t in (cache.k, cache.v)]
    qo = o.mixfp4_kv_append(k, v, cache, slots, q=q, positions=pos, cos_sin=cs, interleaved=inter)
    qr, kr = (rotated(t.float(), cs[pos], inter) if rot else t.float() for t in (q, k))
    assert torch.equal(qo, qr.to(torch.bfloat16))
    kept = (slots >= 0) & (slots < pages * page)
    at, off = slots[kept] // page, slots[kept] % page
    untouched = torch.ones(pages, page, dtype=torch.bool, device=DEV)
    untouched[at, off] = False
    for ref, t, sc, ts, old in ((kr, cache.k, cache.k_scales, cache.k_ts, before[0]),
                                (v.float(), cache.v, cache.v_scales, cache.v_ts, before[1])):
        if fp4:
            codes, scales, _ = oracle.quantize_f32(ref[kept].reshape(-1, D).cpu().numpy(), 0, ts.item())
            assert np.array_equal(t[at, off].reshape(-1, D // 2).cpu().numpy(), codes)
            assert np.array_equal(sc[at, off].reshape(-1, D // 16).cpu().numpy(), scales)
            assert torch.all(t[untouched] == 0x7E) and torch.all(sc[untouched] == 0x7E)
        else:
            assert torch.equal(t[at, off], ref[kept].to(torch.bfloat16))
            assert torch.all(t[untouched].isnan())


@pytest.mark.parametrize("mode", [1, 2, 3])
def test_append_modes(oracle, mode):
    T, H, D = 33, 2, 128
    cache = make_cache(True, 3, 16, H, D)
    k, v = randn(T, H, D, seed=mode), randn(T, H, D, seed=mode + 9) * 3.0  # past the scale's range: saturating
    slots = torch.arange(T, device=DEV)
    ops().mixfp4_kv_append(k, v, cache, slots, mode=mode)
    for x, t, sc, ts in ((k, cache.k, cache.k_scales, cache.k_ts), (v, cache.v, cache.v_scales, cache.v_ts)):
        codes, scales, _ = oracle.quantize_f32(x.reshape(-1, D).cpu().numpy(), mode, ts.item())
        assert np.array_equal(t.reshape(-1, D // 2)[:T * H].cpu().numpy(), codes)
        assert np.array_equal(sc.reshape(-1, D // 16)[:T * H].cpu().numpy(), scales)


def test_appended_rows_equal_the_quantizers():
    """Unrotated bf16 rows are stored as mixfp4_quantize stores them."""
    o = ops()
    T, H, D = 64, 4, 128
    cache = make_cache(True, 4, 16, H, D)
    x = randn(T, H, D, seed=4).to(torch.bfloat16)
    o.mixfp4_kv_append(x, x, cache, torch.arange(T, device=DEV))
    q = o.mixfp4_quantize(x.reshape(T * H, D), tensor_scale=cache.k_ts)
    assert torch.equal(cache.k.reshape(T * H, -1), q.codes) and torch.equal(cache.k_scales.reshape(T * H, -1), q.scales)


def test_position_outside_the_table_keeps_nothing():
    cache = make_cache(False, 1, 16, 2, 64)
    k = randn(3, 2, 64)
    cs = angles(10, 64)
    pos = torch.tensor([-1, 10, 9], device=DEV)
    q = ops().mixfp4_kv_append(k, k, cache, torch.tensor([0, 1, 2], device=DEV), q=k, positions=pos, cos_sin=cs)
    assert q[:2].isnan().all() and not q[2].isnan().any()
    assert cache.k[0, :2].isnan().all() and cache.v[0, :2].isnan().all() and not cache.k[0, 2].isnan().any()


def test_no_tokens_and_no_queries():
    cache = make_cache(False, 1, 16, 2, 64)
    e = torch.empty(0, 2, 64, device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    assert ops().mixfp4_kv_append(e, e, cache, none, q=e).shape == (0, 2, 64)
    assert ops().mixfp4_kv_append(randn(1, 2, 64), randn(1, 2, 64), cache, torch.zeros(1, dtype=torch.int64, device=DEV)) is None
    assert [t.shape[0] for t in ops().mixfp4_kv_gather(cache, none)] == [0, 0]


@pytest.mark.parametrize("fp4,D,page,layout", [(False, 128, 16, "nhd"), (False, 48, 5, "hnd"), (True, 128, 16, "hnd"),
                                               (True, 80, 3, "kv"), (True, 256, 16, "nhd")])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gather(fp4, D, page, layout, dtype):
    o = ops()
    T, H = 29, 3
    cache = make_cache(fp4, 12, page, H, D, layout)
    k, v = randn(T, H, D, seed=7), randn(T, H, D, seed=8)
    slots = torch.randperm(12 * page, generator=torch.Generator().manual_seed(1))[:T].to(DEV)
    o.mixfp4_kv_append(k, v, cache, slots)
    asked = torch.cat([slots.flip(0), torch.tensor([-1, 12 * page], device=DEV), slots[:1]])
    got = o.mixfp4_kv_gather(cache, asked, dtype)
    for x, y, ts in ((k, got[0], cache.k_ts), (v, got[1], cache.v_ts)):
        if fp4:
            ref = _values(x, ts)
        else:
            ref = x.to(torch.bfloat16).float()
        ref = torch.cat([ref.flip(0), torch.zeros(2, H, D, device=DEV), ref[:1]])
        assert torch.equal(y, ref.to(dtype))


def _values(x, ts):
    """mixfp4_dequantize of the oracle's codes."""
    import oracle
    codes, scales, _ = oracle.quantize_f32(x.reshape(-1, x.shape[-1]).cpu().numpy(), 0, ts.item())
    q = ops().QTensor(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), ts)
    return ops().mixfp4_dequantize(q).reshape(x.shape)


def test_rows_beyond_32_bit_offsets():
    """A cache whose last pages lie more than 2^32 elements in: 68 GB of keys and values in one buffer of which only
    the first and last pages are touched."""
    o = ops()
    page, H, D = 64, 8, 128
    pages = (1 << 32) // (2 * page * H * D) + 2  # k and v of a page side by side
    buf = torch.empty(pages, 2, page, H, D, dtype=torch.bfloat16, device=DEV)
    cache = o.KVCache(buf[:, 0], buf[:, 1])
    T = 70
    k, v = randn(T, H, D, seed=1), randn(T, H, D, seed=2)
    slots = torch.cat([torch.arange(6), torch.arange(pages * page - 64, pages * page)]).to(DEV)
    o.mixfp4_kv_append(k, v, cache, slots)
    gk, gv = o.mixfp4_kv_gather(cache, slots)
    assert torch.equal(gk, k.to(torch.bfloat16)) and torch.equal(gv, v.to(torch.bfloat16))
    assert torch.equal(buf[-1, 0, 7], k[13].to(torch.bfloat16))
    q = randn(2, 16, D, seed=3).to(torch.bfloat16)
    table = torch.tensor([[pages - 1, 0], [0, pages - 1]], dtype=torch.int32, device=DEV)
    out = o.mixfp4_paged_attention(q, cache, table, torch.tensor([70, 3], dtype=torch.int32, device=DEV))
    for i, rows in ((0, torch.cat([gk[6:], gk[:6]])), (1, gk[:3])):
        val = torch.cat([gv[6:], gv[:6]]) if i == 0 else gv[:3]
        s = torch.einsum("hgd,nhd->hgn", q[i].double().view(H, 2, D), rows.double()) * D ** -0.5
        ref = torch.einsum("hgn,nhd->hgd", s.softmax(-1), val.double()).reshape(16, D)
        mag = torch.einsum("hgn,nhd->hgd", s.softmax(-1), val.double().abs()).reshape(16, D)
        # the bf16 rounding of a value within 2^-13 of the sum of magnitudes
        lo, hi = (t.float().to(torch.bfloat16) for t in (ref - 2.0 ** -13 * mag, ref + 2.0 ** -13 * mag))
        assert torch.all((lo <= out[i]) & (out[i] <= hi))


def test_on_another_stream():
    o = ops()
    cache = make_cache(True, 4, 16, 2, 128)
    k = randn(64, 2, 128)
    slots = torch.arange(64, device=DEV)
    ref = o.mixfp4_kv_append(k, k, cache, slots, q=k)
    rk, _ = o.mixfp4_kv_gather(cache, slots)
    cache.k.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = o.mixfp4_kv_append(k, k, cache, slots, q=k, stream=side)
    gk, _ = o.mixfp4_kv_gather(cache, slots, stream=side)
    side.synchronize()
    assert torch.equal(got, ref) and torch.equal(gk, rk)


def test_refusals():
    o = ops()
    cache = make_cache(False, 2, 16, 2, 64)
    k, slots = randn(4, 2, 64), torch.arange(4, device=DEV)
    for bad in (dict(k=k.double()), dict(k=k.to(torch.bfloat16)), dict(v=k[:, :1]), dict(v=k[:3]), dict(slots=slots.int()),
                dict(slots=slots[:3]), dict(slots=slots.cpu()), dict(q=k.to(torch.bfloat16)), dict(cos_sin=angles(9, 64)),
                dict(cos_sin=angles(9, 66), positions=slots), dict(cos_sin=angles(9, 64).double(), positions=slots),
                dict(q=k, out=torch.empty(4, 2, 64, device=DEV)), dict(cache=None)):
        with pytest.raises(ValueError):
            o.mixfp4_kv_append(**{**dict(k=k, v=k, cache=cache, slots=slots), **bad})
    with pytest.raises(o.MixFP4Error, match="misaligned"):
        o.mixfp4_kv_append(randn(4, 2, 72)[:, :, 4:68], k, cache, slots)
    with pytest.raises(o.MixFP4Error, match="out of range"):
        o.mixfp4_kv_append(k, k, cache, slots, mode=4)
    b = torch.empty(2, 16, 2, 64, dtype=torch.bfloat16, device=DEV)
    u = torch.empty(2, 16, 2, 32, dtype=torch.uint8, device=DEV)
    s = torch.empty(2, 16, 2, 4, dtype=torch.uint8, device=DEV)
    t = torch.ones(1, device=DEV)
    for bad in ((b, b.float()), (b, b[:1]), (b, b.transpose(1, 2)), (b[..., ::2], b[..., ::2]), (b[..., :40], b[..., :40]),
                (b.cpu(), b.cpu()), (b[0], b[0]), (u, u, s, s), (u, u, s, s[:1], t, t), (u, u, s.int(), s, t, t),
                (u, u, s, s, t, t.double()), (b, b, None, None, t, t), (b[:, :0], b[:, :0])):
        with pytest.raises(ValueError):
            o.KVCache(*bad)
    with pytest.raises(ValueError):
        o.mixfp4_kv_gather(cache, slots, torch.float16)
    with pytest.raises(ValueError):
        o.mixfp4_kv_gather(cache, slots, out=(k, k))
    odd = torch.empty(2 * 16 * 2 * 64 + 8, dtype=torch.bfloat16, device=DEV)[8:].view(2, 16, 2, 64)
    with pytest.raises(o.MixFP4Error, match="misaligned"):
        o.mixfp4_kv_gather(o.KVCache(odd, odd), slots)
