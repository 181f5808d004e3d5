"""Low-rank adapters of many requests beside a shared projection, forward and
backward, against the definition in 64 bits and, for the gradients, against
differences of the forward pass.

Bounds: sums of exact products in fp32, as the GEMMs' 1e-5 of the sum of
magnitudes, and one rounding of the result (2^-24 of it) where a base is added."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def ops():
    from paper_2605_31035_gb300 import ops as o
    return o


def randn(*shape, seed=1):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def problem(T, cuts, ids, K, N, R, L, seed=1):
    gain = torch.where(torch.arange(K, device=DEV) % 97 == 5, 20.0, 1.0)
    x = (randn(T, K, seed=seed) * gain).to(torch.bfloat16)
    a = (randn(L, R, K, seed=seed + 1) * K ** -0.5).to(torch.bfloat16)
    b = (randn(L, N, R, seed=seed + 2) * 0.1).to(torch.bfloat16)
    s = torch.linspace(0.5, 2.0, L, device=DEV)
    return x, ops().Adapters(a, b, s), ints(cuts), ints(ids), randn(T, N, seed=seed + 3)


def reference(x, ad, cuts, ids, base):
    """(u, y) and the sums of magnitudes behind them, in 64 bits."""
    u = torch.zeros(x.shape[0], ad.rank, dtype=torch.float64, device=DEV)
    um = torch.zeros_like(u)
    y, ym = base.double().clone(), torch.zeros_like(base, dtype=torch.float64)
    for i, j in enumerate(ids):
        if not 0 <= j < ad.count:
            continue
        r = slice(cuts[i], cuts[i + 1])
        xd, a, b, s = x[r].double(), ad.a[j].double(), ad.b[j].double(), ad.scaling[j].double()
        u[r], um[r] = xd @ a.T, xd.abs() @ a.abs().T
        y[r] += s * (u[r] @ b.T)
        ym[r] = s * (um[r] @ b.abs().T)
    return u, um, y, ym


CASES = [
    # T, cuts, ids, K, N, R, L
    (1, [0, 1], [0], 16, 1, 8, 1),
    (1, [0, 1], [2], 4096, 4096, 16, 3),
    (7, [0, 1, 1, 2, 5, 7], [0, 1, -1, 1, 5], 272, 1000, 8, 2),      # an empty segment, two without an adapter
    (32, list(range(33)), [i % 5 for i in range(32)], 1024, 1040, 24, 5),
    (300, list(range(301)), [i * 7 % 3 for i in range(300)], 256, 96, 8, 3),
    (100, [0, 9, 70, 100], [1, 0, 1], 512, 333, 64, 2),
    (129, [0, 129], [0], 1536, 2048, 128, 1),
    (500, [0, 31, 32, 64, 200, 333, 500], [3, 0, 2, 3, -1, 0], 2064, 528, 40, 4),
    (65, [0, 33, 65], [0, 1], 48, 64, 120, 2),
    (2000, [0, 700, 2000], [1, 0], 4096, 272, 32, 2),
]
TRAIN = [c if c[4] % 16 == 0 else (*c[:4], (c[4] + 15) // 16 * 16, *c[5:]) for c in CASES]


@pytest.mark.parametrize("T,cuts,ids,K,N,R,L", CASES)
@pytest.mark.parametrize("based", [True, False])
def test_forward(T, cuts, ids, K, N, R, L, based):
    o = ops()
    x, ad, st, ii, base = problem(T, cuts, ids, K, N, R, L, seed=T)
    y, u = o.mixfp4_lora(x, ad, st, ii, base=base if based else None)
    ru, rum, ry, rym = reference(x, ad, cuts, ids, base if based else torch.zeros_like(base))
    assert torch.all((u.double() - ru).abs() <= 1e-5 * rum)
    assert torch.all((y.double() - ry).abs() <= 1e-5 * rym + 2.0 ** -24 * ry.abs())
    y2, u2 = o.mixfp4_lora(x, ad, st, ii, base=base if based else None)
    assert torch.equal(y, y2) and torch.equal(u, u2)


@pytest.mark.parametrize("T,cuts,ids,K,N,R,L", TRAIN)
@pytest.mark.parametrize("based", [True, False])
def test_backward(T, cuts, ids, K, N, R, L, based):
    o = ops()
    x, ad, st, ii, _ = problem(T, cuts, ids, K, N, R, L, seed=T)
    dy = (randn(T, N, seed=9) * 1e-3).to(torch.bfloat16)
    base = randn(T, K, seed=10) * 1e-3
    _, u = o.mixfp4_lora(x, ad, st, ii)
    da, db = (torch.full_like(t, float("nan"), dtype=torch.float32) for t in (ad.a, ad.b))
    dx, ga, gb = o.mixfp4_lora_backward(dy, x, u, ad, st, ii, base=base if based else None, da=da, db=db)
    assert ga is da and gb is db
    rdx = base.double().clone() if based else torch.zeros(T, K, dtype=torch.float64, device=DEV)
    mdx = torch.zeros_like(rdx)
    rda, rdb = torch.zeros_like(ad.a, dtype=torch.float64), torch.zeros_like(ad.b, dtype=torch.float64)
    mda, mdb = torch.zeros_like(rda), torch.zeros_like(rdb)
    for i, j in enumerate(ids):
        if not 0 <= j < L:
            continue
        r = slice(cuts[i], cuts[i + 1])
        xd, dyd = x[r].double(), dy[r].double()
        a, b, s = ad.a[j].double(), ad.b[j].double(), ad.scaling[j].double()
        v, vm = s * (dyd @ b), s * (dyd.abs() @ b.abs())
        rdx[r] += v @ a
        mdx[r] += vm @ a.abs()
        rda[j] += v.T @ xd
        mda[j] += vm.T @ xd.abs()
        rdb[j] += s * (dyd.T @ (xd @ a.T))
        mdb[j] += s * (dyd.abs().T @ (xd.abs() @ a.abs().T))
    assert torch.all((dx.double() - rdx).abs() <= 1e-5 * mdx + 2.0 ** -24 * rdx.abs())
    assert torch.all((da.double() - rda).abs() <= 1e-5 * mda)
    assert torch.all((db.double() - rdb).abs() <= 1e-5 * mdb)
    again = o.mixfp4_lora_backward(dy, x, u, ad, st, ii, base=base if based else None)
    assert torch.equal(dx, again[0]) and torch.equal(da, again[1]) and torch.equal(db, again[2])


def short(lengths, ids):
    """(T, cuts, ids) of segments of the lengths, over and over the ids."""
    cuts = [0]
    for n in lengths:
        cuts.append(cuts[-1] + n)
    return cuts[-1], cuts, [ids[i % len(ids)] for i in range(len(lengths))]


SHORT = [
    (*short([1] * 600, [0, 3, -1, 5, 2, 2, 9]), 272, 336, 16, 6),           # more segments than threads of a block
    (*short([i * 5 % 7 % 4 for i in range(301)], [1, 0, 1, 2, -1]), 512, 1040, 40, 3),
    (*short([1] * 9 + [100] + [1] * 10, [0, 0, 1]), 1024, 80, 8, 2),        # a long segment among short ones
    (*short([1] * 40, [1099, 0, 511, 0, 1023, 1024]), 64, 64, 8, 1100),     # many adapters
    (*short([2, 0, 1] * 1400, [0, 1, 2, 3]), 32, 32, 8, 4),                 # many segments
    (*short([1, 2, 3] * 7, [-1, 7]), 256, 64, 128, 4),                      # none has an adapter
]


@pytest.mark.parametrize("T,cuts,ids,K,N,R,L", SHORT)
def test_short_segments_share_adapters(T, cuts, ids, K, N, R, L):
    test_forward(T, cuts, ids, K, N, R, L, True)
    test_backward(T, cuts, ids, K, N, R, L, True)


def test_long_sums_keep_fp32():
    """A contraction of 13504 features and one of 3000 tokens: products are exact and a sum of n terms is cut into
    short chains added in fp32, some sqrt(40) roundings of 2^-24 in all: within 1e-6 of the result's norm."""
    o = ops()
    N, R = 288, 32
    for T, K, cuts in ((187, 13504, list(range(188))), (3000, 512, [0, 3000])):
        ids = [i % 2 for i in range(len(cuts) - 1)]
        x, ad, st, ii, _ = problem(T, cuts, ids, K, N, R, 2)
        dy = (randn(T, N, seed=9) * 1e-3).to(torch.bfloat16)
        y, u = o.mixfp4_lora(x, ad, st, ii)
        _, da, db = o.mixfp4_lora_backward(dy, x, u, ad, st, ii)
        ru, _, ry, _ = reference(x, ad, cuts, ids, torch.zeros(T, N, device=DEV))
        rda, rdb = torch.zeros_like(ad.a, dtype=torch.float64), torch.zeros_like(ad.b, dtype=torch.float64)
        for i, j in enumerate(ids):
            r, s = slice(cuts[i], cuts[i + 1]), ad.scaling[j].double()
            rda[j] += s * (dy[r].double() @ ad.b[j].double()).T @ x[r].double()
            rdb[j] += s * (dy[r].double().T @ ru[r])
        for got, ref in ((u, ru), (y, ry), (da, rda), (db, rdb)):
            assert (got.double() - ref).norm() <= 1e-6 * ref.norm()


def test_gradients_against_differences():
    """y is linear in x, in a and in b, so <dy, y(p + h) - y(p)> = <gradient, h> for any h; within 1e-4 of the sum of
    magnitudes, the differences' own rounding."""
    o = ops()
    T, K, N, R, L = 90, 256, 320, 16, 3
    cuts, ids = [0, 10, 11, 50, 90], [0, 2, 1, 0]
    x, ad, st, ii, _ = problem(T, cuts, ids, K, N, R, L)
    dy = randn(T, N, seed=9).to(torch.bfloat16)
    y, u = o.mixfp4_lora(x, ad, st, ii)
    dx, da, db = o.mixfp4_lora_backward(dy, x, u, ad, st, ii)
    h = [(randn(*t.shape, seed=20) * t.float().std()).to(torch.bfloat16) for t in (x, ad.a, ad.b)]
    moved = [(x + h[0], ad), (x, o.Adapters(ad.a + h[1], ad.b, ad.scaling)), (x, o.Adapters(ad.a, ad.b + h[2], ad.scaling))]
    for (x2, ad2), old, grad in zip(moved, (x, ad.a, ad.b), (dx, da, db)):
        new = x2 if x2 is not x else (ad2.a if ad2.a is not ad.a else ad2.b)
        d = (o.mixfp4_lora(x2, ad2, st, ii)[0].double() - y.double()) * dy.double()
        g = grad.double() * (new.double() - old.double())
        assert abs(float(d.sum() - g.sum())) <= 1e-4 * float(d.abs().sum())


def test_in_place_and_strides():
    o = ops()
    cuts, ids = [0, 3, 20, 40], [1, -1, 0]
    x, ad, st, ii, base = problem(40, cuts, ids, 256, 500, 16, 2)
    ref, u = o.mixfp4_lora(x, ad, st, ii, base=base)
    wide = torch.full((40, 503), 7.0, device=DEV)
    wide[:, 1:501] = base
    xs = torch.zeros(40, 272, dtype=torch.bfloat16, device=DEV)
    xs[:, :256] = x
    y, _ = o.mixfp4_lora(xs[:, :256], ad, st, ii, base=wide[:, 1:501], out=wide[:, 1:501])
    assert torch.equal(y, ref)
    assert torch.all(wide[:, 0] == 7.0) and torch.all(wide[:, 501:] == 7.0)
    assert torch.equal(y[3:20], base[3:20])


def test_rows_that_belong_to_others_do_not_leak():
    """NaN and infinities in another segment's x and dy stay there."""
    o = ops()
    cuts, ids = [0, 5, 21, 30], [0, 1, 0]
    x, ad, st, ii, _ = problem(30, cuts, ids, 64, 128, 8, 2)
    dy = randn(30, 128, seed=9).to(torch.bfloat16)
    _, u = o.mixfp4_lora(x, ad, st, ii)
    ref = o.mixfp4_lora_backward(dy, x, u, ad, st, ii)
    x2, dy2 = x.clone(), dy.clone()
    x2[5:21], dy2[5:21] = float("nan"), float("inf")
    y, u2 = o.mixfp4_lora(x2, ad, st, ii)
    got = o.mixfp4_lora_backward(dy2, x2, u2, ad, st, ii)
    assert not y[:5].isnan().any() and not y[21:].isnan().any()
    assert torch.equal(got[0][:5], ref[0][:5]) and torch.equal(got[0][21:], ref[0][21:])
    assert torch.equal(got[1][0], ref[1][0]) and torch.equal(got[2][0], ref[2][0])


def test_beside_the_linear_layer():
    """linear() with an adapter equals linear() of the merged result, on the call's stream."""
    o = ops()
    x = randn(48, 512, seed=1).to(torch.bfloat16)
    w = o.mixfp4_quantize((randn(640, 512, seed=2) * 0.02).to(torch.bfloat16))
    _, ad, st, ii, _ = problem(48, [0, 20, 48], [0, 1], 512, 640, 16, 2)
    base = o.linear(x, w)
    ru, rum, ry, rym = reference(x, ad, [0, 20, 48], [0, 1], base)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = o.linear(x, w, stream=side)
    o.mixfp4_lora(x, ad, st, ii, base=y, out=y, stream=side)
    side.synchronize()
    assert torch.all((y.double() - ry).abs() <= 1e-5 * rym + 2.0 ** -23 * ry.abs())


def test_nothing_to_do():
    o = ops()
    x, ad, _, _, _ = problem(1, [0, 1], [0], 64, 32, 8, 2)
    empty = x[:0]
    y, u = o.mixfp4_lora(empty, ad, ints([0]), ints([]))
    assert y.shape == (0, 32) and u.shape == (0, 8)
    dx, da, db = o.mixfp4_lora_backward(torch.empty(0, 32, dtype=torch.bfloat16, device=DEV), empty, u, ad, ints([0]),
                                        ints([]))
    assert dx.shape == (0, 64) and torch.all(da == 0) and torch.all(db == 0)


def test_refusals():
    o = ops()
    x, ad, st, ii, base = problem(8, [0, 4, 8], [0, 1], 64, 48, 8, 2)
    good = dict(x=x, adapters=ad, starts=st, ids=ii, base=base)
    for bad in (dict(x=x.float()), dict(x=x[:, :48]), dict(x=x.cpu()), dict(adapters=None), dict(starts=st.long()),
                dict(starts=st[:2]), dict(ids=ii.long()), dict(ids=ii.cpu()), dict(starts=ints([0]), ids=ints([])),
                dict(base=base[:4]), dict(base=base.double()), dict(base=base.t().contiguous().t()),
                dict(out=base[:, :20]), dict(u=base)):
        with pytest.raises(ValueError):
            o.mixfp4_lora(**{**good, **bad})
    a, b, s = ad.a, ad.b, ad.scaling
    for bad in ((a.float(), b, s), (a[:, :7], b[..., :7], s), (a[..., :40].contiguous(), b, s), (a, b[:1], s),
                (a, b[..., :4], s), (a, b, s[:1]), (a, b, s.double()), (a.cpu(), b, s), (a[..., ::2], b, s),
                (torch.empty(1, 136, 64, dtype=torch.bfloat16, device=DEV),
                 torch.empty(1, 48, 136, dtype=torch.bfloat16, device=DEV), s[:1])):
        with pytest.raises(ValueError):
            o.Adapters(*bad)
    _, u = o.mixfp4_lora(**good)
    dy = randn(8, 48).to(torch.bfloat16)
    good = dict(dy=dy, x=x, u=u, adapters=ad, starts=st, ids=ii)
    for bad in (dict(dy=dy.float()), dict(dy=dy[:4]), dict(u=None), dict(u=u[:4]), dict(da=torch.empty(2, 8, 63, device=DEV)),
                dict(base=base), dict(workspace=torch.empty(8, device=DEV))):
        with pytest.raises(ValueError):
            o.mixfp4_lora_backward(**{**good, **bad})
    odd = torch.empty(8 * 72 + 4, dtype=torch.bfloat16, device=DEV)[4:].view(8, 72)[:, :64]
    with pytest.raises(o.MixFP4Error, match="misaligned"):
        o.mixfp4_lora(odd, ad, st, ii)
    ad5 = o.Adapters(a, torch.zeros(2, 40, 8, dtype=torch.bfloat16, device=DEV), s)
    with pytest.raises(ValueError, match="16"):
        o.mixfp4_lora_backward(dy[:, :40], x, u, ad5, st, ii)
