"""Infinities in the adapters' activations, gradients and weights: results and
gradients are infinite or NaN where the definition in 64 bits is, sign for sign, and
what stays finite keeps the bounds of test_gpu_lora.py."""
import math
import os
import sys

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)
import test_gpu_lora as t  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF = math.inf


def alike(got, ref, bound):
    got = got.double()
    assert torch.equal(got.isnan(), ref.isnan())
    assert torch.equal(got.isposinf(), ref.isposinf()) and torch.equal(got.isneginf(), ref.isneginf())
    fine = ref.isfinite()
    assert torch.all((got - ref).abs()[fine] <= (1e-5 * bound + 2.0 ** -24 * ref.abs())[fine])


def compare(x, dy, ad, cuts, ids, base, dbase):
    o = t.ops()
    st, ii = t.ints(cuts), t.ints(ids)
    y, u = o.mixfp4_lora(x, ad, st, ii, base=base)
    dx, da, db = o.mixfp4_lora_backward(dy, x, u, ad, st, ii, base=dbase)
    ru, rum, ry, rym = t.reference(x, ad, cuts, ids, base)
    alike(u, ru, rum)
    alike(y, ry, rym)
    rdx, mdx = dbase.double().clone(), torch.zeros_like(dbase, dtype=torch.float64)
    rda, rdb = torch.zeros_like(ad.a, dtype=torch.float64), torch.zeros_like(ad.b, dtype=torch.float64)
    mda, mdb = torch.zeros_like(rda), torch.zeros_like(rdb)
    for i, j in enumerate(ids):
        r, s = slice(cuts[i], cuts[i + 1]), ad.scaling[j].double()
        xd, dyd, a, b = x[r].double(), dy[r].double(), ad.a[j].double(), ad.b[j].double()
        v, vm = s * (dyd @ b), s * (dyd.abs() @ b.abs())
        rdx[r] += v @ a
        mdx[r] += vm @ a.abs()
        rda[j] += v.T @ xd
        mda[j] += vm.T @ xd.abs()
        rdb[j] += s * (dyd.T @ ru[r])
        mdb[j] += s * (dyd.abs().T @ rum[r])
    alike(dx, rdx, mdx)
    alike(da, rda, mda)
    alike(db, rdb, mdb)
    return ry, rdx, rda, rdb


def problem(cuts, ids, K, N, R, L):
    x, ad, _, _, base = t.problem(cuts[-1], cuts, ids, K, N, R, L)
    return x, (t.randn(cuts[-1], N, seed=9) * 1e-3).to(torch.bfloat16), ad, base, t.randn(cuts[-1], K, seed=10) * 1e-3


# segments, K, N, rank: short ones (tiles of 8 and 16 tokens) and long ones (32 and 64), one to four tiles of ranks
CASES = [([0, 1, 3, 5, 9], [0, 1, 0, 1], 64, 96, 8), ([0, 1, 3, 5, 9], [0, 1, 0, 1], 272, 528, 24),
         ([0, 400, 900], [1, 0], 256, 512, 16), ([0, 400, 900], [1, 0], 256, 512, 64), ([0, 70], [0], 512, 96, 128),
         ([0, 2500, 2600, 5000], [0, 1, 1], 512, 4096, 32)]


@pytest.mark.parametrize("cuts,ids,K,N,R", CASES)
def test_infinite_activations_and_gradients(cuts, ids, K, N, R):
    """A token with an infinite x, one with an infinite dy, positive adapters so that most results have a sign."""
    x, dy, ad, base, dbase = problem(cuts, ids, K, N, R, 2)
    ad.a.copy_(ad.a.abs() + 0.01)
    ad.b.copy_(ad.b.abs() + 0.01)
    ad.b[:, 1::2] *= -1
    last = cuts[1] - 1
    x[0, 7], x[last, K - 1] = INF, -INF
    dy[0, 2], dy[last, N - 1] = -INF, INF
    y, dx, da, db = compare(x, dy, ad, cuts, ids, base, dbase)
    if last > 0:
        assert y[0, ::2].isposinf().all() and y[last, 1::2].isposinf().all() and dx[0].isneginf().all()
        assert da.isinf().any() and db.isinf().any()


@pytest.mark.parametrize("cuts,ids,K,N,R", CASES)
def test_infinite_weights(cuts, ids, K, N, R):
    """Infinite elements of both matrices against factors of few and of all bits."""
    x, dy, ad, base, dbase = problem(cuts, ids, K, N, R, 2)
    ad.b[0, 5, 3], ad.b[1, N - 1, R - 1] = INF, -INF
    y, dx, da, db = compare(x, dy, ad, cuts, ids, base, dbase)
    assert y.isinf().any()
    x, dy, ad, base, dbase = problem(cuts, ids, K, N, R, 2)
    ad.a[:, 0] = 0  # u is x's first element in rank 0: few bits
    ad.a[:, 0, 0] = 1
    ad.b[0, 5, 0], ad.b[1, 6, 0] = INF, -INF
    y, _, _, _ = compare(x, dy, ad, cuts, ids, base, dbase)
    assert y[:, 5:7].isinf().any() and not y.isnan().any()
    x, dy, ad, base, dbase = problem(cuts, ids, K, N, R, 2)
    ad.a[0, 2, 9], ad.a[1, R - 1, K - 1] = INF, -INF
    _, dx, _, _ = compare(x, dy, ad, cuts, ids, base, dbase)
    assert dx.isinf().any() and not dx.isnan().any()


@pytest.mark.parametrize("cuts,ids,K,N,R", CASES)
def test_infinite_inputs_of_finite_factors(cuts, ids, K, N, R):
    """An infinite x whose token has v of few bits, and an infinite dy whose token has u of few bits: the columns of
    the gradients are infinite, sign for sign, where the factor is not 0."""
    x, dy, ad, base, dbase = problem(cuts, ids, K, N, R, 2)
    ad.scaling.fill_(1.0)
    ad.b.copy_(torch.sign(ad.b.float()))
    dy.zero_()
    dy[:, 1] = 0.5  # v: 0.5 of either sign
    x[0, 7] = INF
    _, _, da, _ = compare(x, dy, ad, cuts, ids, base, dbase)
    assert da[ids[0], :, 7].isinf().all()
    x, dy, ad, base, dbase = problem(cuts, ids, K, N, R, 2)
    ad.a.copy_(torch.sign(ad.a.float()))
    x.zero_()
    x[:, 3] = 2.0  # u: 2 of either sign
    dy[0, 4] = -INF
    _, _, _, db = compare(x, dy, ad, cuts, ids, base, dbase)
    assert db[ids[0], 4].isinf().all()
