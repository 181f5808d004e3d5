"""Caches of more key heads than the calls count with are refused: twice their number and the query heads', in a 32-bit
count, came out negative and divided by zero."""
import ctypes

import pytest

from test_serving_abi import FAKE, append, attend, cache, fp4, gather, lib, ops  # noqa: F401

ERR_SHAPE = -2


@pytest.mark.parametrize("heads", [(1 << 20) + 1, 1 << 30, 1600000000, (1 << 31) - 1])
@pytest.mark.parametrize("make", [cache, fp4])
def test_too_many_heads(ops, lib, make, heads):  # noqa: F811
    c = make(ops, heads=heads)
    assert append(lib, c, T=1, k=FAKE << 1, v=FAKE << 2, q=FAKE << 3, out=FAKE << 4, kh=0, vh=0) == ERR_SHAPE
    assert gather(lib, c) == ERR_SHAPE
    assert attend(lib, c, H=heads) == ERR_SHAPE
    n = ctypes.c_int64(-1)
    assert lib.mixfp4_paged_attention_workspace(ctypes.byref(c), ctypes.c_int64(1), ctypes.c_int64(heads),
                                                ctypes.byref(n)) == ERR_SHAPE


def test_as_many_as_documented(ops, lib):  # noqa: F811
    c = cache(ops, heads=1 << 20)
    assert append(lib, c, T=0) == 0 and gather(lib, c, T=0) == 0 and attend(lib, c, B=0, H=1 << 20) == 0
