"""The entry points for drafted tokens, forks and page copies on CPU: invalid
arguments give the documented status before anything is enqueued, and the native
binding refuses what is not a CUDA tensor before it reaches the library."""
import ctypes
import os
import sys

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)
from test_serving_abi import FAKE, I, P, cache, fp4, lib, ops  # noqa: E402,F401


def tree(lib, c, **kw):
    f = dict(q=FAKE, qs=768, qt=256, qh=64, B=2, t=3, H=4, table=FAKE, ts=8, pages=8, lengths=FAKE, mask=FAKE, ms=3,
             counts=FAKE, window=0, cap=0.0, slopes=FAKE, out=FAKE, lse=FAKE, ws=FAKE, bytes=1 << 40, status=FAKE)
    f.update(kw)
    return lib.mixfp4_tree_attention(P(f["q"]), I(f["qs"]), I(f["qt"]), I(f["qh"]), I(f["B"]), I(f["t"]), I(f["H"]),
                                     ctypes.byref(c) if c else None, P(f["table"]), I(f["ts"]), I(f["pages"]),
                                     P(f["lengths"]), P(f["mask"]), I(f["ms"]), P(f["counts"]), ctypes.c_float(0.1),
                                     I(f["window"]), ctypes.c_float(f["cap"]), P(f["slopes"]), P(f["out"]),
                                     P(f["lse"]), P(f["ws"]), I(f["bytes"]), P(f["status"]), None)


@pytest.mark.parametrize("of", [cache, fp4])
def test_tree_attention_validation(ops, lib, of):  # noqa: F811
    c = of(ops)
    for kw in (dict(B=0), dict(t=0), dict(H=0)):
        assert tree(lib, c, q=0, table=0, lengths=0, out=0, ws=0, bytes=0, **kw) == 0, kw
    assert tree(lib, None) == -1
    for kw in (dict(B=-1), dict(t=-1), dict(t=65), dict(H=3), dict(H=-2), dict(qs=-8), dict(qt=-8), dict(qh=-8),
               dict(ts=7), dict(pages=-1), dict(window=-1), dict(bytes=0), dict(pages=1 << 30, ts=1 << 30), dict(ms=-1),
               dict(ms=2), dict(B=1 << 31)):
        assert tree(lib, c, **kw) == -2, kw
    for cap in (-1.0, 1e-7, 1e7, float("nan"), float("inf")):
        assert tree(lib, c, cap=cap) == -7, cap
    for kw in (dict(q=0), dict(lengths=0), dict(out=0), dict(ws=0), dict(table=0)):
        assert tree(lib, c, **kw) == -1, kw
    for kw in (dict(q=FAKE + 8), dict(qs=772), dict(qt=260), dict(qh=68), dict(out=FAKE + 8), dict(lse=FAKE + 2),
               dict(ws=FAKE + 128), dict(mask=FAKE + 4), dict(counts=FAKE + 2), dict(slopes=FAKE + 1),
               dict(table=FAKE + 2), dict(lengths=FAKE + 1), dict(status=FAKE + 1)):
        assert tree(lib, c, **kw) == -3, kw


def test_tree_workspace(ops, lib):  # noqa: F811
    c = cache(ops)
    n = ctypes.c_int64(-1)

    def ask(B, t, H, to=n):
        return lib.mixfp4_tree_attention_workspace(ctypes.byref(c), I(B), I(t), I(H), None if to is None else ctypes.byref(to))
    for B, t, H in ((0, 3, 4), (2, 0, 4), (2, 3, 0)):
        assert ask(B, t, H) == 0 and n.value == 0
    assert ask(2, 3, 4) == 0 and n.value > 0
    assert ask(2, 65, 4) == ask(-1, 3, 4) == ask(2, 3, 5) == ask(2, -1, 4) == -2
    assert ask(2, 3, 4, None) == -1


def accept(lib, c, **kw):
    f = dict(table=FAKE, ts=8, pages=8, lengths=FAKE, counts=FAKE + 4096, B=2, path=FAKE + 8192, ps=4, depth=4,
             out=FAKE + 65536)
    f.update(kw)
    return lib.mixfp4_kv_accept(ctypes.byref(c) if c else None, P(f["table"]), I(f["ts"]), I(f["pages"]),
                                P(f["lengths"]), P(f["counts"]), I(f["B"]), P(f["path"]), I(f["ps"]), I(f["depth"]),
                                P(f["out"]), None)


def test_accept_validation(ops, lib):  # noqa: F811
    c = cache(ops)
    assert accept(lib, c, B=0, table=0, lengths=0, counts=0, path=0, out=0) == 0
    assert accept(lib, None) == -1
    for kw in (dict(B=-1), dict(depth=-1), dict(depth=65, ps=65), dict(ps=3), dict(ps=-1), dict(ts=7), dict(pages=-1),
               dict(pages=1 << 30, ts=1 << 30)):
        assert accept(lib, c, **kw) == -2, kw
    for kw in (dict(table=0), dict(lengths=0), dict(counts=0), dict(path=0), dict(out=0)):
        assert accept(lib, c, **kw) == -1, kw
    for kw in (dict(table=FAKE + 2), dict(lengths=FAKE + 2), dict(counts=FAKE + 1), dict(path=FAKE + 3),
               dict(out=FAKE + 65537)):
        assert accept(lib, c, **kw) == -3, kw
    # the new lengths on what other CTAs still read (lengths themselves may be the place)
    for kw in (dict(out=FAKE + 4096), dict(out=FAKE + 8192 + 28), dict(out=FAKE + 60, lengths=FAKE + 1024),
               dict(lengths=FAKE + 65540)):
        assert accept(lib, c, **kw) == -7, kw


def fork(lib, c, **kw):
    f = dict(table=FAKE, ts=8, pages=8, lengths=FAKE + 4096, B=2, parents=FAKE + 8192, fresh=FAKE + 12288, n=3,
             table_out=FAKE + 65536, out=FAKE + 131072)
    f.update(kw)
    return lib.mixfp4_kv_fork(ctypes.byref(c) if c else None, P(f["table"]), I(f["ts"]), I(f["pages"]),
                              P(f["lengths"]), I(f["B"]), P(f["parents"]), P(f["fresh"]), I(f["n"]), P(f["table_out"]),
                              P(f["out"]), None)


def test_fork_validation(ops, lib):  # noqa: F811
    c = cache(ops)
    assert fork(lib, c, n=0, table=0, lengths=0, parents=0, fresh=0, table_out=0, out=0) == 0
    assert fork(lib, None) == -1
    for kw in (dict(B=-1), dict(n=-1), dict(ts=7), dict(pages=-1), dict(pages=1 << 30, ts=1 << 30)):
        assert fork(lib, c, **kw) == -2, kw
    assert fork(lib, cache(ops, page_size=1 << 30, heads=64)) == -2
    for kw in (dict(table=0), dict(lengths=0), dict(parents=0), dict(fresh=0), dict(table_out=0), dict(out=0)):
        assert fork(lib, c, **kw) == -1, kw
    for kw in (dict(table=FAKE + 2), dict(lengths=FAKE + 2), dict(parents=FAKE + 1), dict(fresh=FAKE + 3),
               dict(table_out=FAKE + 2), dict(out=FAKE + 2)):
        assert fork(lib, c, **kw) == -3, kw
    for kw in (dict(table_out=FAKE + 60), dict(out=FAKE + 4100), dict(table_out=FAKE + 8192 - 92), dict(out=FAKE + 12296),
               dict(out=FAKE + 65536 + 92)):
        assert fork(lib, c, **kw) == -7, kw


def test_copy_validation(ops, lib):  # noqa: F811
    def copy(c, src=FAKE, dst=FAKE, n=3):
        return lib.mixfp4_kv_copy_pages(ctypes.byref(c) if c else None, P(src), P(dst), I(n), None)
    c = cache(ops)
    assert copy(c, 0, 0, 0) == 0
    assert copy(None) == copy(c, src=0) == copy(c, dst=0) == -1
    assert copy(c, n=-1) == copy(c, n=1 << 31) == copy(cache(ops, page_size=1 << 30, heads=64)) == -2
    assert copy(c, src=FAKE + 2) == copy(c, dst=FAKE + 1) == -3
    assert copy(cache(ops, dtype=2)) == -4


def test_binding_refuses_before_the_library(ops):  # noqa: F811
    native = ops._native()
    c = cache(ops)
    at = ctypes.addressof(c)
    t = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: native.tree_attention(at, 0, t, i, i, None, None, None, 0, 0.0, None, None, None, False, None, None, 0),
                 lambda: native.tree_attention(at, 0, None, i, i, None, None, None, 0, 0.0, None, None, None, False,
                                               None, None, 0),
                 lambda: native.kv_accept(at, 0, i[:, None], i, i[:, None], i, None, 0),
                 lambda: native.kv_accept(at, 0, i[:, None], 3, i[:, None], i, None, 0),
                 lambda: native.kv_fork(at, 0, i[:, None], i, i, i, None, None, 0),
                 lambda: native.kv_copy_pages(at, 0, i, i, 0), lambda: native.kv_copy_pages(at, 0, i, None, 0)):
        with pytest.raises(ValueError):
            call()
    for name in ("tree_attention", "kv_accept", "kv_fork", "kv_copy_pages"):
        with pytest.raises(TypeError):
            getattr(native, name)(at, 0)
