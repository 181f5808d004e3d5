"""Refusals of the attention of drafted trees' failure self-test, on CPU: the documented status before anything is enqueued."""
import ctypes
import os
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)
from test_serving_abi import FAKE, I, P, cache, fp4, lib, ops  # noqa: E402,F401


@pytest.mark.parametrize("of", [cache, fp4])
def test_validation(ops, lib, of):  # noqa: F811
    c = of(ops, head_dim=128, **(dict(scale_token_stride=16, scale_head_stride=8) if of is fp4 else {}))

    def call(c=c, **kw):
        f = dict(q=FAKE, B=2, t=3, H=4, table=FAKE, pages=8, lengths=FAKE, out=FAKE, ws=FAKE, bytes=1 << 40, status=FAKE,
                 limit=1000)
        f.update(kw)
        return lib.mixfp4_selftest_tree_attention_missed_rows(
            P(f["q"]), I(f["B"]), I(f["t"]), I(f["H"]), ctypes.byref(c) if c else None, P(f["table"]), I(f["pages"]),
            P(f["lengths"]), P(f["out"]), P(f["ws"]), I(f["bytes"]), P(f["status"]), ctypes.c_uint64(f["limit"]), None)
    for kw in (dict(B=0), dict(t=0), dict(H=0), dict(t=65), dict(H=3), dict(pages=-1), dict(bytes=0)):
        assert call(**kw) == -2, kw
    assert call(c=of(ops, head_dim=64)) == call(c=of(ops, head_dim=256)) == -2
    assert call(limit=0) == call(limit=2_000_000_001) == -7
    for kw in (dict(c=None), dict(status=0), dict(q=0), dict(table=0), dict(lengths=0), dict(out=0), dict(ws=0)):
        assert call(**kw) == -1, kw
    for kw in (dict(q=FAKE + 8), dict(out=FAKE + 8), dict(ws=FAKE + 128), dict(status=FAKE + 1)):
        assert call(**kw) == -3, kw
