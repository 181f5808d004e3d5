"""The cache, attention and adapter entry points on CPU: the struct of the
binding is the header's, invalid arguments give the documented status before
anything is enqueued, and the native binding refuses what is not a CUDA tensor
before it reaches the library."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FAKE = 1 << 20  # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def ops():
    from paper_2605_31035_gb300 import build, ops
    build.build()
    return ops


@pytest.fixture(scope="module")
def lib(ops):
    return ctypes.CDLL(ops._LIB_PATH)  # a handle of its own: no argument types set


def cache(ops, **kw):
    f = dict(dtype=0, page_size=16, heads=2, head_dim=64, pages=4, k=FAKE, v=FAKE, page_stride=2048, token_stride=128,
             head_stride=64, k_scales=None, v_scales=None, scale_page_stride=0, scale_token_stride=0,
             scale_head_stride=0, k_ts=None, v_ts=None)
    f.update(kw)
    return ops._CKVCache(*[f[n] for n, _ in ops._CKVCache._fields_])


def fp4(ops, **kw):
    f = dict(dtype=1, page_stride=1024, token_stride=64, head_stride=32, k_scales=FAKE, v_scales=FAKE,
             scale_page_stride=128, scale_token_stride=8, scale_head_stride=4, k_ts=FAKE, v_ts=FAKE)
    f.update(kw)
    return cache(ops, **f)


def test_struct_is_the_headers(ops, tmp_path):
    """Offsets and size of mixfp4_kv_cache as the C compiler lays it out."""
    names = [n for n, _ in ops._CKVCache._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "mixfp4.h"\nint main(void) {\n' + "".join(
        f'  printf("%zu ", offsetof(mixfp4_kv_cache, {n}));\n' for n in names) +
        '  printf("%zu\\n", sizeof(mixfp4_kv_cache));\n  return 0;\n}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", f"-I{ROOT}/include", str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(ops._CKVCache, n).offset for n in names] + [ctypes.sizeof(ops._CKVCache)]


def P(v):
    return ctypes.c_void_p(v)


def I(v):
    return ctypes.c_int64(v)


def gather(lib, c, T=3, slots=FAKE, out=FAKE, dtype=0):
    return lib.mixfp4_kv_gather(ctypes.byref(c) if c else None, P(slots), I(T), P(out), P(out), dtype, None)


def test_cache_validation(ops, lib):
    assert gather(lib, None) == -1
    assert gather(lib, cache(ops, dtype=2)) == -4
    for kw in (dict(page_size=0), dict(heads=0), dict(head_dim=0), dict(head_dim=24), dict(head_dim=272),
               dict(pages=-1), dict(page_stride=-16), dict(pages=1 << 31)):
        assert gather(lib, cache(ops, **kw)) == -2, kw
    for kw in (dict(k=None), dict(v=None)):
        assert gather(lib, cache(ops, **kw)) == -1, kw
    for kw in (dict(k=FAKE + 16), dict(v=FAKE + 2), dict(token_stride=136), dict(head_stride=8), dict(page_stride=2056)):
        assert gather(lib, cache(ops, **kw)) == -3, kw
    assert gather(lib, fp4(ops, k_ts=None)) == -1
    assert gather(lib, fp4(ops, v_scales=None)) == -1
    assert gather(lib, fp4(ops, scale_token_stride=-8)) == -2
    for kw in (dict(k=FAKE + 4), dict(head_stride=36), dict(k_scales=FAKE + 2), dict(scale_head_stride=6),
               dict(v_ts=FAKE + 2)):
        assert gather(lib, fp4(ops, **kw)) == -3, kw
    # rows of a head dimension that is no multiple of 64 have scale bytes anywhere
    odd = dict(head_dim=48, head_stride=24, token_stride=48, page_stride=768, k_scales=FAKE + 1, v_scales=FAKE + 3,
               scale_head_stride=3, scale_token_stride=6, scale_page_stride=96)
    assert gather(lib, fp4(ops, **odd), T=0) == 0
    assert gather(lib, fp4(ops, **odd), T=-1) == -2


def test_gather_validation(ops, lib):
    c = cache(ops)
    assert gather(lib, c, T=0, slots=0, out=0) == 0
    assert gather(lib, c, dtype=2) == -4
    assert gather(lib, c, slots=0) == -1
    assert gather(lib, c, out=0) == -1
    assert gather(lib, c, out=FAKE + 16) == -3
    assert gather(lib, c, slots=FAKE + 4) == -3


def append(lib, c, **kw):
    f = dict(q=FAKE, qt=128, qh=64, H=4, k=FAKE, kt=128, kh=64, v=FAKE, vt=128, vh=64, dtype=1, T=3, positions=FAKE,
             cos_sin=FAKE, table=10, rot=64, inter=0, slots=FAKE, out=FAKE, mode=0)
    f.update(kw)
    return lib.mixfp4_kv_append(P(f["q"]), I(f["qt"]), I(f["qh"]), I(f["H"]), P(f["k"]), I(f["kt"]), I(f["kh"]),
                                P(f["v"]), I(f["vt"]), I(f["vh"]), f["dtype"], I(f["T"]), P(f["positions"]),
                                P(f["cos_sin"]), I(f["table"]), I(f["rot"]), f["inter"], ctypes.byref(c), P(f["slots"]),
                                P(f["out"]), f["mode"], None)


def test_append_validation(ops, lib):
    c = cache(ops)
    assert append(lib, c, T=0, k=0, v=0, q=0, slots=0, out=0) == 0
    assert append(lib, c, dtype=2) == -4
    assert append(lib, c, mode=4) == append(lib, c, mode=-1) == -7
    for kw in (dict(T=-1), dict(H=-1), dict(rot=65), dict(rot=66), dict(rot=-2), dict(table=-1), dict(kt=-128)):
        assert append(lib, c, **kw) == -2, kw
    for kw in (dict(k=0), dict(v=0), dict(q=0), dict(out=0), dict(slots=0), dict(positions=0), dict(cos_sin=0)):
        assert append(lib, c, **kw) == -1, kw
    for kw in (dict(k=FAKE + 16), dict(v=FAKE + 4), dict(q=FAKE + 16), dict(out=FAKE + 16), dict(kt=136), dict(vh=72),
               dict(qt=130), dict(cos_sin=FAKE + 16), dict(slots=FAKE + 4)):
        assert append(lib, c, **kw) == -3, kw


def attend(lib, c, **kw):
    f = dict(q=FAKE, qs=256, qh=64, B=2, H=4, table=FAKE, ts=8, pages=8, lengths=FAKE, window=0, out=FAKE, lse=FAKE,
             ws=FAKE, bytes=1 << 30)
    f.update(kw)
    return lib.mixfp4_paged_attention(P(f["q"]), I(f["qs"]), I(f["qh"]), I(f["B"]), I(f["H"]), ctypes.byref(c),
                                      P(f["table"]), I(f["ts"]), I(f["pages"]), P(f["lengths"]), ctypes.c_float(0.1),
                                      I(f["window"]), P(f["out"]), P(f["lse"]), P(f["ws"]), I(f["bytes"]), None)


def test_attention_validation(ops, lib):
    c = cache(ops)
    assert attend(lib, c, B=0, q=0, table=0, lengths=0, out=0, ws=0, bytes=0) == 0
    for kw in (dict(B=-1), dict(H=3), dict(H=-2), dict(qs=-8), dict(ts=7), dict(pages=-1), dict(window=-1),
               dict(bytes=100), dict(pages=1 << 30, ts=1 << 30)):
        assert attend(lib, c, **kw) == -2, kw
    for kw in (dict(q=0), dict(out=0), dict(lengths=0), dict(table=0), dict(ws=0)):
        assert attend(lib, c, **kw) == -1, kw
    for kw in (dict(q=FAKE + 8), dict(qs=260), dict(qh=68), dict(out=FAKE + 8), dict(table=FAKE + 2),
               dict(lengths=FAKE + 1), dict(lse=FAKE + 2), dict(ws=FAKE + 16)):
        assert attend(lib, c, **kw) == -3, kw
    n = ctypes.c_int64(-1)
    for kw, B, H in ((dict(), 3, 4), (dict(head_dim=256, head_stride=256, token_stride=512, page_stride=8192), 1, 64)):
        assert lib.mixfp4_paged_attention_workspace(ctypes.byref(cache(ops, **kw)), I(B), I(H), ctypes.byref(n)) == 0
        assert n.value > 0
    assert lib.mixfp4_paged_attention_workspace(ctypes.byref(c), I(3), I(5), ctypes.byref(n)) == -2
    assert lib.mixfp4_paged_attention_workspace(ctypes.byref(c), I(3), I(4), None) == -1


def lora(lib, **kw):
    f = dict(x=FAKE, dtype=0, T=4, K=64, ldx=64, a=FAKE, b=FAKE, s=FAKE, L=2, R=8, N=40, starts=FAKE, ids=FAKE, S=2,
             base=0, ldb=0, out=FAKE, ldo=40, u=FAKE)
    f.update(kw)
    return lib.mixfp4_lora(P(f["x"]), f["dtype"], I(f["T"]), I(f["K"]), I(f["ldx"]), P(f["a"]), P(f["b"]), P(f["s"]),
                           I(f["L"]), I(f["R"]), I(f["N"]), P(f["starts"]), P(f["ids"]), I(f["S"]), P(f["base"]),
                           I(f["ldb"]), P(f["out"]), I(f["ldo"]), P(f["u"]), None)


def backward(lib, **kw):
    f = dict(dy=FAKE, ldy=48, x=FAKE, ldx=64, dtype=0, T=4, K=64, u=FAKE, a=FAKE, b=FAKE, s=FAKE, L=2, R=8, N=48,
             starts=FAKE, ids=FAKE, S=2, base=0, ldb=0, dx=FAKE, ldd=64, da=FAKE, db=FAKE, v=FAKE)
    f.update(kw)
    return lib.mixfp4_lora_backward(P(f["dy"]), I(f["ldy"]), P(f["x"]), I(f["ldx"]), f["dtype"], I(f["T"]), I(f["K"]),
                                    P(f["u"]), P(f["a"]), P(f["b"]), P(f["s"]), I(f["L"]), I(f["R"]), I(f["N"]),
                                    P(f["starts"]), P(f["ids"]), I(f["S"]), P(f["base"]), I(f["ldb"]), P(f["dx"]),
                                    I(f["ldd"]), P(f["da"]), P(f["db"]), P(f["v"]), None)


def test_lora_validation(lib):
    assert lora(lib, T=0) == 0
    assert backward(lib, T=0, L=0) == 0
    for call in (lora, backward):
        assert call(lib, dtype=1) == -4
        for kw in (dict(T=-1), dict(K=72), dict(R=4), dict(R=12), dict(R=136), dict(N=-16), dict(L=-1), dict(L=65536),
                   dict(S=-1), dict(ldx=48), dict(base=FAKE, ldb=8), dict(N=1 << 25)):
            assert call(lib, **kw) == -2, kw
        for kw in (dict(x=0), dict(a=0), dict(b=0), dict(s=0), dict(starts=0), dict(ids=0), dict(u=0)):
            assert call(lib, **kw) == -1, kw
        for kw in (dict(x=FAKE + 16), dict(ldx=72), dict(a=FAKE + 16), dict(b=FAKE + 2), dict(u=FAKE + 8),
                   dict(starts=FAKE + 2), dict(s=FAKE + 1)):
            assert call(lib, **kw) == -3, kw
    assert lora(lib, ldo=39) == -2 and lora(lib, out=0) == -1 and lora(lib, out=FAKE + 2) == -3
    assert backward(lib, N=40) == -2 and backward(lib, ldd=63) == -2 and backward(lib, ldy=32) == -2
    assert backward(lib, da=0) == -1 and backward(lib, v=0) == -1 and backward(lib, dy=0) == -1
    assert backward(lib, db=FAKE + 16) == -3 and backward(lib, dy=FAKE + 16) == -3


def test_binding_refuses_before_the_library(ops):
    import torch
    native = ops._native()
    c = cache(ops)
    at = ctypes.addressof(c)
    k = torch.zeros(3, 2, 64)
    slots = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="k must be"):
        native.kv_append(at, 0, k, k, slots, None, None, None, False, 0, None, 0)
    with pytest.raises(ValueError, match="k must be"):
        native.kv_append(at, 0, 3, k, slots, None, None, None, False, 0, None, 0)
    with pytest.raises(ValueError, match="slots"):
        native.kv_gather(at, 0, slots, False, None, None, 0)
    with pytest.raises(ValueError, match="q must be"):
        native.paged_attention(at, 0, k.to(torch.bfloat16), slots, slots, None, 0, None, None, False, None, 0)
    with pytest.raises(ValueError, match="adapters"):
        native.lora(k, k, k, 0, k, slots, slots, None, None, None, 0)
    with pytest.raises(ValueError, match="adapters"):
        native.lora_backward(k, k, k, 0, k, k, k, slots, slots, None, None, None, None, None, 0)
    with pytest.raises(TypeError):
        native.kv_append(at, 0)
    with pytest.raises(ValueError, match="CUDA"):
        ops.KVCache(torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="CUDA"):
        ops.Adapters(k.to(torch.bfloat16), k.to(torch.bfloat16), torch.ones(3))
    for call in (lambda: ops.mixfp4_kv_append(k, k, None, slots), lambda: ops.mixfp4_kv_gather(None, slots),
                 lambda: ops.mixfp4_paged_attention(k, None, slots, slots)):
        with pytest.raises(ValueError, match="KVCache"):
            call()
    with pytest.raises(ValueError, match="Adapters"):
        ops.mixfp4_lora(k, None, slots, slots)


def test_native_binding_is_loud_when_missing(ops, tmp_path, monkeypatch):
    monkeypatch.setattr(ops, "_binding", None)
    monkeypatch.setattr(ops, "_BINDING_PATH", str(tmp_path / "missing.so"))
    with pytest.raises(RuntimeError, match="missing"):
        ops._native()


def test_binding_calls_every_entry_point_once():
    text = open(os.path.join(ROOT, "paper_2605_31035_gb300", "csrc", "binding.cpp")).read()
    for name in ("kv_append", "kv_gather", "paged_attention", "lora", "lora_backward"):
        assert len(re.findall(rf"st = mixfp4_{name}\(", text)) == 1, name
