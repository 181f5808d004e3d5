"""mixfp4_kv_append's q_out on its inputs: queries may be rotated in place only
where a thread has both elements of each pair; other overlaps are refused before
anything is enqueued, by the entry point and by the binding."""
import ctypes

import pytest
import torch

from test_serving_abi import FAKE, append, cache, lib, ops  # noqa: F401

ERR_ARG = -7


@pytest.mark.parametrize("rot", [16, 24, 40, 48, 80])
def test_in_place_is_refused_where_pairs_are_shared(ops, lib, rot):  # noqa: F811
    c = cache(ops, head_dim=80, head_stride=80, token_stride=160, page_stride=2560)
    f = dict(dtype=0, qt=320, qh=80, kt=160, kh=80, vt=160, vh=80, k=FAKE << 1, v=FAKE << 2, rot=rot)
    assert append(lib, c, **f) == ERR_ARG


def test_overlaps_are_refused(ops, lib):  # noqa: F811
    """Of fp32 or strided queries, of another place of theirs, of keys and of values: 3 tokens of 4 heads of 64."""
    c = cache(ops)
    f = dict(dtype=0, qt=256, qh=64, k=FAKE << 1, v=FAKE << 2)
    size = 3 * 256 * 2
    for kw in (dict(dtype=1), dict(qt=512), dict(qh=128), dict(out=FAKE + size - 32), dict(out=FAKE - size + 32),
               dict(out=FAKE + 512, q=FAKE), dict(k=FAKE), dict(v=FAKE + 32), dict(k=FAKE - 3 * 256 + 32),
               dict(q=FAKE - 4096 * 2, qt=4096, out=FAKE + 256), dict(q=FAKE << 3, k=FAKE, out=FAKE)):
        assert append(lib, c, **{**f, **kw}) == ERR_ARG, kw


def test_binding_says_why(ops):  # noqa: F811
    """The binding's own refusal needs CUDA tensors: its text is checked against the source here, its effect on the GPU."""
    import os
    text = open(os.path.join(os.path.dirname(ops.__file__), "csrc", "binding.cpp")).read()
    assert "must not overlap k, v or q" in text and "append_overlaps(" in text


@pytest.mark.gpu
@pytest.mark.parametrize("D,rot,inter", [(128, 128, False), (128, 64, False), (80, 40, True), (64, 0, False), (96, 32, False)])
@pytest.mark.parametrize("fp4", [False, True])
def test_in_place_gives_the_same(ops, D, rot, inter, fp4):  # noqa: F811
    import test_gpu_kv_cache as t
    T, H = 300, 6
    slots = torch.arange(T, device=t.DEV)
    q, k = (t.randn(T, h, D, seed=h).to(torch.bfloat16) for h in (H, 2))
    args = dict(positions=slots, cos_sin=t.angles(T, rot) if rot else None, interleaved=inter)
    got = []
    for out in (None, q):
        c = t.make_cache(fp4, 20, 16, 2, D)
        got.append((ops.mixfp4_kv_append(k, k, c, slots, q=q, out=out, **args).clone(), c.k.clone(), c.v.clone()))
    for a, b in zip(*got):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    one = t.randn(1, H, D + 16, seed=3).to(torch.bfloat16)[..., :D]  # not dense over its heads
    with pytest.raises(ValueError):
        ops.mixfp4_kv_append(k[:1], k[:1], t.make_cache(fp4, 1, 16, 2, D), slots[:1], q=one, out=one, **{**args, "positions": slots[:1]})


@pytest.mark.gpu
def test_binding_refuses_overlaps(ops):  # noqa: F811
    import test_gpu_kv_cache as t
    slots = torch.arange(5, device=t.DEV)
    c = t.make_cache(False, 1, 16, 2, 80)
    q, k = (t.randn(5, h, 80, seed=h).to(torch.bfloat16) for h in (4, 2))
    for rot, out in ((80, q), (40, q), (0, torch.cat([q, q])[5:])):
        before = q.clone()
        args = dict(positions=slots, cos_sin=t.angles(9, rot) if rot else None, q=q, out=out)
        if out is q:
            with pytest.raises(ValueError, match="overlap"):
                ops.mixfp4_kv_append(k, k, c, slots, **args)
        else:
            assert torch.equal(ops.mixfp4_kv_append(k, k, c, slots, **args), q)
        assert torch.equal(q, before)
    both = torch.zeros(5 * 4 * 80 + 160, dtype=torch.bfloat16, device=t.DEV)
    with pytest.raises(ValueError, match="overlap"):
        ops.mixfp4_kv_append(k, k, c, slots, q=both[160:].view(5, 4, 80), out=both[:-160].view(5, 4, 80))
    with pytest.raises(ValueError, match="overlap"):
        ops.mixfp4_kv_append(both[:800].view(5, 2, 80), k, c, slots, q=q, out=both[:-160].view(5, 4, 80))
    wide = torch.zeros(5, 8, 80, dtype=torch.float32, device=t.DEV)
    halves = wide.view(torch.bfloat16)  # fp32 queries and their bf16 result in one memory
    with pytest.raises(ValueError, match="overlap"):
        ops.mixfp4_kv_append(k.float(), k.float(), c, slots, q=wide[:, :4], out=halves.view(-1)[:1600].view(5, 4, 80))
