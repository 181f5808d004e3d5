"""The decode example's step (projections, adapters, append, attention together)
against the same layer in 64 bits on the weights and the cache as stored, and
its replay from a CUDA graph."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("decode_step", os.path.join(ROOT, "examples", "decode_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def small(m, cache, seed=0):
    return m.Layer(5, 70, 8, hidden=512, q_heads=8, kv_heads=2, head_dim=64, rank=8, adapters=2, cache=cache, seed=seed)


def projection(x, w, lora, ids):
    """x_deq W^T and the adapters' share in 64 bits; x quantized as the layer quantizes it."""
    from paper_2605_31035_gb300 import ops
    y = ops.mixfp4_dequantize(ops.mixfp4_quantize(x)).double() @ ops.mixfp4_dequantize(w).double().T
    for i, j in enumerate(ids.tolist()):
        if j >= 0:
            y[i] += 2.0 * (x[i].double() @ lora.a[j].double().T) @ lora.b[j].double().T
    return y


@pytest.mark.parametrize("cache", ["bf16", "mixfp4"])
def test_step_matches_the_layer_in_64_bits(cache):
    from paper_2605_31035_gb300 import ops
    m = example()
    layer = small(m, cache)
    x, n = layer.x, layer.lengths.tolist()
    pos = layer.positions.clone()
    y = layer.step(x)
    qkv = projection(x, layer.w_qkv, layer.lora_qkv, layer.ids)
    cs = layer.cos_sin[pos].double()
    c, s = cs[:, None, :32], cs[:, None, 32:]

    def turn(t):
        a, b = t[..., :32], t[..., 32:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    q, k, v = qkv[:, :512].view(5, 8, 64), qkv[:, 512:640].view(5, 2, 64), qkv[:, 640:].view(5, 2, 64)
    q, k = turn(q).to(torch.bfloat16).double(), turn(k)
    out = torch.empty(5, 8, 64, dtype=torch.float64, device=x.device)
    for b in range(5):
        at = torch.arange(n[b] + 1, device=x.device)
        rk, rv = (t.double() for t in ops.mixfp4_kv_gather(layer.cache, layer.slots_of(b, at), torch.float32))
        # the new token's row is what was computed here: to the cache's own rounding
        step = 2.0 ** -8 if cache == "bf16" else 0.2
        assert (rk[-1] - k[b]).abs().max() <= step * k[b].abs().max()
        assert (rv[-1] - v[b]).abs().max() <= step * v[b].abs().max()
        p = (torch.einsum("hgd,nhd->hgn", q[b].view(2, 4, 64), rk) / 8).softmax(-1)
        out[b] = torch.einsum("hgn,nhd->hgd", p, rv).reshape(8, 64)
    ref = projection(out.flatten(1).to(torch.bfloat16), layer.w_o, layer.lora_o, layer.ids)
    # q, the attention's result and its quantized form may round to a neighbour of the reference's
    assert (y.double() - ref).norm() <= 0.02 * ref.norm()
    assert layer.lengths.tolist() == [k + 1 for k in n]


@pytest.mark.parametrize("cache", ["bf16", "mixfp4"])
def test_steps_from_a_graph_equal_steps(cache):
    m = example()
    a, b = small(m, cache), small(m, cache)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.step(b.x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = b.step(b.x)
    ref = a.step(a.x)
    for _ in range(3):
        ref = a.step(a.x)
        graph.replay()
        assert torch.equal(y, ref)
    assert torch.equal(a.lengths, b.lengths)


def test_example_runs(capsys):
    m = example()
    m.main(["--batch", "4", "--context", "100", "--steps", "3", "--graph"])
    m.main(["--batch", "3", "--context", "64", "--steps", "2", "--cache", "bf16"])
    assert capsys.readouterr().out.count("us a step") == 2
