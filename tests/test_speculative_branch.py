"""Which pages a branch gets, on CPU tensors: of parents within a page, at its end, and with a full table."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def step():
    spec = importlib.util.spec_from_file_location("speculative_step", os.path.join(ROOT, "examples", "speculative_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("page,width", [(16, 3), (1, 4), (7, 1)])
def test_pages_of_a_branch(step, page, width):
    lengths = torch.arange(page * width + 1, dtype=torch.int32)
    parents = torch.arange(page * width + 1, dtype=torch.int32).flip(0)
    own = torch.arange(parents.numel() * width, dtype=torch.int32).view(-1, width) + 100
    fresh, part = step.branch_pages(own, lengths, parents, page)
    assert fresh.dtype == torch.int32
    for i, p in enumerate(parents.tolist()):
        n = int(lengths[p])
        assert int(part[i]) == n // page
        assert int(fresh[i]) == (int(own[i, n // page]) if n % page else -1)
    later = torch.arange(width) >= part[:, None]
    assert not later[0].any() and later[-1].all()  # a full table is shared as a whole, an empty one not at all


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["bf16", "mixfp4"])
def test_branches_of_a_full_table(step, cache):
    """Requests that fill their tables, end with a page or lie within one branch; their rows are the parents'."""
    layer = step.Layer(3, 100, 28, hidden=256, q_heads=4, kv_heads=2, head_dim=64, cache=cache)
    width = layer.table.shape[1]
    layer.lengths = torch.tensor([width * 16, 32, 37], dtype=torch.int32, device="cuda:0")
    parents = torch.tensor([0, 1, 2, 0], dtype=torch.int32, device="cuda:0")

    def rows(b):
        slots = layer.slots(b, torch.arange(int(layer.lengths[b]), device="cuda:0"))
        return [x[slots // 16, slots % 16].view(torch.uint8).clone() for x in (layer.cache.k, layer.cache.v)]
    before, tables = [rows(b) for b in range(3)], layer.table.clone()
    layer.branch(parents)
    assert layer.lengths.tolist() == [width * 16, 32, 37, width * 16]
    for i, p in enumerate(parents.tolist()):
        assert all(torch.equal(x, y) for x, y in zip(rows(i), before[p]))
    assert torch.equal(layer.table[0], tables[0]) and torch.equal(layer.table[3], tables[0])
    shared = (layer.table[1] == tables[1]).tolist(), (layer.table[2] == tables[2]).tolist()
    assert shared[0] == [True] * 2 + [False] * (width - 2) and shared[1] == [True] * 2 + [False] * (width - 2)
