"""Budgets that differ from sequence to sequence, through forks that are replayed or find no pages, with an eviction behind them."""
import pytest
import torch

from paper_2602_03203_b200 import binding

pytestmark = pytest.mark.gpu

HKV, G, D = 2, 2, 64


def make(lens, budgets, num_pages=0):
    """One-layer cache; pair i of sequence s has a feature row of its own, so every eviction keeps other pairs."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    cache = binding.Cache(1, HKV, G, D, len(lens), 16, 400, num_pages=num_pages)
    for s, (n, budget) in enumerate(zip(lens, budgets)):
        cache.set_budget(s, budget)
        k = torch.randn((HKV, 400, D), generator=gen, device="cuda").to(torch.bfloat16)
        f = torch.rand((HKV, 400, 6 * G), generator=gen, device="cuda")
        if n:
            cache.prefill(0, s, k[:, :n].contiguous(), -k[:, :n], f[:, :n].contiguous())
    return cache


def same(a, b, lens):
    assert a.lengths(0) == b.lengths(0) == lens
    for s, n in enumerate(lens):
        for h in range(HKV if n else 0):
            for x, y in zip(a.export_head(0, s, h), b.export_head(0, s, h)):
                assert torch.equal(x, y), (s, h)


def evict(cache):
    cache.sync_lengths()
    cache.evict_by_feature(4)
    on_host = cache.lengths(0)
    cache.sync_lengths()
    assert cache.lengths(0) == on_host and cache.device_status()[0] == 0   # (the device has come to the same lengths)


@pytest.mark.parametrize("source,replays,budgets", [
    ([1, 0, 2], 2, [20, 200, 300]),      # a swap and back
    ([1, 2, 0], 2, [20, 60, 300]),       # a cycle, two steps on
    ([1, 2, 0], 4, [300, 200, 20]),
    ([0, 0, 1], 2, [20, 300, 300]),      # a chain: the first replay leaves two small budgets, the second three
    ([0, 0, 1], 3, [300, 20, 20]),       # ... and none
    ([2, -1, 0], 3, [300, 30, 17])])     # an end that keeps its place's own budget
def test_replayed_forks_and_an_eviction(source, replays, budgets):
    lens = [100, 90, 80]
    a, b = make(lens, budgets), make(lens, budgets)
    a.fork([0, 1, 2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.fork(source)
    for _ in range(replays):
        graph.replay()
        b.fork(source)
        lens, budgets = [lens[r] if r >= 0 else 0 for r in source], [budgets[r] if r >= 0 else x for r, x in zip(source, budgets)]
    for cache in (a, b):
        evict(cache)
    same(a, b, [min(n, x) for n, x in zip(lens, budgets)])
    for cache in (a, b):   # and the budgets go on with their sequences
        cache.fork([1, 2, 0])
        k = torch.randn((330, HKV, D), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
        cache.append_chunk(0, k, k, [110, 110, 110])
        evict(cache)
    lens = [min(n, x) for n, x in zip(lens, budgets)]
    same(a, b, [min(lens[r] + 110, budgets[r]) for r in (1, 2, 0)])


def test_a_fork_without_pages_leaves_the_budgets():
    lens, budgets = [48, 20, 0, 0], [100, 17, 30, 40]
    a, b = make(lens, budgets, num_pages=14), make(lens, budgets, num_pages=14)
    a.fork([0, 0, 0, 0])   # 18 pages, of 4 free ones and 4 that sequence 1 gives back
    assert a.device_status() == (binding.DEV_POOL_EXHAUSTED, 4)
    for cache in (a, b):
        evict(cache)
    same(a, b, [48, 17, 0, 0])
    a.fork([1, 0, 2, 3])   # (moves tables only)
    a.set_budget(2, 5)
    evict(a)
    assert a.lengths(0) == [17, 48, 0, 0]


def test_a_restored_workspace_brings_its_budgets():
    a = make([100, 90], [50, 60])
    saved = a.snapshot()
    a.set_budget(0, 10)
    a.restore(saved)
    evict(a)
    assert a.lengths(0) == [50, 60]
