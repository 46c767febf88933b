"""Sequences that are copied, change places or end: against plain lists, bit for bit."""
import random

import pytest
import torch

import tree_ref
from paper_2602_03203_b200 import binding
from test_gpu_chunk import Case
from test_gpu_tree import run_tree

pytestmark = pytest.mark.gpu


def fork(c, source):
    c.cache.fork(source)
    old = [(s.k, s.v, s.f, s.pos) for s in c.seqs]
    for s, r in enumerate(source):
        seq = c.seqs[s]
        if r < 0:
            seq.k, seq.v, seq.f, seq.pos = ([x[:0] for x in part] for part in old[s])
        else:
            seq.k, seq.v, seq.f, seq.pos = (list(part) for part in old[r])


def pages(c):
    return sum(-(-len(s) // 16) for s in c.seqs) * c.Hkv


MAPS = [[0, 0, 0, 0, 0, 0], [0, 1, 2, 3, 4, 5], [1, 0, 3, 2, 5, 4], [1, 2, 3, 4, 5, 0], [-1, -1, -1, -1, -1, -1], [5, 5, 5, -1, -1, -1],
        [-1, 0, 1, 2, 3, 4], [1, 2, 0, 2, 1, 0], [3, 3, 3, 4, 4, 3], [0, 0, -1, 3, 2, 2], [2, 2, 2, 2, 2, -1]]


@pytest.mark.parametrize("D,g,Hkv", [(64, 4, 2), (128, 7, 3), (128, 8, 1)])
@pytest.mark.parametrize("source", MAPS)
def test_every_kind_of_map(D, g, Hkv, source):
    c = Case(Hkv, g, D, [40, 0, 1, 16, 200, 33], gap=2, seed=sum(source) + D)
    free0, used = c.cache.device_status()[1], pages(c)
    for _ in range(2):   # and once more on what came out
        fork(c, source)
        c.check_stored()
        assert c.cache.device_status() == (0, free0 + used - pages(c))
    run_tree(c, [tree_ref.tree(t, 3, t) for t in (3, 17, 0, 1, 40, 5)])   # every sequence goes on by itself
    c.check_stored()
    c.cache.reset()
    assert c.cache.device_status()[1] == free0 + used


def test_random_maps_over_layers():
    rng, batch = random.Random(3), 9
    cache = binding.Cache(3, 2, 2, 64, batch, 16, 200)
    total = cache.device_status()[1]
    state = {}
    for layer in range(3):
        for s in range(batch):
            n = rng.choice((0, 1, 15, 16, 17, 90, 150))
            k = torch.randn((2, n, 64), device="cuda").to(torch.bfloat16)
            f = torch.rand((2, n, 12), device="cuda")
            if n:
                cache.prefill(layer, s, k, -k, f)
            state[layer, s] = (k, f)
    for _ in range(12):
        source = [rng.choice((s, -1, rng.randrange(batch), rng.randrange(batch))) for s in range(batch)]
        cache.fork(source)
        old = dict(state)
        for layer in range(3):
            for s, r in enumerate(source):
                state[layer, s] = old[layer, r] if r >= 0 else (torch.zeros((2, 0, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 0, 12), device="cuda"))
            lens = [state[layer, s][0].shape[1] for s in range(batch)]
            assert cache.lengths(layer) == lens
            k, v, f, pos = cache.export_chunk(layer, lens)
            assert torch.equal(k, torch.cat([state[layer, s][0].transpose(0, 1) for s in range(batch)]))
            assert torch.equal(f, torch.cat([state[layer, s][1].transpose(0, 1) for s in range(batch)])) and torch.equal(v, -k)
        used = sum(-(-state[layer, s][0].shape[1] // 16) * 2 for layer in range(3) for s in range(batch))
        assert cache.device_status() == (0, total - used)
        cache.sync_lengths()
        assert cache.lengths(2) == lens


def test_pages_that_end_serve_the_copies():
    """A full pool: the copies take the pages of the sequences that they replace, and of those that end."""
    c = Case(2, 2, 64, [64, 64, 32, 64], num_pages=28, cap=64)
    fork(c, [0, 0, -1, 0])
    c.check_stored()
    assert c.cache.device_status() == (0, 4)
    c = Case(2, 2, 64, [48, 20, 0, 0], num_pages=10, cap=64)
    before = c.cache.lengths(0)
    c.cache.fork([0, 0, 0, 0])   # 24 pages: nothing is done
    status, free = c.cache.device_status()
    assert status == binding.DEV_POOL_EXHAUSTED and free == 0
    c.cache.sync_lengths()
    assert c.cache.lengths(0) == before
    c.check_stored()
    fork(c, [1, 1, -1, -1])   # four pages, of the six that sequence 0 gives back
    c.check_stored()


def test_budgets_and_decode_records_go_along():
    """Two caches, one of them shuffled by a fork: decoding, evicting and the features that follow agree bit for bit."""
    Hkv, g, D, batch = 2, 4, 64, 6
    gen = torch.Generator(device="cuda").manual_seed(7)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    caches = [binding.Cache(2, Hkv, g, D, batch, 64, 400, feature_window=16) for _ in range(2)]
    source = [2, 0, 1, 3, 3, -1]   # a cycle, one that stays with a copy, and an end
    for layer in range(2):
        for s in range(batch):
            # (the longest one is in both caches after the fork: how an attention is split goes by it)
            k, v = rand(Hkv, 200 - 10 * s, D), rand(Hkv, 200 - 10 * s, D)
            for i, cache in enumerate(caches):
                cache.set_budget(s, 60 + s)
                cache.prefill(layer, s, k, v)
    for step in range(11):   # queries on record, different numbers of them
        mask = 0b111111 if step < 5 else 0b001011
        for layer in range(2):
            k, v, q = rand(batch, Hkv, D), rand(batch, Hkv, D), rand(batch, Hkv * g, D)
            for cache in caches:
                cache.append_decode_attn(layer, k, v, q, seq_mask=mask)
    caches[1].fork(source)
    place = {s: r for s, r in enumerate(source) if r >= 0}
    for layer in range(2):
        n0, n1 = caches[0].lengths(layer), caches[1].lengths(layer)
        assert n1 == [n0[place[s]] if s in place else 0 for s in range(batch)]
    idx = torch.tensor([place.get(s, 0) for s in range(batch)], device="cuda")
    for step in range(9):
        for layer in range(2):
            k, v, q = rand(batch, Hkv, D), rand(batch, Hkv, D), rand(batch, Hkv * g, D)
            a = caches[0].append_decode_attn(layer, k, v, q)
            b = caches[1].append_decode_attn(layer, k[idx].contiguous(), v[idx].contiguous(), q[idx].contiguous(), seq_mask=0b011111)
            assert torch.equal(a[idx][:5], b[:5])
    for cache in caches:
        cache.evict_by_feature(4)
    for layer in range(2):
        n0, n1 = caches[0].lengths(layer), caches[1].lengths(layer)
        assert n1 == [n0[place[s]] if s in place else 0 for s in range(batch)] and n0 == [60 + s for s in range(batch)]
        for s, r in place.items():
            for h in range(Hkv):
                for x, y in zip(caches[0].export_head(layer, r, h), caches[1].export_head(layer, s, h)):
                    assert torch.equal(x, y), (layer, s, h)
    assert caches[1].device_status()[0] == 0


def test_forks_in_a_graph():
    c = Case(2, 4, 64, [50, 20, 33])
    source = [2, 0, 0]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.cache.fork([0, 1, 2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.fork(source)
    for _ in range(3):
        graph.replay()
        old = [(s.k, s.v, s.f, s.pos) for s in c.seqs]
        for s, r in enumerate(source):
            c.seqs[s].k, c.seqs[s].v, c.seqs[s].f, c.seqs[s].pos = old[r]
    c.cache.sync_lengths()
    assert c.status() == 0
    c.check_stored()


def test_a_large_batch():
    c = Case(1, 1, 64, [(s * 13) % 60 for s in range(256)], cap=64)
    rng = random.Random(1)
    perm = list(range(256))
    rng.shuffle(perm)
    for source in (perm, [s // 2 for s in range(256)], [255 - s if s % 3 else -1 for s in range(256)]):
        fork(c, source)
        assert c.status() == 0
        c.check_stored()


@pytest.mark.parametrize("layers", [2, 3])
def test_many_layers_of_a_large_batch(layers):
    """512 and 768 entries (layer, sequence)."""
    batch, rng = 256, random.Random(layers)
    cache = binding.Cache(layers, 2, 1, 64, batch, 16, 48)
    total, lens, parts = cache.device_status()[1], [], []
    for layer in range(layers):
        n = [rng.choice((0, 1, 7, 16, 17, 33)) for _ in range(batch)]
        k = torch.randn((sum(n), 2, 64), device="cuda").to(torch.bfloat16)
        cache.append_chunk(layer, k, -k, n)
        lens.append(n)
        parts.append(k.split(n))
    for source in ([rng.randrange(-1, batch) for _ in range(batch)], [(s + 1) % batch for s in range(batch)], [s // 8 * 8 for s in range(batch)]):
        cache.fork(source)
        for layer in range(layers):
            old, part = lens[layer], parts[layer]
            lens[layer] = [old[r] if r >= 0 else 0 for r in source]
            parts[layer] = [part[r] if r >= 0 else part[0][:0] for r in source]
            k, v, _, _ = cache.export_chunk(layer, lens[layer])
            assert cache.lengths(layer) == lens[layer] and torch.equal(k, torch.cat(parts[layer])) and torch.equal(v, -k)
        used = sum(-(-n // 16) * 2 for row in lens for n in row)
        assert cache.device_status() == (0, total - used)


def test_refusals():
    c = Case(1, 1, 64, [5, 6, 7])
    for bad in ([0, 1, 3], [0, 1, -2], [2 ** 20, 1, 2]):
        with pytest.raises(binding.FkvError):
            c.cache.fork(bad)
    for bad in ([0, 1], [0, 1, 2, 3], [0, 1, 2 ** 33]):
        with pytest.raises(ValueError):
            c.cache.fork(bad)
    c.check_stored()
