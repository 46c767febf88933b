"""Long mixtures of the calls on one cache whose pool is nearly full, against plain lists: trees, paths, roll-backs, forks, chunks."""
import random

import pytest
import torch

import tree_ref
from paper_2602_03203_b200 import binding
from test_gpu_chunk import Case
from test_gpu_fork import fork
from test_gpu_tree import commit, extend, make_trees, packed, path_tensors, run_tree

pytestmark = pytest.mark.gpu


def pages(c, lens=None):
    return sum(-(-n // 16) for n in (lens or [len(s) for s in c.seqs])) * c.Hkv


@pytest.mark.parametrize("D,g,Hkv,batch,pool", [(64, 4, 2, 5, 120), (128, 3, 1, 12, 90), (128, 8, 3, 2, 100)])
@pytest.mark.parametrize("seed", [1, 2])
def test_mixtures(D, g, Hkv, batch, pool, seed):
    rng = random.Random(seed)
    c = Case(Hkv, g, D, [rng.choice((0, 1, 15, 16, 17, 40)) for _ in range(batch)], num_pages=pool, cap=320)
    total = pages(c) + c.cache.device_status()[1]
    for step in range(60):
        n = [len(s) for s in c.seqs]
        lens = [rng.choice((0, 0, 1, 2, 7, 16, 33, 60)) for _ in range(batch)]
        keep = [rng.randrange(x + 1) if rng.random() < 0.3 else x for x in n] if rng.random() < 0.4 else None
        kind = rng.choice(("tree", "tree", "tree", "chunk", "fork", "fork"))
        if kind == "fork":
            source = [rng.choice((s, s, -1, rng.randrange(batch))) for s in range(batch)]
            if pages(c, [n[r] if r >= 0 else 0 for r in source]) > total:
                c.cache.fork(source)   # (too few pages, nothing moves)
                assert c.cache.device_status() == (binding.DEV_POOL_EXHAUSTED, total - pages(c))
                c.cache.sync_lengths()
            else:
                fork(c, source)
        else:
            if any((k + t > 320) for k, t in zip(keep or n, lens)) or pages(c, [k + t for k, t in zip(keep or n, lens)]) > total:
                lens, keep = [0] * batch, [x // 2 for x in n]   # make room
                k, v, _ = c.chunk(lens)
                c.cache.append_chunk(0, k, v, lens, keep_lens=keep)
                c.extend(k, v, lens, keep=keep)
            elif kind == "chunk":
                k, v, _ = c.chunk(lens)
                c.cache.append_chunk(0, k, v, lens, keep_lens=keep)
                c.extend(k, v, lens, keep=keep)
            else:
                trees = make_trees(lens, rng.randint(1, 4), seed=step, near=rng.choice((2, 1000)))
                if rng.random() < 0.5:
                    run_tree(c, trees, keep=keep)
                else:
                    k, v, _ = c.chunk(lens)
                    c.cache.append_tree(0, k, v, lens, c.cache.tree_masks(packed(trees), lens), keep_lens=keep)
                    extend(c, k, v, trees, keep)
                if rng.random() < 0.8:
                    paths = [sorted(tree_ref.path_up(t, rng.randrange(len(t)))) if t and rng.random() < 0.9 else [] for t in trees]
                    c.cache.commit_tree(lens, *path_tensors(paths, max(1, max(lens))))
                    commit(c, trees, paths)
                    c.cache.sync_lengths()
        assert c.cache.device_status() == (0, total - pages(c)), step
        if step % 6 == 5:
            c.check_stored()
    c.check_stored()
    c.cache.reset()
    assert c.cache.device_status() == (0, total)


@pytest.mark.parametrize("batch", [9, 10, 17, 18, 40])
def test_more_copies_of_one_sequence_than_one_reading_serves(batch):
    """A page goes to eight copies at a time; with the last sequence as the source too, and with the source itself going away."""
    for n in (1, 100, 330):
        for source in ([0] * batch, [batch - 1] * batch, [-1] + [0] * (batch - 1), [1] + [0] * (batch - 1)):
            c = Case(2, 3, 64, [n] + [7 * s % 40 for s in range(1, batch - 1)] + [n // 2 + 1], cap=340)
            fork(c, source)
            assert c.status() == 0
            c.check_stored()


@pytest.mark.parametrize("short", [0, 1])
def test_a_pool_that_is_just_large_enough_for_a_fork(short):
    lens = [50, 33, 16, 0]
    source = [0, 0, 1, 0]   # copies for places 1 and 3, 8 pages each; place 2 takes over those of 1 and gives back 2
    c = Case(2, 2, 64, lens, num_pages=16 + 14 - short, cap=64)
    before = c.cache.device_status()[1]
    if short:
        c.cache.fork(source)
        assert c.cache.device_status() == (binding.DEV_POOL_EXHAUSTED, before)
        c.cache.sync_lengths()
    else:
        fork(c, source)
        assert c.status() == 0
    c.check_stored()
