"""Attention of trees that are stored already (tree_attn by itself): every form of the kernels against the 64-bit form."""
import math

import pytest
import torch

import tree_ref
from paper_2602_03203_b200 import binding
from test_gpu_chunk import Case
from test_gpu_tree import check, depths, extend, make_trees, packed

pytestmark = pytest.mark.gpu


def run_stored(c, trees, window=0, sinks=0, pos=None, scale=0.0, launches=None, seen_of=None, masks=None):
    """append_tree, then tree_attn; twice, since nothing of the second call may depend on the first."""
    lens = [len(t) for t in trees]
    k, v, q = c.chunk(lens)
    if masks is None:
        masks = c.cache.tree_masks(packed(trees), lens)
    c.cache.append_tree(0, k, v, lens, masks, pos=pos)
    extend(c, k, v, trees, pos=pos)
    before = c.cache.launch_count()
    out = torch.full((q.shape[0] + 3,) + q.shape[1:], 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((q.shape[0] + 3, q.shape[1]), 7.0, device="cuda")
    c.cache.tree_attn(0, q, lens, masks, window=window, sinks=sinks, out=out[:-3], lse=lse[:-3], scale=scale)
    assert launches is None or c.cache.launch_count() - before == launches
    assert c.status() == 0
    check(c, out, lse, q, trees, window, sinks, scale or None, seen_of)
    assert bool((out[-3:] == 3).all()) and bool((lse[-3:] == 7).all())   # rows behind the last node stay
    again = c.cache.tree_attn(0, q, lens, masks, window=window, sinks=sinks, scale=scale)   # (without a log-sum-exp)
    assert torch.equal(again, out[:-3])
    c.check_stored()
    return q, out, lse, masks


# Trees of up to 64 query rows stand twice in a tile, longer ones once: both forms for both head dimensions, with and without windows.
@pytest.mark.parametrize("D,g,lens", [(128, 4, [16, 0, 9, 3]), (128, 8, [30, 1, 0, 100]), (64, 4, [16, 1, 7, 0]), (64, 3, [40, 256, 5, 0])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (256, 0), (256, 4), (300, 64), (1000, 1)])
@pytest.mark.parametrize("stored", [[0, 1, 15, 16], [333, 17, 80, 1000], [1203, 96, 0, 255]])
def test_every_form_of_the_cluster_kernel(D, g, lens, window, sinks, stored):
    for near, gap in ((1000, 1), (2, 4)):
        c = Case(2, g, D, stored, gap=gap, sinks=64, seed=window + D, cap=1600)
        run_stored(c, make_trees(lens, 2, near=near), window, sinks, launches=1)


@pytest.mark.parametrize("D,g,Hkv,launches", [(128, 4, 4, 1), (128, 4, 6, 2), (64, 7, 4, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (256, 4)])
def test_the_general_kernel(D, g, Hkv, launches, window, sinks):
    """144 blocks of query rows, a CTA each, and more than the card has SMs: attention and join."""
    lens = [100, 33, 0, 256, 64, 19, 20, 128, 90, 37, 18, 255]
    c = Case(Hkv, g, D, [(s * 67) % 500 for s in range(len(lens))], gap=3, sinks=sinks, cap=800)
    run_stored(c, make_trees(lens, 3, near=6), window, sinks, launches=launches)


@pytest.mark.parametrize("D,g", [(128, 1), (64, 1), (128, 7)])
@pytest.mark.parametrize("nodes", [1, 15, 16, 17, 63, 64, 65, 128, 129, 256])
def test_trees_that_begin_and_end_inside_pages(D, g, nodes):
    """The tree's first pairs share a page with the last ones ahead of it, at every place of a key tile of five pages."""
    for n in (0, 1, 15, 16, 64, 79, 80, 81, 95, 97, 500):
        c = Case(1, g, D, [n], seed=n, cap=n + 300)
        run_stored(c, [tree_ref.tree(nodes, 3, nodes + n, near=4)])


def test_given_positions_and_scale():
    for D, g, T in ((128, 4, 30), (64, 8, 8)):
        c = Case(2, g, D, [600], gap=40, sinks=8)
        parents = tree_ref.tree(T, 3, 5)
        pos = int(c.seqs[0].pos[0][-1]) + 5 + 3 * depths(parents)
        run_stored(c, [parents], window=400, sinks=4, pos=pos.to(torch.int32), scale=0.2)


@pytest.mark.parametrize("window", [0, 64])
def test_masks_of_other_kinds_and_rows_that_see_nothing(window):
    lens = [50, 33]
    c = Case(2, 4, 128, [0, 90])
    gen = torch.Generator().manual_seed(3)
    seen = [torch.tril(torch.rand((t, t), generator=gen) < 0.4) for t in lens]
    seen[0][:20] = False   # nothing ahead of the tree either
    words = torch.zeros((sum(lens), 8), dtype=torch.int64)
    row = 0
    for m in seen:
        for j in range(len(m)):
            for i in m[j].nonzero()[:, 0].tolist():
                words[row + j, i // 32] |= 1 << (i % 32)
        row += len(m)
    masks = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32).cuda()
    pos = torch.cat([torch.arange(t, dtype=torch.int32) + p for t, p in zip(lens, (0, 90))]).cuda()
    trees = [[j - 1 for j in range(t)] for t in lens]
    _, out, lse, _ = run_stored(c, trees, window=window, pos=pos, seen_of=lambda s: seen[s].cuda(), masks=masks)
    assert bool((out[:20] == 0).all()) and bool((lse[:20] == -math.inf).all())


def test_infinities_behind_the_tree():
    """Pairs of an earlier, longer tree behind this one's in its last page."""
    for D, g, T in ((128, 4, 12), (64, 2, 60), (128, 8, 40)):
        c = Case(1, g, D, [200], cap=600)
        bad = torch.full((90, 1, D), math.inf, dtype=torch.bfloat16, device="cuda")
        c.cache.append_chunk(0, bad, bad, [90])
        c.cache.append_chunk(0, bad[:0], bad[:0], [0], keep_lens=[200])
        run_stored(c, make_trees([T], near=4))


def test_a_long_cache_and_a_replayed_call():
    c = Case(2, 4, 128, [20000], cap=20200)
    trees = make_trees([64])
    q, out, lse, masks = run_stored(c, trees)
    fixed = torch.empty_like(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.tree_attn(0, q, [64], masks, out=fixed)
    for by in (1.0, -0.5):
        q.mul_(by)
        graph.replay()
        check(c, fixed, lse_of(c, q, masks), q, trees)
    assert c.status() == 0


def lse_of(c, q, masks):
    lse = torch.empty(q.shape[:2], device="cuda")
    c.cache.tree_attn(0, q, [q.shape[0]], masks, lse=lse)
    return lse


def test_a_tree_longer_than_its_segment_is_refused():
    c = Case(2, 4, 64, [8, 30])
    q, masks = c.chunk([9, 0])[2], torch.zeros((9, 8), dtype=torch.int32, device="cuda")
    with pytest.raises(binding.FkvError):
        c.cache.tree_attn(0, q, [9, 0], masks)
    assert c.status() == 0
