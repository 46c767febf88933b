"""Draft trees where a call can go wrong: full pools, replays over growing caches, other streams, many sequences, every kernel that may serve."""
import math

import pytest
import torch

import tree_ref
from paper_2602_03203_b200 import binding
from test_gpu_chunk import Case
from test_gpu_tree import check, extend, make_trees, packed, run_tree

pytestmark = pytest.mark.gpu


def pages(c):
    return sum(-(-len(s) // 16) for s in c.seqs) * c.Hkv


# ------------------------------------------------------------------ pages
@pytest.mark.parametrize("attend", [True, False])
def test_returned_pages_serve_the_growth_of_others(attend):
    """A full pool: sequence 0 gives its drafts back while sequence 1 grows by as many pages."""
    c = Case(2, 4, 64, [16, 16], num_pages=8, cap=64)
    trees = make_trees([32, 0])
    lens = [32, 0]
    k, v, q = c.chunk(lens)
    c.cache.append_tree(0, k, v, lens, c.cache.tree_masks(packed(trees), lens))
    extend(c, k, v, trees)
    assert c.cache.device_status() == (0, 0)
    trees, lens, keep = make_trees([0, 32], seed=3), [0, 32], [16, 16]
    k, v, q = c.chunk(lens)
    masks = c.cache.tree_masks(packed(trees), lens)
    if attend:
        lse = torch.empty(q.shape[:2], device="cuda")
        out = c.cache.append_tree_attn(0, k, v, q, lens, masks, keep_lens=keep, lse=lse)
    else:
        c.cache.append_tree(0, k, v, lens, masks, keep_lens=keep)
    extend(c, k, v, trees, keep)
    if attend:
        check(c, out, lse, q, trees)
    assert c.cache.device_status() == (0, 0)
    c.check_stored()


@pytest.mark.parametrize("attend", [True, False])
def test_without_pages_nothing_is_stored(attend):
    c = Case(2, 4, 64, [16, 20], num_pages=8, cap=96)   # six in use
    lens = [17, 13]                                      # two sequences that each need two more pages a head ... or one
    trees = make_trees(lens)
    k, v, q = c.chunk(lens)
    masks = c.cache.tree_masks(packed(trees), lens)
    if attend:
        c.cache.append_tree_attn(0, k, v, q, lens, masks)
    else:
        c.cache.append_tree(0, k, v, lens, masks)
    assert c.cache.device_status() == (binding.DEV_POOL_EXHAUSTED, 2)
    c.cache.sync_lengths()
    c.check_stored()
    run_tree(c, make_trees([0, 12], seed=1))             # and what fits is stored
    c.check_stored()


def test_pages_come_and_go_in_every_step():
    """Steps of trees of all sizes with their roll-backs: the pool's count is that of the lengths."""
    c = Case(3, 2, 64, [0, 15, 16, 100], cap=420)
    free0, used = c.cache.device_status()[1], pages(c)
    keep = [len(s) for s in c.seqs]
    for step, lens in enumerate([[1, 17, 33, 0], [64, 0, 3, 100], [5, 1, 1, 31], [256, 16, 0, 200], [2, 2, 2, 2]]):
        keep = [min(k + step, len(s)) for k, s in zip(keep, c.seqs)]
        run_tree(c, make_trees(lens, seed=step, near=5), keep=keep)
        c.check_stored()
        assert c.cache.device_status() == (0, free0 + used - pages(c))


# ------------------------------------------------------------------ replays
@pytest.mark.parametrize("window", [0, 300])
def test_replays_go_by_the_devices_lengths(window):
    """A captured call appends one more tree at every replay, behind whatever the cache holds by then.  (With a window the stored
    positions have to grow from pair to pair: chains.)"""
    c = Case(2, 4, 128, [30, 0, 500], cap=1400)
    lens = [20, 3, 9]
    trees = [[j - 1 for j in range(t)] for t in lens] if window else make_trees(lens)
    k, v, q = c.chunk(lens)
    masks = c.cache.tree_masks(packed(trees), lens)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    c.cache.append_tree_attn(0, k, v, q, lens, masks, window=window, out=out, lse=lse, keep_lens=[30, 0, 500])   # (once ahead of the capture)
    extend(c, k, v, trees)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.append_tree_attn(0, k, v, q, lens, masks, window=window, out=out, lse=lse)
    for step in range(25):
        k2, v2, q2 = c.chunk(lens)
        for a, b in ((k, k2), (v, v2), (q, q2)):
            a.copy_(b)
        graph.replay()
        extend(c, k2, v2, trees)
        if step % 8 == 7:
            check(c, out, lse, q2, trees, window)
    c.cache.sync_lengths()
    assert c.status() == 0
    c.check_stored()
    n = [len(s) for s in c.seqs]
    for _ in range(50):   # into the capacity (550 + 50 * 20 > 1408): a sequence that is full is left alone, the others go on
        graph.replay()
        n = [x + t if x + t <= 1408 else x for x, t in zip(n, lens)]
    c.cache.sync_lengths()
    assert c.status() == binding.DEV_CAPACITY and c.cache.lengths(0) == n


def test_replayed_attention_of_a_shorter_cache_is_left_out():
    c = Case(2, 4, 64, [40, 50])
    lens = [9, 4]
    trees = make_trees(lens)
    k, v, q = c.chunk(lens)
    masks = c.cache.tree_masks(packed(trees), lens)
    c.cache.append_tree(0, k, v, lens, masks)
    out = c.cache.tree_attn(0, q, lens, masks)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.tree_attn(0, q, lens, masks, out=out)
    c.cache.append_tree(0, k[:0], v[:0], [0, 0], masks[:0], keep_lens=[3, 54])
    graph.replay()
    assert c.status() == binding.DEV_BAD_INDEX
    extend(c, k, v, trees)
    lse = torch.full(q.shape[:2], 0.0, device="cuda")
    one = c.cache.tree_attn(0, q[9:].contiguous(), [0, 4], masks[9:].contiguous(), lse=lse[9:])
    assert torch.equal(one, out[9:])


# ------------------------------------------------------------------ streams, batches
def test_other_streams_and_two_caches_at_once():
    """Two caches on streams of their own, their steps in turn, against the same steps alone."""
    cases = [Case(2, 4, 128, [200, 31], seed=s) for s in (1, 2)]
    alone = [Case(2, 4, 128, [200, 31], seed=s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in cases]
    lens = [12, 7]
    steps = [[(make_trees(lens, seed=10 * i + s), c.chunk(lens)) for s in range(4)] for i, c in enumerate(cases)]
    torch.cuda.synchronize()
    got = [[], []]
    for s in range(4):
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                trees, (k, v, q) = steps[i][s]
                masks = c.cache.tree_masks(packed(trees), lens)
                got[i].append(c.cache.append_tree_attn(0, k, v, q, lens, masks))
                path = torch.tensor([list(range(6)), [0, -1, -1, -1, -1, -1]], dtype=torch.int32, device="cuda")
                c.cache.commit_tree(lens, path, torch.tensor([6, 1], dtype=torch.int32, device="cuda"))
                c.cache.sync_lengths()
    torch.cuda.synchronize()
    for i, c in enumerate(alone):
        for s in range(4):
            trees, (k, v, q) = steps[i][s]
            out = c.cache.append_tree_attn(0, k, v, q, lens, c.cache.tree_masks(packed(trees), lens))
            path = torch.tensor([list(range(6)), [0, -1, -1, -1, -1, -1]], dtype=torch.int32, device="cuda")
            c.cache.commit_tree(lens, path, torch.tensor([6, 1], dtype=torch.int32, device="cuda"))
            c.cache.sync_lengths()
            assert torch.equal(out, got[i][s])
        for x, y in zip(c.cache.export_chunk(0, c.cache.lengths(0)), cases[i].cache.export_chunk(0, cases[i].cache.lengths(0))):
            assert torch.equal(x, y)


@pytest.mark.parametrize("D,g,Hkv,batch,window", [(128, 4, 8, 19, 0), (64, 8, 4, 40, 300), (128, 1, 32, 5, 0), (128, 2, 1, 150, 0), (64, 4, 2, 74, 256)])
def test_as_many_sequences_as_the_card_has_room_for_and_more(D, g, Hkv, batch, window):
    stored = [(s * 53) % 333 for s in range(batch)]
    lens = [(s * 11) % 24 for s in range(batch)]
    c = Case(Hkv, g, D, stored, cap=400)
    run_tree(c, make_trees(lens), window)


@pytest.mark.parametrize("window", [0, 256])
@pytest.mark.parametrize("D,g,Hkv,batch", [(128, 4, 8, 64), (64, 8, 2, 256), (128, 1, 1, 256)])
def test_few_trees_in_many_places(D, g, Hkv, batch, window):
    """One launch whose blocks are those of the sequences that have a tree: two blocks and more of one, the last place, gaps."""
    lens = [0] * batch
    for s, n in ((0, 3), (batch // 3, 40), (batch - 1, 17)):
        lens[s] = n
    c = Case(Hkv, g, D, [700 if s % 5 == 0 or n else 1 for s, n in enumerate(lens)])
    before = c.cache.launch_count()
    run_tree(c, make_trees(lens), window=window, sinks=4 if window else 0)
    assert c.cache.launch_count() - before == 2   # masks, and everything else


@pytest.mark.parametrize("calls", ["append_tree", "append_tree_attn"])
def test_a_call_without_trees_rolls_back(calls):
    c = Case(2, 4, 64, [40, 0, 17])
    lens, keep = [0, 0, 0], [9, 0, 16]
    k, v, q = c.chunk(lens)
    masks = torch.empty((0, binding.TREE_WORDS), dtype=torch.int32, device="cuda")
    getattr(c.cache, calls)(0, k, v, *([q] if calls.endswith("attn") else []), lens, masks, keep_lens=keep)
    assert c.cache.lengths(0) == keep and c.status() == 0
    extend(c, k, v, [[], [], []], keep)
    run_tree(c, make_trees([5, 3, 0]))   # (and goes on from there)
    c.cache.commit_tree([0, 0, 0], torch.empty((3, 1), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"))
    c.cache.sync_lengths()
    assert c.cache.lengths(0) == [14, 3, 16] and c.status() == 0


@pytest.mark.parametrize("window,sinks", [(0, 0), (256, 4)])
@pytest.mark.parametrize("D,g", [(128, 4), (64, 7)])
def test_large_trees_of_large_batches(D, g, window, sinks):
    """More blocks of query rows than SMs: one and two tiles to an item, windows of later tokens that begin earlier."""
    lens = [100, 33, 0, 256, 64, 19, 20, 128, 90, 37, 18, 255]
    stored = [(s * 67) % 500 for s in range(len(lens))]
    c = Case(4, g, D, stored, gap=3, sinks=sinks, cap=800)
    run_tree(c, make_trees(lens, 3, near=6), window, sinks)


@pytest.mark.parametrize("rows", [1, 8, 63, 64, 65, 127, 128, 129, 256])
@pytest.mark.parametrize("D,g", [(128, 1), (64, 1)])
def test_numbers_of_rows_at_the_borders_of_the_forms(D, g, rows):
    for n in (0, 79, 80, 81, 95, 96, 97, 1000):
        c = Case(1, g, D, [n], seed=n, cap=n + 300)
        run_tree(c, [tree_ref.tree(min(rows, 256), 3, rows + n, near=4)])


@pytest.mark.parametrize("D,g,T", [(128, 4, 16), (64, 4, 16), (128, 8, 30)])
def test_far_references(D, g, T):
    """Scores that pass the first reference by far in later tiles, and some that never come near it: nothing overflows, nothing is lost."""
    c = Case(2, g, D, [700], cap=1000)
    trees = make_trees([T])
    k, v, q = c.chunk([T])
    for s, (at, by) in enumerate([(90, 30.0), (300, 80.0), (650, 160.0)]):   # keys along the queries' mean direction, ever longer
        for h in range(2):
            c.seqs[0].k[h][at] = (by * q[:, h * g].float().mean(0)).to(torch.bfloat16)
    c.cache.reset()
    c.cache.prefill(0, 0, torch.stack(c.seqs[0].k), torch.stack(c.seqs[0].v), torch.stack(c.seqs[0].f), c.seqs[0].pos[0].contiguous())
    masks = c.cache.tree_masks(packed(trees), [T])
    lse = torch.empty(q.shape[:2], device="cuda")
    out = c.cache.append_tree_attn(0, k, v, q, [T], masks, lse=lse)
    extend(c, k, v, trees)
    check(c, out, lse, q, trees)


@pytest.mark.parametrize("window", [0, 64])
def test_infinities_behind_the_pairs_and_outside_the_windows(window):
    """V rows of infinity in the last page behind the pairs that stay, and (windows) between sinks and window, reach no output."""
    for D, g, T in ((128, 4, 12), (64, 2, 60), (128, 8, 40)):
        c = Case(1, g, D, [200], sinks=4, cap=600)
        bad = c.rand(20, 1)
        c.cache.append_chunk(0, bad, torch.full_like(bad, math.inf), [20])
        if window:
            k, v, f, pos = c.cache.export_head(0, 0, 0)
            v[20:100] = math.inf
            c.seqs[0].v[0][20:100] = math.inf
            c.cache.reset()
            c.cache.prefill(0, 0, k[None].contiguous(), v[None].contiguous(), f[None].contiguous(), pos)
        run_tree(c, make_trees([T], near=4), window, 4, keep=[200])


def test_nan_queries_stay_in_their_rows():
    c = Case(2, 4, 128, [150], cap=400)
    for T in (10, 30):
        trees = make_trees([T])
        k, v, q = c.chunk([T])
        masks = c.cache.tree_masks(packed(trees), [T])
        a = c.cache.append_tree_attn(0, k, v, q, [T], masks, keep_lens=[150])
        q2 = q.clone()
        q2[3, 5] = math.nan
        lse = torch.empty(q.shape[:2], device="cuda")
        b = c.cache.append_tree_attn(0, k, v, q2, [T], masks, keep_lens=[150], lse=lse)
        assert bool(torch.isnan(b[3, 5].float()).all()) and bool(torch.isnan(lse[3, 5]))
        a[3, 5] = b[3, 5] = 0
        assert torch.equal(a, b)


def test_results_do_not_depend_on_the_run():
    c = Case(4, 4, 128, [3000, 200, 0], cap=3400)
    lens = [40, 13, 5]
    trees = make_trees(lens)
    k, v, q = c.chunk(lens)
    masks = c.cache.tree_masks(packed(trees), lens)
    first = None
    for _ in range(20):
        lse = torch.empty(q.shape[:2], device="cuda")
        out = c.cache.append_tree_attn(0, k, v, q, lens, masks, keep_lens=[3000, 200, 0], lse=lse)
        if first is None:
            first = (out, lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
