"""Draft trees over the paged cache: masks, storing, attention, the accepted path moved together, read-out."""
import math

import pytest
import torch

import chunk_ref as ref
import tree_ref
from paper_2602_03203_b200 import binding
from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


def make_trees(lens, fan=3, seed=0, near=1000):
    return [tree_ref.tree(t, fan, seed + 17 * s, near) for s, t in enumerate(lens)]


def packed(trees):
    return torch.tensor([p for t in trees for p in t], dtype=torch.int32, device="cuda")


def depths(parents):
    return torch.tensor([tree_ref.depth(parents, j) for j in range(len(parents))], dtype=torch.int32, device="cuda")


def extend(c, k, v, trees, keep=None, pos=None):
    """The tree's pairs in the plain cache: positions by depth, or given ones."""
    row = 0
    for s, parents in enumerate(trees):
        t = len(parents)
        if t or keep is not None:
            seq, part = c.seqs[s], slice(row, row + t)
            n = len(seq) if keep is None else keep[s]
            for h in range(c.Hkv):
                first = int(seq.pos[h][n - 1]) + 1 if n else 0
                p = first + depths(parents) if pos is None else pos[part]
                seq.k[h] = torch.cat([seq.k[h][:n], k[part, h]])
                seq.v[h] = torch.cat([seq.v[h][:n], v[part, h]])
                seq.f[h] = torch.cat([seq.f[h][:n], seq.f[h].new_zeros((t, seq.f[h].shape[1]))])
                seq.pos[h] = torch.cat([seq.pos[h][:n], p])
        row += t


def check(c, out, lse, q, trees, window=0, sinks=0, scale=None, seen_of=None):
    """seen_of(s) -> [t][t] bool: the nodes that every node sees (default: ancestors and itself)."""
    scale = scale or c.D ** -0.5
    row = 0
    for s, parents in enumerate(trees):
        t, seq = len(parents), c.seqs[s]
        if not t:
            continue
        own = torch.zeros((t, t), dtype=torch.bool, device="cuda")
        if seen_of is None:
            for j in range(t):
                own[j, list(tree_ref.path_up(parents, j))] = True
        else:
            own = seen_of(s)
        for h in range(c.Hkv):
            n = seq.k[h].shape[0]
            base = n - t
            ok = torch.zeros((t, n), dtype=torch.bool, device="cuda")
            ok[:, base:] = own
            here, x = seq.pos[h][base:].long(), seq.pos[h][:base].long()
            ok[:, :base] = ((here[:, None] - x < window) | (x < sinks)) if window else True
            for j in range(c.g):
                hq = h * c.g + j
                o, l, _, tol, ltol = ref.attend(q[row:row + t, hq], seq.k[h], seq.v[h], ok, scale)
                some = ok.any(1)
                o, l = torch.where(some[:, None], o, torch.zeros_like(o)), torch.where(some, l, torch.full_like(l, -math.inf))
                d = (out[row:row + t, hq].double() - o).abs()
                assert bool((d <= tol.nan_to_num(nan=1e-30)).all()), (s, h, j, float((d / tol).max()))
                got = lse[row:row + t, hq].double()
                assert torch.equal(got[~some], l[~some])
                d = (got[some] - l[some]).abs()
                assert bool((d <= ltol[some]).all()), (s, h, j, float((d / ltol[some]).max()))
        row += t


def run_tree(c, trees, window=0, sinks=0, keep=None, pos=None, scale=0.0):
    lens = [len(t) for t in trees]
    k, v, q = c.chunk(lens)
    masks = c.cache.tree_masks(packed(trees), lens)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    out = c.cache.append_tree_attn(0, k, v, q, lens, masks, pos=pos, keep_lens=keep, window=window, sinks=sinks, lse=lse, scale=scale)
    extend(c, k, v, trees, keep, pos)
    assert c.status() == 0
    check(c, out, lse, q, trees, window, sinks, scale or None)
    return k, v, q, out, lse, masks


# ------------------------------------------------------------------ masks
@pytest.mark.parametrize("lens,near", [([1, 2, 0, 33], 1000), ([256, 255, 31, 32], 2), ([256, 0, 0, 64], 1), ([0, 0, 0, 97], 1000)])
def test_masks_name_the_ancestors(lens, near):
    c = Case(1, 1, 64, [0, 0, 0, 0])
    trees = make_trees(lens, 2 if near < 1000 else 6, near=near)
    out = torch.full((sum(lens) + 1, 8), -7, dtype=torch.int32, device="cuda")
    c.cache.tree_masks(packed(trees), lens, out=out[:-1])
    want = [tree_ref.mask_words(t) for t in trees if t]
    got = out[:-1].cpu().numpy().astype("int64") & 0xFFFFFFFF
    row = 0
    for w in want:
        assert (got[row:row + len(w)] == w).all()
        row += len(w)
    assert bool((out[-1] == -7).all()) and c.status() == 0


def test_masks_of_several_roots_and_of_bad_parents():
    c = Case(1, 1, 64, [0])
    parents = torch.tensor([-1, -1, 0, 1, -1, 3], dtype=torch.int32, device="cuda")
    got = c.cache.tree_masks(parents, [6]).cpu()[:, 0].tolist()
    assert got == [1, 2, 5, 10, 16, 42] and c.status() == 0
    parents = torch.tensor([0, 5, -2, 2 ** 30, 1, 4], dtype=torch.int32, device="cuda")   # four of them are no parents
    got = c.cache.tree_masks(parents, [6]).cpu()[:, 0].tolist()
    assert got == [1, 2, 4, 8, 2 + 16, 2 + 16 + 32] and c.status() == binding.DEV_BAD_INDEX


# ------------------------------------------------------------------ storing
@pytest.mark.parametrize("D,g,Hkv", [(64, 4, 2), (128, 7, 3), (128, 1, 1)])
def test_append_tree_stores_by_depth_and_rolls_back(D, g, Hkv):
    c = Case(Hkv, g, D, [0, 5, 16, 31, 40])
    for lens, keep in [([3, 11, 16, 1, 0], None), ([40, 1, 2, 17, 15], [0, 5, 0, 31, 33]), ([1, 1, 1, 1, 1], [3, 6, 2, 31, 33])]:
        trees = make_trees(lens, seed=sum(lens))
        k, v, _ = c.chunk(lens)
        masks = c.cache.tree_masks(packed(trees), lens)
        c.cache.append_tree(0, k, v, lens, masks, keep_lens=keep)
        extend(c, k, v, trees, keep)
        assert c.status() == 0
        c.check_stored()


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("D,g,Hkv,stored,lens", [
    (128, 4, 2, [100], [16]), (128, 4, 2, [0], [16]), (128, 4, 2, [1], [1]), (64, 8, 1, [15, 0, 300], [16, 33, 1]),
    (128, 7, 2, [333, 5, 0, 80], [64, 0, 19, 256]), (64, 1, 3, [79, 80, 81], [256, 255, 129]), (128, 2, 1, [700], [200]),
    (64, 3, 2, [95, 96, 97, 1], [31, 32, 33, 96]), (128, 8, 1, [1000, 17], [256, 100]), (128, 5, 4, [2500], [48])])
def test_tree_attention(D, g, Hkv, stored, lens):
    for near, fan in ((1000, 3), (2, 2)):
        c = Case(Hkv, g, D, stored, seed=D + g, cap=max(stored) + 700)
        run_tree(c, make_trees(lens, fan, near=near))


@pytest.mark.parametrize("window,sinks", [(256, 0), (256, 4), (300, 64), (512, 1), (4096, 16)])
@pytest.mark.parametrize("D,g", [(128, 8), (64, 3)])
def test_tree_attention_with_windows(D, g, window, sinks):
    for gap in (1, 4):
        c = Case(2, g, D, [1500, 90, 0, 257], gap=gap, sinks=64, seed=window)
        run_tree(c, make_trees([200, 40, 17, 256], 2, near=4), window, sinks)


def test_windows_as_short_as_the_tree():
    c = Case(2, 4, 128, [500, 3, 40], gap=2, sinks=8)
    run_tree(c, make_trees([20, 7, 1], 2, near=3), 20, 5)
    c = Case(1, 4, 64, [50], gap=2)
    run_tree(c, [[-1]], 1, 0)   # the node alone


def test_positions_of_pruned_and_far_caches():
    c = Case(2, 4, 128, [600], gap=40, sinks=8)
    last = int(c.seqs[0].pos[0][-1])
    parents = tree_ref.tree(30, 3, 5)
    pos = last + 5 + 3 * depths(parents)   # given positions with gaps of their own
    run_tree(c, [parents], window=400, sinks=4, pos=pos.to(torch.int32))


def test_scale_and_rows_behind_the_last_node():
    c = Case(2, 4, 128, [60, 0])
    trees = make_trees([9, 5])
    lens = [9, 5]
    k, v, q = c.chunk(lens)
    masks = c.cache.tree_masks(packed(trees), lens)
    out = torch.full((20, 8, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((20, 8), 3.0, device="cuda")
    c.cache.append_tree_attn(0, k, v, q, lens, masks, out=out[:14], lse=lse[:14], scale=0.3)
    extend(c, k, v, trees)
    check(c, out, lse, q, trees, scale=0.3)
    assert bool((out[14:] == 3).all()) and bool((lse[14:] == 3).all())


def test_chain_equals_a_chunk():
    """A tree without branches is a chunk: both calls, which may be different kernels, are within the bounds of the 64-bit form of
    the one, and store the same."""
    lens = [37, 5]
    chain = [[j - 1 for j in range(t)] for t in lens]
    for window in (512, 0):
        a, b = Case(2, 4, 128, [300, 17]), Case(2, 4, 128, [300, 17])
        k, v, q = a.chunk(lens)
        la, lb = torch.empty(q.shape[:2], device="cuda"), torch.empty(q.shape[:2], device="cuda")
        masks = a.cache.tree_masks(packed(chain), lens)
        x = a.cache.append_tree_attn(0, k, v, q, lens, masks, window=window, lse=la)
        y = b.cache.append_chunk_attn(0, k, v, q, lens, window=window, lse=lb)
        extend(a, k, v, chain)
        check(a, x, la, q, chain, window)
        check(a, y, lb, q, chain, window)
        for s in range(2):
            for m, n in zip(a.cache.export_head(0, s, 1), b.cache.export_head(0, s, 1)):
                assert torch.equal(m, n)


def test_masks_of_other_kinds_and_rows_that_see_nothing():
    c = Case(2, 4, 128, [0, 90])
    lens = [70, 40]
    gen = torch.Generator().manual_seed(3)
    seen = [torch.tril(torch.rand((t, t), generator=gen) < 0.4) for t in lens]
    seen[0][:20] = False   # nothing ahead of the tree either: zeros, log-sum-exp -inf
    words = torch.zeros((sum(lens), 8), dtype=torch.int64)
    row = 0
    for m in seen:
        for j in range(len(m)):
            for i in m[j].nonzero()[:, 0].tolist():
                words[row + j, i // 32] |= 1 << (i % 32)
        row += len(m)
    words[5, 1] |= 1 << 8    # a node behind, and one that is not there: not seen all the same
    words[5, 7] |= 1 << 31
    masks = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32).cuda()
    k, v, q = c.chunk(lens)
    pos = torch.cat([torch.arange(t, dtype=torch.int32) + p for t, p in zip(lens, (0, 90))]).cuda()
    lse = torch.empty(q.shape[:2], device="cuda")
    out = c.cache.append_tree_attn(0, k, v, q, lens, masks, pos=pos, lse=lse)
    trees = [[j - 1 for j in range(t)] for t in lens]
    extend(c, k, v, trees, pos=pos)
    check(c, out, lse, q, trees, seen_of=lambda s: seen[s].cuda())
    assert bool((out[:20] == 0).all()) and bool(torch.isinf(lse[:20]).all())


def test_infinite_keys_of_unseen_nodes():
    """A sibling's key of infinity or NaN stays out of the scores of those that do not see it."""
    c = Case(1, 4, 128, [50])
    parents = [-1, 0, 0, 1, 2, 1, 2]
    k, v, q = c.chunk([7])
    bad = k.clone()
    bad[2] = math.inf
    bad[4] = math.nan
    masks = c.cache.tree_masks(packed([parents]), [7])
    lse = [torch.empty(q.shape[:2], device="cuda") for _ in range(2)]
    a = c.cache.append_tree_attn(0, k, v, q, [7], masks, keep_lens=[50], lse=lse[0])
    b = c.cache.append_tree_attn(0, bad, v, q, [7], masks, keep_lens=[50], lse=lse[1])
    free = [0, 1, 3, 5]
    assert torch.equal(a[free], b[free]) and torch.equal(lse[0][free], lse[1][free])
    assert bool(torch.isnan(b[4].float()).all())


def test_rejected_nodes_leave_no_trace():
    """Infinities in the pairs of a tree that was dropped do not reach the next one's output."""
    c = Case(2, 4, 128, [37])
    k, v, q = c.chunk([30])
    masks = c.cache.tree_masks(packed([tree_ref.tree(30, 3, 1)]), [30])
    c.cache.append_tree(0, k, torch.full_like(v, math.inf), [30], masks)
    run_tree(c, [tree_ref.tree(6, 3, 2)], keep=[37])


@pytest.mark.parametrize("n", [30000])
def test_long_cache(n):
    c = Case(2, 4, 128, [n], cap=n + 300)
    run_tree(c, [tree_ref.tree(64, 4, 1)])


def test_a_batch_of_many_sequences():
    stored = [(s * 37) % 200 for s in range(256)]
    lens = [0 if s % 3 == 1 else 1 + s % 9 for s in range(256)]
    c = Case(1, 2, 64, stored, cap=260)
    run_tree(c, make_trees(lens))


# ------------------------------------------------------------------ the accepted path
def commit(c, trees, paths):
    """The plain form: of every tree the pairs on the path stay."""
    for s, parents in enumerate(trees):
        if not parents:
            continue
        seq = c.seqs[s]
        base = len(seq) - len(parents)
        idx = torch.tensor(list(range(base)) + [base + i for i in paths[s]], dtype=torch.long, device="cuda")
        for h in range(c.Hkv):
            seq.k[h], seq.v[h], seq.f[h], seq.pos[h] = seq.k[h][idx], seq.v[h][idx], seq.f[h][idx], seq.pos[h][idx]


def path_tensors(paths, width):
    path = torch.full((len(paths), width), -1, dtype=torch.int32)
    for s, p in enumerate(paths):
        path[s, :len(p)] = torch.tensor(p, dtype=torch.int32)
    return path.cuda(), torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("D,g,Hkv", [(64, 4, 2), (128, 7, 3), (128, 8, 1), (64, 1, 32)])
@pytest.mark.parametrize("kind", ["leaf", "root", "none", "all", "far"])
def test_commit_moves_the_path_together(D, g, Hkv, kind):
    stored, lens = [0, 5, 16, 31, 40, 7], [30, 1, 100, 17, 0, 256]
    c = Case(Hkv, g, D, stored, cap=320)
    trees = make_trees(lens, 3, near=5)
    k, v, _ = c.chunk(lens)
    masks = c.cache.tree_masks(packed(trees), lens)
    c.cache.append_tree(0, k, v, lens, masks)
    extend(c, k, v, trees)
    feats = [torch.rand((Hkv, len(s), 6 * g), device="cuda") for s in c.seqs]
    for s, f in enumerate(feats):   # features move with their pairs
        if len(c.seqs[s]):
            c.cache.set_features(0, s, f)
            c.seqs[s].f = [f[h] for h in range(Hkv)]
    paths = {"leaf": [sorted(tree_ref.path_up(t, len(t) - 1)) for t in trees], "root": [[0] if t else [] for t in trees],
             "none": [[] for t in trees], "all": [list(range(len(t))) for t in trees],
             "far": [list(range(len(t) // 2, len(t))) for t in trees]}[kind]
    before = sum(-(-len(s) // 16) for s in c.seqs) * Hkv
    free0 = c.cache.device_status()[1]
    c.cache.commit_tree(lens, *path_tensors(paths, 256))
    commit(c, trees, paths)
    c.cache.sync_lengths()
    status, free = c.cache.device_status()
    after = sum(-(-len(s) // 16) for s in c.seqs) * Hkv
    assert status == 0 and free == free0 + before - after
    c.check_stored()
    run_tree(c, make_trees([5, 0, 9, 33, 2, 1], seed=9))   # and the cache goes on
    c.cache.reset()
    assert c.cache.device_status()[1] == free0 + before


def test_commit_refuses_paths_that_are_none():
    c = Case(2, 4, 64, [20, 30, 40, 50, 60])
    lens = [6, 6, 6, 6, 6]
    trees = make_trees(lens)
    k, v, _ = c.chunk(lens)
    c.cache.append_tree(0, k, v, lens, c.cache.tree_masks(packed(trees), lens))
    extend(c, k, v, trees)
    paths = [[0, 2, 1], [0, 6], [-1, 2], [1, 3], [2, 2]]
    path, n = path_tensors(paths, 6)
    c.cache.commit_tree(lens, path, n)
    trees[0] = trees[1] = trees[2] = trees[4] = []
    commit(c, trees, paths)
    c.cache.sync_lengths()
    assert c.status() == binding.DEV_BAD_INDEX
    c.check_stored()
    path, n = path_tensors([[0]] * 5, 6)
    for bad in (-1, 7, 2 ** 30):
        n[1] = bad
        c.cache.commit_tree([0, 6, 0, 0, 0], path, n)
        assert c.status() == binding.DEV_BAD_INDEX
    c.cache.sync_lengths()
    c.check_stored()


def test_commit_of_several_layers_and_of_one():
    cache = binding.Cache(3, 2, 2, 64, 2, 16, 200)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda n: torch.randn((n, 2, 64), generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    lens, trees = [20, 12], make_trees([20, 12])
    masks, given = cache.tree_masks(packed(trees), lens), []
    for layer, m in enumerate((18, 40, 7)):
        cache.append_chunk(layer, rand(2 * m), rand(2 * m), [m, m])
        given.append((rand(32), rand(32)))
        cache.append_tree(layer, *given[-1], lens, masks)
    path, n = path_tensors([[0, 3, 11], [0, 1]], 20)
    cache.commit_tree(lens, path, n, layer=1)
    cache.sync_lengths()
    assert [cache.lengths(i) for i in range(3)] == [[38, 30], [43, 42], [27, 19]]
    for layer in (0, 2):
        cache.commit_tree(lens, path, n, layer=layer)
    cache.sync_lengths()
    assert [cache.lengths(i) for i in range(3)] == [[21, 20], [43, 42], [10, 9]]
    rows = [0, 3, 11, 20, 21]
    for layer in range(3):
        k, v, f, pos = cache.export_chunk(layer, [3, 2])
        assert torch.equal(k, given[layer][0][rows]) and torch.equal(v, given[layer][1][rows])
        assert bool((f == 0).all()) and pos.shape == (5, 2)


# ------------------------------------------------------------------ read-out
@pytest.mark.parametrize("lens", [[0, 5, 16, 31, 40], [0, 0, 1, 31, 17], [0, 0, 0, 0, 0]])
def test_export_chunk_is_what_was_stored(lens):
    c = Case(3, 7, 128, [0, 5, 16, 31, 40], gap=3)
    k, v, f, pos = c.cache.export_chunk(0, lens)
    row = 0
    for s, t in enumerate(lens):
        for h in range(3 if t else 0):
            seq, part = c.seqs[s], slice(row, row + t)
            assert torch.equal(k[part, h], seq.k[h][-t:]) and torch.equal(v[part, h], seq.v[h][-t:])
            assert torch.equal(f[part, h], seq.f[h][-t:]) and torch.equal(pos[part, h], seq.pos[h][-t:])
        row += t
    some = torch.full((sum(lens), 3), -1, dtype=torch.int32, device="cuda")
    c.cache.export_chunk(0, lens, (None, None, None, some))
    assert torch.equal(some, pos) and c.status() == 0
    with pytest.raises(binding.FkvError):
        c.cache.export_chunk(0, [1, 0, 0, 0, 0])


# ------------------------------------------------------------------ refusals
def test_refusals():
    c = Case(2, 4, 64, [20, 30], cap=400)
    lens, trees = [4, 3], make_trees([4, 3])
    k, v, q = c.chunk(lens)
    masks = c.cache.tree_masks(packed(trees), lens)
    calls = [lambda: c.cache.tree_attn(0, q, lens, masks, window=3),                # a window that does not hold the tree
             lambda: c.cache.append_tree_attn(0, k, v, q, lens, masks, window=3),
             lambda: c.cache.append_tree_attn(0, k, v, q, lens, masks, window=-1),
             lambda: c.cache.append_tree(1, k, v, lens, masks),                      # a layer that is none
             lambda: c.cache.append_tree(0, k, v, lens, masks, keep_lens=[21, 30]),
             lambda: c.cache.append_tree_attn(0, k, v, q, lens, masks, scale=1e-40),
             lambda: c.cache.commit_tree(lens, *path_tensors([[0], [0]], 4), layer=1),
             lambda: c.cache.commit_tree([31, 0], *path_tensors([[0], [0]], 4))]
    for call in calls:
        with pytest.raises(binding.FkvError):
            call()
    n = 257
    big = torch.zeros((n, 8), dtype=torch.int32, device="cuda")
    kk, vv, qq = c.chunk([n, 0])
    for call in (lambda: c.cache.append_tree(0, kk, vv, [n, 0], big), lambda: c.cache.tree_masks(big[:, 0].contiguous(), [n, 0]),
                 lambda: c.cache.append_tree_attn(0, kk, vv, qq, [n, 0], big)):
        with pytest.raises(binding.FkvError):
            call()
    for call in (lambda: c.cache.append_tree(0, k, v, lens, masks[:-1]), lambda: c.cache.tree_attn(0, q[:-1], lens, masks),
                 lambda: c.cache.tree_masks(packed(trees), [4, 2]), lambda: c.cache.append_tree(0, k, v, lens, masks.float()),
                 lambda: c.cache.append_tree(0, k, v, lens, masks.cpu()), lambda: c.cache.tree_attn(0, q, [4, 3, 1], masks)):
        with pytest.raises((ValueError, binding.FkvError)):
            call()
    c.check_stored()
    assert c.status() == 0
