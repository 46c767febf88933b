"""Positions of nodes whose masks are the caller's own: as many behind the last pair as the mask names nodes ahead of the node's own, and one."""
import pytest
import torch

from test_gpu_chunk import Case
from test_gpu_tree import check, extend

pytestmark = pytest.mark.gpu


def words_of(seen):
    """[t][t] bool -> [t][8] int64, bit i of row j: j names i."""
    words = torch.zeros((len(seen), 8), dtype=torch.int64)
    for j in range(len(seen)):
        for i in seen[j].nonzero()[:, 0].tolist():
            words[j, i // 32] |= 1 << (i % 32)
    return words


def own_masks(lens, seed):
    """Random sets of nodes: some name nothing, some not themselves, some nodes behind them or beyond the tree."""
    gen = torch.Generator().manual_seed(seed)
    named, words = [], []
    for t in lens:
        m = torch.rand((t, t), generator=gen) < 0.3
        m[::5] = False
        m[1::7] = True
        named.append(m)
        w = words_of(m)
        w[::3, 7] |= 1 << 31
        m[::3, 255:] = True   # (a tree of 256 has that node, and it may be the row's own)
        words.append(w)
    words = torch.cat(words)
    return named, torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32).cuda()


@pytest.mark.parametrize("D,g,stored,lens", [(128, 4, [0, 90, 33], [70, 40, 1]), (64, 2, [0, 16, 200], [9, 100, 33]),
                                             (128, 8, [300] * 24, [12] * 24), (64, 8, [5, 700], [256, 200])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (256, 4)])
@pytest.mark.parametrize("attend", [True, False])
def test_positions_follow_the_masks(D, g, stored, lens, window, sinks, attend):
    c = Case(2, g, D, stored, gap=3, cap=1000)
    named, masks = own_masks(lens, sum(lens))
    k, v, q = c.chunk(lens)
    pos = torch.cat([(int(s.pos[0][-1]) if len(s) else -1) + 1 + torch.tril(m, -1).sum(1) for s, m in zip(c.seqs, named)]).to(torch.int32).cuda()
    if attend:
        lse = torch.empty(q.shape[:2], device="cuda")
        out = c.cache.append_tree_attn(0, k, v, q, lens, masks, window=window, sinks=sinks, lse=lse)
    else:
        c.cache.append_tree(0, k, v, lens, masks)
    trees = [[j - 1 for j in range(t)] for t in lens]
    extend(c, k, v, trees, pos=pos)
    assert c.status() == 0
    c.check_stored()
    if attend:
        check(c, out, lse, q, trees, window, sinks, seen_of=lambda s: torch.tril(named[s]).cuda())
