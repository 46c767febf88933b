"""Features from a chunk's queries: what is masked counts exactly zero, and a NaN stays one."""
import math

import pytest
import torch

import chunk_ref as ref
from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


def stored_chunk(c, lens, window, sinks):
    """A chunk stored and attended from: its queries, log-sum-exp and the features ahead of the call under test."""
    k, v, q = c.chunk(lens)
    lse = torch.empty(q.shape[:2], device="cuda")
    c.cache.append_chunk_attn(0, k, v, q, lens, window=window, sinks=sinks, lse=lse)
    c.extend(k, v, lens)
    return q, lse, [c.cache.export_features(0, s) for s in range(c.batch)]


@pytest.mark.parametrize("D,g,lens", [(128, 4, [150, 40]), (64, 3, [300, 1]), (128, 1, [9, 128])])
@pytest.mark.parametrize("window,sinks,gap", [(1, 0, 1), (20, 4, 1), (77, 0, 2), (100, 17, 1), (130, 3, 3)])
def test_pairs_outside_the_windows_hold_exact_zeros(D, g, lens, window, sinks, gap):
    c = Case(2, g, D, [700, 333], gap=gap)
    q, lse, old = stored_chunk(c, lens, window, sinks)
    c.cache.chunk_features(0, q, lse, lens, window=window, sinks=sinks)
    hidden = 0
    for s, t in enumerate(lens):
        got = c.cache.export_features(0, s).unflatten(2, (g, 6))
        was = old[s].unflatten(2, (g, 6))
        for h in range(2):
            pos = c.seqs[s].pos[h]
            n = pos.shape[0]
            ok = ref.seen(pos, torch.arange(n - t, n, device="cuda"), pos[n - t:], window, sinks)
            for i, w in enumerate((8, 16, 32, t)):
                assert bool((got[h][~ok[-w:].any(0)][:, :, i] == 0).all()), (s, h, i)
            none = ~ok.any(0)
            hidden += int(none.sum())
            assert torch.equal(got[h][none][:, :, 4], was[h][none][:, :, 4])
            assert torch.equal(got[h][none][:, :, 5], was[h][none][:, :, 5] * 0.9)   # (one rounding on either side)
    assert hidden > 300 and c.status() == 0


def test_eviction_after_a_windowed_prompt_keeps_what_the_definition_says():
    """More budget than pairs that a query has seen: the others tie at zero, and the lowest slots of them stay."""
    n, t, window, sinks, budget, recent = 600, 50, 90, 4, 300, 16
    c = Case(2, 2, 64, [n], budget=budget, recent_keep=recent)
    c.cache.set_features(0, 0, torch.zeros((2, n, 12), device="cuda"))
    c.cache.evict_by_feature(0, 0)   # (by zeros: the first 284 pairs and the last 16 stay)
    for h in range(2):
        k, v, f, pos = c.cache.export_head(0, 0, h)
        assert torch.equal(pos.long(), torch.cat([torch.arange(284), torch.arange(584, 600)]).cuda())
        c.seqs[0].k[h], c.seqs[0].v[h], c.seqs[0].f[h], c.seqs[0].pos[h] = k, v, f, pos
    q, lse, _ = stored_chunk(c, [t], window, sinks)
    c.cache.chunk_features(0, q, lse, [t], window=window, sinks=sinks)
    c.cache.evict_by_feature(4, 0)
    for h in range(2):
        pos = c.seqs[0].pos[h]
        m = pos.shape[0]
        ok = ref.seen(pos, torch.arange(m - t, m, device="cuda"), pos[m - t:], window, sinks).any(0)
        must = ok.clone()
        must[m - recent:] = True
        rest = torch.nonzero(~must)[:, 0][: budget - int(must.sum())]
        kept = torch.sort(torch.cat([torch.nonzero(must)[:, 0], rest])).values
        assert torch.equal(c.cache.export_head(0, 0, h)[3], pos[kept])


@pytest.mark.parametrize("row", [*range(8), 64, 121])
@pytest.mark.parametrize("window,sinks", [(0, 0), (260, 4)])
def test_a_query_of_nan_shows_in_every_pair_that_it_sees(row, window, sinks):
    T, g = 128, 2
    c = Case(1, g, 64, [500])
    k, v, q = c.chunk([T])
    q[row, 1, 5] = math.nan   # the second head of the group only
    lse = torch.empty(q.shape[:2], device="cuda")
    c.cache.append_chunk_attn(0, k, v, q, [T], window=window, sinks=sinks, lse=lse)
    c.extend(k, v, [T])
    assert torch.equal(torch.isnan(lse).nonzero(), torch.tensor([[row, 1]], device="cuda"))
    pos = c.seqs[0].pos[0]
    ok = ref.seen(pos, torch.arange(500, 628, device="cuda"), pos[500:], window, sinks)
    for given in (lse, lse.nan_to_num(nan=3.0)):   # NaN from the log-sum-exp, and from the scores alone
        c.cache.set_features(0, 0, torch.zeros((1, 628, 12), device="cuda"))
        c.cache.chunk_features(0, q, given.contiguous(), [T], window=window, sinks=sinks)
        got = c.cache.export_features(0, 0)[0].unflatten(1, (g, 6))
        assert bool(torch.isfinite(got[:, 0]).all())
        for i, w in enumerate((8, 16, 32, T, T, T)):
            sees = ok[row] & (row >= T - w)
            assert torch.equal(torch.isnan(got[:, 1, i]), sees), (i, int(torch.isnan(got[:, 1, i]).sum()), int(sees.sum()))
