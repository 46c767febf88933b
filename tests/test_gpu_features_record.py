"""Decode queries on record when a chunk's queries move the features on: they came first, and count first."""
import pytest
import torch

import chunk_ref as ref
import oracle
from test_gpu_chunk import Case
from test_gpu_chunk_features import check_features
from util import npf

pytestmark = pytest.mark.gpu
SNAPKV, CUM_SUM = 0, 4


def decode(cs, tokens, seq_mask=0):
    for k, v, q in tokens:
        for c in cs:
            c.cache.append_decode_attn(0, k, v, q, seq_mask=seq_mask)
            for s in range(c.batch):
                if not seq_mask or seq_mask >> s & 1:
                    c.seqs[s].extend(k[s:s + 1], v[s:s + 1])


@pytest.mark.parametrize("steps", [1, 5, 16, 21])   # the record holds the last 16
@pytest.mark.parametrize("D,g", [(64, 2), (128, 4)])
def test_the_record_is_a_chunk_of_its_own_ahead_of_the_chunk(steps, D, g):
    # `a` takes the decode queries, then the chunk; `b` shows what the decode queries alone make of the features.
    a, b = (Case(2, g, D, [90, 40, 33], feature_window=16, cap=400) for _ in range(2))
    tokens = [(a.rand(3, 2), a.rand(3, 2), a.rand(3, 2 * g)) for _ in range(steps)]
    decode((a, b), tokens)
    b.cache.update_features(0)
    lens = [70, 0, 5]
    k, v, q = a.chunk(lens)
    lse = torch.empty(q.shape[:2], device="cuda")
    a.cache.append_chunk_attn(0, k, v, q, lens, lse=lse)
    old = [a.cache.export_features(0, s) for s in range(3)]
    a.extend(k, v, lens)
    for s in (0, 2):   # the decode queries saw none of the chunk's pairs
        moved = b.cache.export_features(0, s)
        assert not torch.equal(moved, old[s][:, :moved.shape[1]])
        old[s] = torch.cat([moved, torch.zeros_like(old[s][:, moved.shape[1]:])], 1)
    a.cache.chunk_features(0, q, lse, lens)
    check_features(a, q, lens, old)   # (sequence 1 has no tokens in the chunk: untouched)
    # They have left the record: nothing is applied a second time.  Sequence 1's are still there.
    now = [a.cache.export_features(0, s) for s in range(3)]
    a.cache.update_features(0)
    for s in (0, 2):
        assert torch.equal(a.cache.export_features(0, s), now[s])
    assert torch.equal(a.cache.export_features(0, 1), b.cache.export_features(0, 1))
    # Later decode queries begin a record of their own.
    decode((a,), [(a.rand(3, 2), a.rand(3, 2), a.rand(3, 2 * g)) for _ in range(3)])
    a.cache.update_features(0)
    for s in (0, 2):
        f = a.cache.export_features(0, s).unflatten(2, (g, 6))
        # three probabilities per query head: over all pairs the windows' sums are 3 / w and 3 / 3
        total = f[..., :4].double().sum(1)
        want = torch.tensor([3 / 8, 3 / 16, 3 / 32, 1.0], dtype=torch.float64, device="cuda")
        assert bool(((total - want).abs() < 1e-4).all())
    assert a.status() == 0


@pytest.mark.parametrize("column", [SNAPKV, CUM_SUM])
def test_eviction_after_decode_steps_and_a_chunk(column):
    c = Case(2, 2, 64, [120], feature_window=32, cap=400, budget=64, recent_keep=8)
    decode((c,), [(c.rand(1, 2), c.rand(1, 2), c.rand(1, 4)) for _ in range(9)])
    k, v, q = c.chunk([60])
    lse = torch.empty(q.shape[:2], device="cuda")
    c.cache.append_chunk_attn(0, k, v, q, [60], lse=lse)
    c.cache.chunk_features(0, q, lse, [60])
    feats = c.cache.export_features(0, 0)
    c.extend(k, v, [60])
    c.cache.evict_by_feature(column, 0)
    for h in range(2):
        kept = torch.from_numpy(oracle.select(oracle.score_feature(npf(feats[h]), 2, column), 64, 8)).long().cuda()
        pos = c.cache.export_head(0, 0, h)[3]
        assert torch.equal(pos, c.seqs[0].pos[h][kept])
        if column == SNAPKV:   # the window is the chunk's: its last 8 queries by the definition
            n = c.seqs[0].k[h].shape[0]
            ok = torch.ones((8, n), dtype=torch.bool, device="cuda").tril(n - 8)
            for j in range(2):
                _, _, p, _, err = ref.attend(q[-8:, 2 * h + j], c.seqs[0].k[h], c.seqs[0].v[h], ok, 64 ** -0.5)
                w8 = p.sum(0) / 8
                assert bool(((feats[h][:, 6 * j].double() - w8).abs() <= (2 * float(err.max()) + 2.0 ** -18) * w8 + 1e-30).all())


def test_record_and_chunk_in_a_graph():
    c, d = (Case(2, 2, 64, [50], feature_window=8, cap=200) for _ in range(2))
    decode((c, d), [(c.rand(1, 2), c.rand(1, 2), c.rand(1, 4)) for _ in range(3)])
    k, v, q = c.chunk([20])
    lse = torch.empty(q.shape[:2], device="cuda")
    for x in (c, d):
        x.cache.append_chunk_attn(0, k, v, q, [20], lse=lse)
        x.extend(k, v, [20])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.chunk_features(0, q, lse, [20])
    graph.replay()
    d.cache.chunk_features(0, q, lse, [20])
    once = c.cache.export_features(0, 0)
    assert torch.equal(once, d.cache.export_features(0, 0))
    graph.replay()
    check_features(c, q, [20], [once])   # the record was used once


def test_a_call_captured_before_the_first_decode_step_leaves_the_record():
    c, d = (Case(2, 2, 64, [50], feature_window=8, cap=200) for _ in range(2))
    k, v, q = c.chunk([5])
    lse = torch.empty(q.shape[:2], device="cuda")
    for x in (c, d):
        x.cache.append_chunk_attn(0, k, v, q, [5], lse=lse)
        x.extend(k, v, [5])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.chunk_features(0, q, lse, [5])
    decode((c, d), [(c.rand(1, 2), c.rand(1, 2), c.rand(1, 4)) for _ in range(3)])
    graph.replay()   # (of the last five pairs as they are now; its sums do not matter here)
    for x in (c, d):
        x.cache.update_features(0)
    got, want = (x.cache.export_features(0, 0).unflatten(2, (2, 6)) for x in (c, d))
    assert torch.equal(got[..., :4], want[..., :4])   # the windows and the mean of the three decode queries
