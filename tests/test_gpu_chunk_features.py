"""Attention features from the queries of a chunk, against a plain 64-bit implementation, and the evictions that follow."""
import ctypes

import pytest
import torch

import chunk_ref as ref
import oracle
from paper_2602_03203_b200 import binding
from test_gpu_chunk import Case
from util import npf

pytestmark = pytest.mark.gpu
CUM_SUM = 4   # the feature column that holds the accumulated attention


def check_features(c, q, lens, old, window=0, sinks=0, scale=None):
    """The cache's features after a chunk against `old` ([sequence][head] rows before it) moved on by the definition.

    A probability is off by its score's error (the bound of chunk_ref.attend, twice: the given log-sum-exp carries it too),
    a sum of T of them in fp32 by T 2^-24 at most, and the updates round a few times more.
    """
    row = 0
    for s, t in enumerate(lens):
        got = c.cache.export_features(0, s)
        for h in range(c.Hkv):
            if not t:
                assert torch.equal(got[h], old[s][h])
                continue
            seq = c.seqs[s]
            n = seq.k[h].shape[0]
            slot = torch.arange(n - t, n, device="cuda")
            ok = ref.seen(seq.pos[h], slot, seq.pos[h][n - t:], window, sinks)
            for j in range(c.g):
                _, _, p, _, err = ref.attend(q[row:row + t, h * c.g + j], seq.k[h], seq.v[h], ok, scale or c.D ** -0.5)
                new = ref.features(old[s][h][:, 6 * j:6 * j + 6], p, t)
                tol = (2 * float(err.max()) + t * 2.0 ** -24 + 2.0 ** -21) * new.abs() + 1e-30
                d = (got[h][:, 6 * j:6 * j + 6].double() - new).abs()
                assert bool((d <= tol).all()), (s, h, j, float((d / tol).max()))
        row += t
    assert c.status() == 0


def run_features(c, lens, window=0, sinks=0, scale=0.0, pos=None):
    k, v, q = c.chunk(lens)
    lse = torch.empty(q.shape[:2], device="cuda")
    c.cache.append_chunk_attn(0, k, v, q, lens, window=window, sinks=sinks, lse=lse, scale=scale, pos=pos)
    c.extend(k, v, lens, pos)
    old = [c.cache.export_features(0, s) for s in range(c.batch)]
    c.cache.chunk_features(0, q, lse, lens, window=window, sinks=sinks, scale=scale)
    check_features(c, q, lens, old, window, sinks, scale or None)


@pytest.mark.parametrize("g", range(1, 9))
@pytest.mark.parametrize("D", [64, 128])
def test_features_groups(g, D):
    c = Case(2, g, D, [150, 0, 33])
    run_features(c, [21, 40, 0])
    run_features(c, [9, 140, 3])


@pytest.mark.parametrize("n", [0, 1, 127, 128, 129, 255, 256, 257, 700])
@pytest.mark.parametrize("T", [1, 7, 8, 9, 16, 31, 32, 33, 127, 128, 129, 300])
def test_features_lengths(n, T):
    run_features(Case(1, 2, 128, [n]), [T])


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 0), (16, 4), (100, 17), (128, 0), (200, 300), (5000, 4),
                                          (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("gap", [1, 3])
def test_features_windows(window, sinks, gap):
    c = Case(2, 3, 64, [450, 130, 0, 1200], gap=gap)
    run_features(c, [70, 5, 290, 1], window, sinks)
    run_features(c, [1, 64, 3, 0], window, sinks)


@pytest.mark.parametrize("window", [1, 25, 150])
def test_features_windows_over_a_chunk_with_gaps(window):
    c = Case(2, 2, 64, [300, 5])
    step = torch.randint(1, 6, (400,), generator=c.gen, device="cuda", dtype=torch.int32)
    pos = torch.cat([300 + torch.cumsum(step[:250], 0, dtype=torch.int32), 5 + torch.cumsum(step[250:], 0, dtype=torch.int32)])
    run_features(c, [250, 150], window, 3, pos=pos)


def test_features_long_and_scaled():
    c = Case(2, 4, 128, [5000], cap=6000)
    run_features(c, [900], scale=0.05)


def test_features_many_sequences():
    c = Case(1, 2, 64, [(s * 7) % 400 for s in range(100)], cap=512)
    run_features(c, [(s * 11) % 40 for s in range(100)])


def test_features_in_a_graph():
    c = Case(2, 4, 64, [300])
    lens = [40]
    k, v, q = c.chunk(lens)
    lse = torch.empty(q.shape[:2], device="cuda")
    c.cache.append_chunk_attn(0, k, v, q, lens, lse=lse)
    c.extend(k, v, lens)
    old = [c.cache.export_features(0, 0)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.chunk_features(0, q, lse, lens)
    graph.replay()
    check_features(c, q, lens, old)
    old = [c.cache.export_features(0, 0)]
    graph.replay()
    check_features(c, q, lens, old)


@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 4)])
def test_prompt_in_chunks_then_eviction_by_accumulated_attention(window, sinks):
    # A prompt in uneven chunks: attention, features; then the pairs with the least accumulated attention go, and decoding
    # and further chunks run on what is left.
    c = Case(2, 4, 128, [0, 0], budget=96, recent_keep=16, cap=1024)
    for lens in ([130, 40], [64, 0], [257, 200], [31, 90]):
        run_features(c, lens, window, sinks)
    feats = [c.cache.export_features(0, s) for s in range(2)]
    c.cache.evict_by_feature(CUM_SUM, 0)
    for s in range(2):
        for h in range(2):
            phi = oracle.score_feature(npf(feats[s][h]), 4, CUM_SUM)
            kept = torch.from_numpy(oracle.select(phi, 96, 16)).long().cuda()
            seq = c.seqs[s]
            k, v, f, pos = c.cache.export_head(0, s, h)
            assert torch.equal(pos, seq.pos[h][kept]) and torch.equal(k, seq.k[h][kept]) and torch.equal(v, seq.v[h][kept])
            assert torch.equal(f, feats[s][h][kept]) and seq.k[h].shape[0] > 96
            seq.k[h], seq.v[h], seq.f[h], seq.pos[h] = k, v, f, pos
    run_features(c, [17, 3], window, sinks)
    k, v, q = c.rand(2, 2), c.rand(2, 2), c.rand(2, 8)
    c.cache.append_decode_attn_window(0, k, v, q, 50, 4)


def test_features_refusals():
    c = Case(2, 4, 64, [20, 10], cap=64)
    lib, h, st = binding.lib(), c.cache._h, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    _, _, q = c.chunk([3, 2])
    lse = torch.zeros(q.shape[:2], device="cuda")
    p = lambda t, off=0: ctypes.c_void_p(t.data_ptr() + off)  # noqa: E731
    i2 = lambda *x: (ctypes.c_int32 * 2)(*x)                  # noqa: E731
    old = [c.cache.export_features(0, s) for s in range(2)]

    def call(layer=0, qq=p(q), ll=p(lse), lens=i2(3, 2), window=0, sinks=0, scale=0.0):
        return lib.fkv_chunk_features(h, layer, qq, ll, lens, window, sinks, scale, st)

    for bad in [dict(layer=1), dict(qq=None), dict(qq=p(q, 2)), dict(ll=None), dict(ll=p(lse, 2)), dict(lens=None), dict(lens=i2(-1, 0)),
                dict(lens=i2(21, 0)), dict(window=-1), dict(sinks=-1), dict(scale=-1.0), dict(scale=float("inf"))]:
        assert call(**bad) == -1, bad
    assert call(lens=i2(0, 0), qq=None, ll=None) == 0
    with pytest.raises(ValueError):
        c.cache.chunk_features(0, q, lse[:4], [3, 2])
    for s in range(2):
        assert torch.equal(c.cache.export_features(0, s), old[s])
    assert c.status() == 0
