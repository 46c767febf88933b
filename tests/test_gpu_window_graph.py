"""Windowed decode steps in captured graphs, and long first chunks of a prompt."""
import pytest
import torch

import chunk_ref as ref
from test_gpu_chunk import Case, check_window

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,n", [(1, 700), (3, 20), (40, 90)])
@pytest.mark.parametrize("window,sinks", [(33, 4), (5000, 0)])
def test_replayed_windowed_steps_follow_the_cache(batch, n, window, sinks):
    c = Case(2, 4, 128, [n + s % 3 for s in range(batch)], cap=n + 120, gap=2, sinks=sinks)
    k, v, q = c.rand(batch, 2), c.rand(batch, 2), c.rand(batch, 8)
    out, again = torch.zeros_like(q), torch.zeros_like(q)
    c.cache.decode_attn_window(0, q, window, sinks, out=again)   # (a kernel's first launch sets its attributes)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.append_decode_attn_window(0, k, v, q, window, sinks, out=out)
        c.cache.decode_attn_window(0, q, window, sinks, out=again)
    for step in range(70):
        for t, heads in ((k, 2), (v, 2), (q, 8)):
            t.copy_(c.rand(batch, heads))
        graph.replay()
        c.extend(k, v, [1] * batch)
        if step in (0, 1, 17, 69):
            check_window(c, out, q, window, sinks)
            check_window(c, again, q, window, sinks)
    c.cache.sync_lengths()
    c.check_stored()


@pytest.mark.parametrize("D,g,window", [(128, 4, 0), (64, 8, 0), (128, 4, 1000)])
def test_long_first_chunk_of_a_prompt(D, g, window):
    T = 6000
    c = Case(2, g, D, [0, 0], cap=T + 64)
    lens = [T, 17]
    k, v, q = c.chunk(lens)
    lse = torch.empty(q.shape[:2], device="cuda")
    out = c.cache.append_chunk_attn(0, k, v, q, lens, window=window, sinks=4, lse=lse)
    c.extend(k, v, lens)
    c.check_stored()
    c.check_chunk(out, lse, q, lens, window, 4)
    old = [c.cache.export_features(0, s) for s in range(2)]
    c.cache.chunk_features(0, q, lse, lens, window=window, sinks=4)
    for h in range(2):
        seq = c.seqs[0]
        ok = ref.seen(seq.pos[h], torch.arange(T, device="cuda"), seq.pos[h], window, 4)
        for j in range(g):
            _, _, p, _, err = ref.attend(q[:T, h * g + j], seq.k[h], seq.v[h], ok, D ** -0.5)
            want = ref.features(old[0][h][:, 6 * j:6 * j + 6], p, T)
            d = (c.cache.export_features(0, 0)[h][:, 6 * j:6 * j + 6].double() - want).abs()
            assert bool((d <= (2 * float(err.max()) + T * 2.0 ** -24 + 2.0 ** -21) * want + 1e-30).all())
    assert c.status() == 0
