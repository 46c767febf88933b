"""Roll-backs of chunks: in captured graphs, in a pool without free pages, and what rejected drafts leave behind."""
import math

import pytest
import torch

import chunk_ref as ref
from paper_2602_03203_b200 import binding
from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


def used_pages(c):
    return sum(-(-len(s) // 16) for s in c.seqs) * c.Hkv


def test_a_captured_roll_back_to_the_length_at_capture_rolls_every_replay_back():
    c = Case(2, 2, 64, [30, 47], cap=96)
    total = c.cache.device_status()[1] + used_pages(c)
    lens, keep = [20, 3], [30, 47]
    k, v, q = c.chunk(lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):   # (the lengths are `keep` as it is captured: nothing to drop yet)
        c.cache.append_chunk(0, None, None, [0, 0], keep_lens=keep)
        c.cache.append_chunk(0, k, v, lens)
    for _ in range(6):
        graph.replay()
    c.cache.sync_lengths()
    c.extend(k, v, lens)
    c.check_stored()
    assert c.cache.device_status() == (0, total - used_pages(c))


@pytest.mark.parametrize("spare", [0, 2, 3])
def test_pages_that_a_call_returns_serve_its_own_growth(spare):
    # Two sequences shrink and two grow in one call; the pool has `spare` free pages, fewer than the growth takes.
    Hkv = 2
    c = Case(Hkv, 4, 64, [48, 17, 40, 16], cap=160, num_pages=(3 + 2 + 3 + 1) * Hkv + spare)
    assert c.cache.device_status() == (0, spare)
    keep, lens = [10, 17, 2, 16], [0, 32, 5, 30]      # pages a head: 3 -> 1, 2 -> 4, 3 -> 1, 1 -> 3
    k, v, q = c.chunk(lens)
    lse = torch.empty(q.shape[:2], device="cuda")
    out = c.cache.append_chunk_attn(0, k, v, q, lens, keep_lens=keep, lse=lse)
    c.extend(k, v, lens, keep=keep)
    assert c.cache.device_status() == (0, spare)
    c.check_stored()
    c.check_chunk(out, lse, q, lens)
    # A net demand of exactly what is free, then of more: refused as a whole, nothing lost.
    keep, lens = [10, 49, 7, 46], [32 if spare else 0, 0, 0, 0]
    if spare == 2:
        lens[0] = 22
        k, v, q = c.chunk(lens)
        c.cache.append_chunk(0, k, v, lens, keep_lens=keep)
        c.extend(k, v, lens, keep=keep)
        assert c.cache.device_status() == (0, 0)
    free = c.cache.device_status()[1]
    keep = [len(c.seqs[0]), 48, 7, 46]                 # a page a head comes back ...
    lens = [0, 0, 0, 16 * (free // Hkv) + 35]          # ... and one more than it and the free ones is wanted
    k, v, q = c.chunk(lens)
    c.cache.append_chunk(0, k, v, lens, keep_lens=keep)
    assert c.cache.device_status() == (binding.DEV_POOL_EXHAUSTED, free)
    c.cache.sync_lengths()
    c.check_stored()
    c.cache.append_chunk(0, None, None, [0] * 4, keep_lens=[0] * 4)
    assert c.cache.device_status() == (0, (3 + 2 + 3 + 1) * Hkv + spare)
    # No page is on the stack twice: the whole pool is taken again and holds what was stored.
    c.seqs = [ref.Seq(Hkv, 64, 24) for _ in range(4)]
    lens = [16 * ((9 * Hkv + spare) // Hkv // 4)] * 4
    k, v, q = c.chunk(lens)
    c.cache.append_chunk(0, k, v, lens)
    c.extend(k, v, lens)
    c.check_stored()
    assert c.status() == 0


@pytest.mark.parametrize("D,g,n", [(128, 4, 35), (64, 2, 3000), (128, 7, 1), (64, 8, 16)])
def test_infinities_of_rejected_drafts_do_not_reach_decode_steps(D, g, n):
    # A decode step reads the last page whole: rows behind the last pair hold what was rolled back.
    c = Case(2, g, D, [n, n + 9], cap=n + 60)
    bad = c.rand(12, 2)
    bad[::2], bad[1::2] = math.inf, math.nan
    c.cache.append_chunk(0, bad, bad, [6, 6])
    c.cache.append_chunk(0, None, None, [0, 0], keep_lens=[n, n + 9])

    def check(out, q):
        for s, seq in enumerate(c.seqs):
            m = len(seq)
            ok = torch.ones((1, m), dtype=torch.bool, device="cuda")
            for hq in range(2 * g):
                o, _, _, tol, _ = ref.attend(q[s:s + 1, hq], seq.k[hq // g], seq.v[hq // g], ok, D ** -0.5)
                d = (out[s:s + 1, hq].double() - o).abs()
                assert bool((d <= tol).all()), (s, hq, float(d.max()))

    q = c.rand(2, 2 * g)
    check(c.cache.decode_attn(0, q), q)
    for _ in range(2):
        k, v, q = c.rand(2, 2), c.rand(2, 2), c.rand(2, 2 * g)
        out = c.cache.append_decode_attn(0, k, v, q)
        c.extend(k, v, [1, 1])
        check(out, q)
    k, v, q = c.rand(2, 2), c.rand(2, 2), c.rand(2, 2 * g)
    out = c.cache.decode_step(k[None], v[None], q[None])[0]
    c.extend(k, v, [1, 1])
    check(out, q)
    c.check_stored()
    assert c.status() == 0


def test_infinities_in_a_page_of_another_sequence_do_not_reach_decode_steps():
    # The same with a page that another sequence held before.
    c = Case(1, 4, 128, [0, 0], num_pages=4, cap=64)
    bad = torch.full((60, 1, 128), math.inf, dtype=torch.bfloat16, device="cuda")
    c.cache.append_chunk(0, bad, bad, [60, 0])
    c.cache.append_chunk(0, None, None, [0, 0], keep_lens=[0, 0])
    k, v = c.rand(21, 1), c.rand(21, 1)
    c.cache.prefill(0, 1, k.transpose(0, 1).contiguous(), v.transpose(0, 1).contiguous())
    q = c.rand(2, 4)
    out = c.cache.decode_attn(0, q)
    assert bool((out[0] == 0).all())
    for h in range(4):
        o, _, _, tol, _ = ref.attend(q[1:2, h], k[:, 0], v[:, 0], torch.ones((1, 21), dtype=torch.bool, device="cuda"), 128 ** -0.5)
        assert bool(((out[1:2, h].double() - o).abs() <= tol).all())
