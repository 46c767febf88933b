"""Chunks of new tokens over the paged cache, sliding windows and sinks: against plain 64-bit implementations."""
import ctypes
import math

import pytest
import torch

import chunk_ref as ref
from paper_2602_03203_b200 import binding

pytestmark = pytest.mark.gpu


class Case:
    """A one-layer cache and what it should hold, filled with `stored` pairs per sequence."""

    def __init__(self, Hkv, g, D, stored, seed=0, gap=1, cap=None, window=0, sinks=4, **kw):
        self.Hkv, self.g, self.D, self.batch = Hkv, g, D, len(stored)
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.cache = binding.Cache(1, Hkv, g, D, self.batch, kw.pop("budget", 16), cap or max(max(stored) + 700, 64), **kw)
        self.seqs = [ref.Seq(Hkv, D, 6 * g) for _ in stored]
        for s, n in enumerate(stored):
            if not n:
                continue
            k, v = self.rand(n, Hkv), self.rand(n, Hkv)
            step = torch.randint(1, 2 * gap, (n,), generator=self.gen, device="cuda", dtype=torch.int32)
            step[: sinks + 1] = 1
            pos = torch.cumsum(step, 0, dtype=torch.int32) - 1
            f = torch.rand((Hkv, n, 6 * g), generator=self.gen, device="cuda")
            self.seqs[s].extend(k, v, pos)
            for h in range(Hkv):
                self.seqs[s].f[h] = f[h]
            self.cache.prefill(0, s, k.transpose(0, 1).contiguous(), v.transpose(0, 1).contiguous(), f, pos)

    def rand(self, n, heads, scale=1.0):
        return (torch.randn((n, heads, self.D), generator=self.gen, device="cuda") * scale).to(torch.bfloat16)

    def chunk(self, lens):
        total = sum(lens)
        return self.rand(total, self.Hkv), self.rand(total, self.Hkv), self.rand(total, self.Hkv * self.g, 2.0)

    def extend(self, k, v, lens, pos=None, keep=None):
        row = 0
        for s, t in enumerate(lens):
            part = slice(row, row + t)
            if t or keep is not None:
                self.seqs[s].extend(k[part], v[part], None if pos is None else pos[part], None if keep is None else keep[s])
            row += t

    def check_chunk(self, out, lse, q, lens, window=0, sinks=0, scale=None):
        scale = scale or self.D ** -0.5
        row = 0
        for s, t in enumerate(lens):
            seq = self.seqs[s]
            for h in range(self.Hkv):
                n = seq.k[h].shape[0]
                slot = torch.arange(n - t, n, device="cuda")
                ok = ref.seen(seq.pos[h], slot, seq.pos[h][n - t:], window, sinks)
                for j in range(self.g if t else 0):
                    hq = h * self.g + j
                    o, l, _, tol, ltol = ref.attend(q[row:row + t, hq], seq.k[h], seq.v[h], ok, scale)
                    d = (out[row:row + t, hq].double() - o).abs()
                    assert bool((d <= tol).all()), (s, h, j, float((d / tol).max()))
                    if lse is not None:
                        d = (lse[row:row + t, hq].double() - l).abs()
                        assert bool((d <= ltol).all()), (s, h, j, float((d / ltol).max()))
            row += t

    def check_stored(self):
        assert self.cache.lengths(0) == [len(s) for s in self.seqs]
        for s, seq in enumerate(self.seqs):
            for h in range(self.Hkv if len(seq) else 0):
                k, v, f, pos = self.cache.export_head(0, s, h)
                assert torch.equal(k.view(torch.int16), seq.k[h].view(torch.int16)), (s, h)
                assert torch.equal(v.view(torch.int16), seq.v[h].view(torch.int16)), (s, h)
                assert torch.equal(pos, seq.pos[h]), (s, h)
                assert torch.equal(f, seq.f[h]), (s, h)

    def status(self):
        return self.cache.device_status()[0]


def run_chunk(c, lens, window=0, sinks=0, keep=None, pos=None, scale=0.0):
    k, v, q = c.chunk(lens)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    out = c.cache.append_chunk_attn(0, k, v, q, lens, pos=pos, keep_lens=keep, window=window, sinks=sinks, lse=lse, scale=scale)
    c.extend(k, v, lens, pos, keep)
    assert c.status() == 0
    c.check_chunk(out, lse, q, lens, window, sinks, scale or None)
    return k, v, q, out, lse


# ------------------------------------------------------------------ storing
@pytest.mark.parametrize("D,g,Hkv", [(64, 4, 2), (128, 7, 3), (128, 1, 1)])
def test_append_chunk_stores_and_rolls_back(D, g, Hkv):
    c = Case(Hkv, g, D, [0, 5, 16, 31, 40])
    for lens, keep in [([3, 11, 16, 1, 0], None), ([0, 0, 0, 0, 0], [1, 16, 0, 32, 33]), ([40, 1, 2, 17, 15], [1, 15, 0, 31, 33]),
                       ([1, 1, 1, 1, 1], [41, 16, 2, 48, 48]), ([0, 0, 0, 0, 0], [0, 0, 0, 0, 0]), ([16, 0, 33, 0, 1], None)]:
        k, v, _ = c.chunk(lens)
        free0 = c.cache.device_status()[1]
        before = sum(-(-len(s) // 16) for s in c.seqs) * Hkv
        c.cache.append_chunk(0, k if sum(lens) else None, v if sum(lens) else None, lens, keep_lens=keep)
        c.extend(k, v, lens, keep=keep)
        after = sum(-(-len(s) // 16) for s in c.seqs) * Hkv
        status, free = c.cache.device_status()
        assert status == 0 and free == free0 + before - after
        c.check_stored()
    c.cache.reset()
    assert c.cache.device_status()[1] == free + sum(-(-len(s) // 16) for s in c.seqs) * Hkv


def test_append_chunk_positions_given():
    c = Case(2, 4, 64, [20, 0], gap=3)
    lens = [5, 7]
    first = int(c.seqs[0].pos[0][-1])
    pos = torch.tensor([first + x for x in (2, 3, 9, 11, 12)] + [4, 6, 7, 20, 21, 22, 40], dtype=torch.int32, device="cuda")
    k, v, _ = c.chunk(lens)
    c.cache.append_chunk(0, k, v, lens, pos=pos)
    c.extend(k, v, lens, pos)
    c.check_stored()


def test_append_chunk_equals_single_appends():
    a, b = Case(2, 4, 128, [30, 0, 47]), Case(2, 4, 128, [30, 0, 47])
    lens = [18, 18, 18]
    k, v, _ = a.chunk(lens)
    a.cache.append_chunk(0, k, v, lens)
    for j in range(18):
        rows = torch.tensor([j, 18 + j, 36 + j], device="cuda")
        b.cache.append(0, k[rows].contiguous(), v[rows].contiguous())
    for s in range(3):
        for h in range(2):
            for x, y in zip(a.cache.export_head(0, s, h), b.cache.export_head(0, s, h)):
                assert torch.equal(x, y)


def test_append_chunk_without_pages_stores_nothing():
    c = Case(2, 2, 64, [16, 16], num_pages=10, cap=160)   # four pages in use, six free
    k, v, _ = c.chunk([17, 33])                            # needs 4 + 6
    c.cache.append_chunk(0, k, v, [17, 33])
    status, free = c.cache.device_status()
    assert status == binding.DEV_POOL_EXHAUSTED and free == 6
    c.cache.sync_lengths()
    c.check_stored()
    k, v, _ = c.chunk([17, 16])                            # exactly the six
    c.cache.append_chunk(0, k, v, [17, 16])
    c.extend(k, v, [17, 16])
    assert c.cache.device_status() == (0, 0)
    c.check_stored()


# ------------------------------------------------------------------ attention of a chunk
@pytest.mark.parametrize("g", range(1, 9))
@pytest.mark.parametrize("D", [64, 128])
def test_chunk_attention_groups(g, D):
    c = Case(2, g, D, [150, 0, 33])
    run_chunk(c, [21, 40, 3])
    c.check_stored()


@pytest.mark.parametrize("n", [0, 1, 15, 16, 17, 111, 112, 127, 128, 129, 1000])
@pytest.mark.parametrize("T", [1, 2, 16, 31, 32, 33, 64, 65, 129])
def test_chunk_attention_lengths(n, T):
    c = Case(1, 4, 128, [n])
    run_chunk(c, [T])


@pytest.mark.parametrize("T", [127, 128, 129, 255, 256, 257, 600])
def test_chunk_attention_single_head_groups(T):
    c = Case(2, 1, 64, [70, 3])
    run_chunk(c, [T, 5])


def test_chunk_attention_ragged_batch_with_idle_sequences():
    stored = [(s * 97) % 500 for s in range(20)]
    lens = [0 if s % 5 == 3 else (s * 53) % 90 for s in range(20)]
    lens[0] = 1
    c = Case(2, 7, 128, stored)
    run_chunk(c, lens)
    run_chunk(c, lens[::-1])
    c.check_stored()


def test_chunk_attention_many_sequences():
    c = Case(1, 2, 64, [(s * 7) % 40 for s in range(256)], cap=128)
    run_chunk(c, [(s * 11) % 4 for s in range(256)])


def test_chunk_attention_long():
    c = Case(2, 4, 128, [20000, 300], cap=21000)
    run_chunk(c, [700, 40])


@pytest.mark.parametrize("D,g", [(128, 4), (64, 7), (128, 1), (64, 3)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1500, 4)])
def test_chunk_attention_cut_items_of_both_forms(D, g, window, sinks):
    """Items of one and of two query tiles, each gone on with by several CTAs, in the same call."""
    c = Case(2, g, D, [3000, 5000, 0], cap=6000)
    run_chunk(c, [400, 5, 37], window=window, sinks=sinks)
    run_chunk(c, [3, 256 // g, 128 // g], window=window, sinks=sinks)
    c.check_stored()


def test_chunk_attention_drafts_accepted_and_rejected():
    c = Case(4, 4, 128, [500, 77, 1])
    keep = [500, 77, 1]
    for accepted in ([2, 0, 5], [5, 5, 5], [0, 1, 0], [3, 2, 1]):
        run_chunk(c, [5, 5, 5], keep=keep)
        keep = [n + a for n, a in zip(keep, accepted)]
    c.check_stored()


@pytest.mark.parametrize("scale", [0.05, 0.7])
def test_chunk_attention_scale(scale):
    c = Case(2, 3, 64, [200])
    run_chunk(c, [30], scale=scale)


def test_chunk_attention_growing_scores_rescale():
    # Keys grow along the cache, so the running maximum moves on in nearly every tile.
    c = Case(1, 4, 128, [0])
    lens = [600]
    k, v, q = c.chunk(lens)
    ramp = torch.linspace(0.05, 8.0, 600, device="cuda")[:, None, None]
    k = (q[:, :1].float() * 0 + 1).to(torch.bfloat16) * ramp.to(torch.bfloat16)
    q = q.abs()
    lse = torch.empty((600, 4), device="cuda")
    out = c.cache.append_chunk_attn(0, k.contiguous(), v, q, lens, lse=lse)
    c.extend(k, v, lens)
    c.check_chunk(out, lse, q, lens)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 0), (16, 4), (64, 4), (100, 17), (128, 0), (200, 40), (5000, 4),
                                          (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("gap", [1, 3])
def test_chunk_attention_windows(window, sinks, gap):
    c = Case(2, 4, 128, [450, 130, 0, 31], gap=gap)
    run_chunk(c, [70, 5, 90, 1], window, sinks)
    run_chunk(c, [1, 64, 3, 0], window, sinks)


def test_chunk_attention_window_after_eviction_per_head():
    # Every head keeps pairs of its own, so the window begins at a slot of its own.
    c = Case(3, 2, 64, [900, 400], budget=128, recent_keep=16)
    c.cache.evict_by_feature(4, 0)
    for s in range(2):
        for h in range(3):
            k, v, f, pos = c.cache.export_head(0, s, h)
            c.seqs[s].k[h], c.seqs[s].v[h], c.seqs[s].f[h], c.seqs[s].pos[h] = k, v, f, pos
    assert not torch.equal(c.seqs[0].pos[0], c.seqs[0].pos[1])
    for window, sinks in [(150, 4), (400, 0), (40, 300)]:
        run_chunk(c, [20, 7], window, sinks, keep=[128, 128])


def test_chunk_attention_leaves_rows_behind_alone():
    c = Case(2, 4, 64, [100, 50])
    lens = [9, 4]
    k, v, q = c.chunk(lens)
    big = torch.full((20, 8, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((20, 8), 5.0, device="cuda")
    c.cache.append_chunk_attn(0, k, v, q, lens, out=big[:13], lse=lse[:13])
    assert bool((big[13:] == 3.0).all()) and bool((lse[13:] == 5.0).all())


def test_chunk_attention_ignores_what_freed_pages_held():
    # Pages that held infinities and NaN go back to the pool and are taken again, half filled, by another sequence.
    c = Case(1, 4, 128, [0, 0], num_pages=4, cap=64)
    bad = torch.full((60, 1, 128), math.inf, dtype=torch.bfloat16, device="cuda")
    bad[::2] = math.nan
    c.cache.append_chunk(0, bad, bad, [60, 0])
    c.cache.append_chunk(0, None, None, [0, 0], keep_lens=[0, 0])
    run_chunk(c, [0, 21])
    run_chunk(c, [0, 1], window=3, sinks=2)


@pytest.mark.parametrize("D,T", [(128, 9), (64, 200)])
def test_chunk_attention_ignores_what_no_query_sees(D, T):
    # Infinities and NaN in keys and values that lie outside the window of every query of the chunk.
    c = Case(2, 4, D, [0, 0])
    n, window, sinks = [333, 90], 20, 5
    for s in range(2):
        k, v = c.rand(n[s], 2), c.rand(n[s], 2)
        hidden = slice(sinks, n[s] - window + 1)
        k[hidden][::2], k[hidden][1::2], v[hidden][::2], v[hidden][1::2] = math.inf, math.nan, math.nan, -math.inf
        lens = [n[s] if i == s else 0 for i in range(2)]
        c.cache.append_chunk(0, k, v, lens)
        k[hidden], v[hidden] = 0, 0
        c.extend(k, v, lens)
    run_chunk(c, [T, 3], window, sinks)


def test_chunks_of_two_caches_on_two_streams():
    cases = [Case(2, 4, 128, [700, 90], seed=s) for s in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    lens, calls = [60, 7], []
    torch.cuda.synchronize()
    for c in cases:
        calls.append([c.chunk(lens) for _ in range(4)])
    torch.cuda.synchronize()
    results = [[], []]
    for step in range(4):
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                k, v, q = calls[i][step]
                lse = torch.empty(q.shape[:2], device="cuda")
                results[i].append((c.cache.append_chunk_attn(0, k, v, q, lens, lse=lse), lse))
    torch.cuda.synchronize()
    for i, c in enumerate(cases):
        for (k, v, q), (out, lse) in zip(calls[i], results[i]):
            c.extend(k, v, lens)
            c.check_chunk(out, lse, q, lens)
        assert c.status() == 0


def test_chunk_attention_on_pages_past_four_gigabytes():
    # 16 sequences of 65536 pairs on eight heads take 4.5 GB of pages; the last one's lie behind 2^32 bytes.
    Hkv, D, n = 8, 128, 65536
    cache = binding.Cache(1, Hkv, 1, D, 17, 16, n, num_pages=17 * Hkv * (n // 16) - 8 * 3000)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    k = torch.randn((Hkv, n, D), generator=gen, device="cuda").to(torch.bfloat16)
    v = torch.randn((Hkv, n, D), generator=gen, device="cuda").to(torch.bfloat16)
    for s in range(16):
        cache.prefill(0, s, k, v)
    c = Case(Hkv, 1, D, [0], seed=8)   # (its own small cache is not used)
    c.cache, c.batch = cache, 17
    c.seqs = [ref.Seq(Hkv, D, 6) for _ in range(17)]
    for h in range(Hkv):
        c.seqs[15].k[h], c.seqs[15].v[h] = k[h], v[h]
        c.seqs[15].pos[h] = torch.arange(n, dtype=torch.int32, device="cuda")
    keep = [n] * 15 + [n - 40, 0]
    lens = [0] * 15 + [40, 300]
    kn, vn, q = c.chunk(lens)
    lse = torch.empty(q.shape[:2], device="cuda")
    out = cache.append_chunk_attn(0, kn, vn, q, lens, keep_lens=keep, lse=lse)
    c.seqs[15].extend(kn[:40], vn[:40], keep=n - 40)
    c.seqs[16].extend(kn[40:], vn[40:])
    assert cache.device_status()[0] == 0
    c.check_chunk(out, lse, q, lens)
    cache.chunk_features(0, q, lse, lens)
    assert bool(torch.isfinite(cache.export_features(0, 15)).all())
    out = cache.decode_attn_window(0, q[:17].contiguous(), 5000, 4)
    o, _, _, tol, _ = ref.attend(q[15:16, 3], c.seqs[15].k[3], c.seqs[15].v[3],
                                 ref.seen(c.seqs[15].pos[3], torch.tensor([n - 1], device="cuda"), c.seqs[15].pos[3][-1:], 5000, 4), D ** -0.5)
    assert bool(((out[15:16, 3].double() - o).abs() <= tol).all())


def test_chunk_attention_reproducible_and_independent_of_the_split():
    c = Case(2, 4, 128, [3000, 20])
    lens = [100, 33]
    k, v, q = c.chunk(lens)
    c.cache.append_chunk(0, k, v, lens)
    first = c.cache.chunk_attn(0, q, lens)
    for _ in range(20):
        assert torch.equal(c.cache.chunk_attn(0, q, lens), first)


def test_chunk_attention_on_another_stream_and_in_a_graph():
    c = Case(2, 4, 128, [300, 90])
    lens, keep = [6, 3], [300, 90]
    k, v, q = c.chunk(lens)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.cache.append_chunk_attn(0, k, v, q, lens, keep_lens=keep, out=out, lse=lse)
    side.synchronize()
    c.extend(k, v, lens, keep=keep)
    c.check_chunk(out, lse, q, lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.append_chunk_attn(0, k, v, q, lens, out=out, lse=lse)   # behind all pairs: every replay grows the cache
    c.cache.sync_lengths()
    assert c.cache.lengths(0) == [306, 93]
    for _ in range(40):
        k2, v2, q2 = c.chunk(lens)
        k.copy_(k2), v.copy_(v2), q.copy_(q2)
        graph.replay()
        c.extend(k, v, lens)
    torch.cuda.synchronize()
    c.check_chunk(out, lse, q, lens)
    c.cache.sync_lengths()
    c.check_stored()
    assert c.status() == 0


def test_replayed_chunks_stop_at_the_capacity():
    c = Case(1, 2, 64, [40], cap=64)
    k, v, q = c.chunk([10])
    out = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.append_chunk_attn(0, k, v, q, [10], out=out)
    for _ in range(5):
        graph.replay()
    torch.cuda.synchronize()
    assert c.status() == binding.DEV_CAPACITY
    c.cache.sync_lengths()
    assert c.cache.lengths(0) == [60]


def test_decode_queries_of_rolled_back_tokens_leave_the_record():
    # Two caches take the same tokens; one of them also takes tokens that are rolled back again.  Their features agree.
    torch.manual_seed(3)
    a, b = (Case(2, 2, 64, [60, 33], feature_window=16) for _ in range(2))

    def step(cs, x):
        for c in cs:
            c.cache.append_decode_attn(0, x[0], x[1], x[2])

    def tokens():
        return a.rand(2, 2), a.rand(2, 2), a.rand(2, 4)

    for _ in range(5):
        step((a, b), tokens())
    for _ in range(3):
        step((b,), tokens())
    b.cache.append_chunk(0, None, None, [0, 0], keep_lens=[65, 38])
    for _ in range(4):
        step((a, b), tokens())
    a.cache.update_features(0)
    b.cache.update_features(0)
    for s in range(2):
        assert torch.equal(a.cache.export_features(0, s), b.cache.export_features(0, s))


# ------------------------------------------------------------------ one token: windows and sinks
def check_window(c, out, q, window, sinks, q_pos=None, scale=None):
    for s, seq in enumerate(c.seqs):
        for h in range(c.Hkv):
            n = seq.k[h].shape[0]
            p = seq.pos[h][-1:] if q_pos is None else q_pos[s:s + 1]
            ok = ref.seen(seq.pos[h], torch.tensor([n - 1], device="cuda"), p, window, sinks) if n else None
            for j in range(c.g):
                hq = h * c.g + j
                o, _, _, tol, _ = ref.attend(q[s:s + 1, hq], seq.k[h], seq.v[h], ok, scale or c.D ** -0.5)
                if n and not bool(ok.any()):
                    o, tol = torch.zeros_like(out[s:s + 1, hq]).double(), 0.0
                d = (out[s:s + 1, hq].double() - o).abs()
                assert bool((d <= tol).all()), (s, h, j, float(d.max()))
    assert c.status() == 0


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (17, 4), (100, 16), (300, 33), (4000, 4), (4096, 0),
                                          (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("D,g,gap", [(128, 4, 1), (128, 7, 3), (64, 8, 2), (64, 1, 1)])
def test_window_decode(window, sinks, D, g, gap):
    c = Case(2, g, D, [5000, 1, 16, 300, 0], gap=gap)
    q = c.rand(5, 2 * g)
    check_window(c, c.cache.decode_attn_window(0, q, window, sinks), q, window, sinks)


@pytest.mark.parametrize("batch", [1, 3, 40])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 2000])
def test_window_decode_appends(batch, n):
    # Few sequences: a cluster per segment; more: splits joined in global memory; many: one CTA per segment.
    c = Case(4, 4, 128, [n] * batch, gap=2)
    for window, sinks in [(40, 4), (1000, 0)]:
        for _ in range(3):
            k, v, q = c.rand(batch, 4), c.rand(batch, 4), c.rand(batch, 16)
            out = c.cache.append_decode_attn_window(0, k, v, q, window, sinks)
            c.extend(k, v, [1] * batch)
            check_window(c, out, q, window, sinks)
    c.check_stored()


def test_window_decode_from_an_empty_cache_across_pages():
    c = Case(2, 4, 64, [0, 0], cap=64)
    for _ in range(50):
        k, v, q = c.rand(2, 2), c.rand(2, 2), c.rand(2, 8)
        out = c.cache.append_decode_attn_window(0, k, v, q, 20, 3)
        c.extend(k, v, [1, 1])
        check_window(c, out, q, 20, 3)
    c.check_stored()


def test_window_decode_masked_sequences_and_positions():
    c = Case(2, 4, 128, [50, 70, 20], gap=3)
    k, v, q = c.rand(3, 2), c.rand(3, 2), c.rand(3, 8)
    pos = torch.tensor([int(s.pos[0][-1]) + 25 for s in c.seqs], dtype=torch.int32, device="cuda")
    out = c.cache.append_decode_attn_window(0, k, v, q, 30, 2, pos=pos, seq_mask=0b101)
    c.seqs[0].extend(k[:1], v[:1], pos[:1])
    c.seqs[2].extend(k[2:], v[2:], pos[2:])
    check_window(c, out, q, 30, 2)
    c.check_stored()


@pytest.mark.parametrize("sinks", [0, 3])
def test_window_decode_at_other_positions(sinks):
    c = Case(2, 4, 64, [400, 400, 400, 400], gap=2)
    last = int(c.seqs[0].pos[0][-1])
    # before every pair, in the middle, past the end but with pairs in the window, and so far that the window is empty
    q_pos = torch.tensor([0, 200, last + 10, last + 5000], dtype=torch.int32, device="cuda")
    q = c.rand(4, 8)
    out = c.cache.decode_attn_window(0, q, 60, sinks, q_pos=q_pos)
    check_window(c, out, q, 60, sinks, q_pos)
    if sinks == 0:
        assert bool((out[3] == 0).all())


def test_window_decode_ignores_what_it_does_not_see():
    c = Case(2, 4, 128, [333, 40])
    bad = c.rand(333, 2)
    bad[::2], bad[1::2] = math.inf, math.nan
    for s, n in enumerate([333, 40]):
        k, v = c.seqs[s].k, c.seqs[s].v
        for h in range(2):
            k[h][5:n - 20], v[h][5:n - 20] = bad[5:n - 20, h], bad[5:n - 20, h]
        c.cache.append_chunk(0, None, None, [0, 0], keep_lens=[0 if i == s else len(c.seqs[i]) if i > s else n0
                                                               for i, n0 in enumerate([333, 40])])
        c.cache.prefill(0, s, torch.stack(k), torch.stack(v))
        for h in range(2):
            c.seqs[s].pos[h] = torch.arange(n, dtype=torch.int32, device="cuda")
            c.seqs[s].f[h].zero_()
    q = c.rand(2, 8)
    out = c.cache.decode_attn_window(0, q, 20, 5)
    assert bool(torch.isfinite(out).all())
    for s in range(2):
        for h in range(2):
            n = c.seqs[s].k[h].shape[0]
            c.seqs[s].k[h][5:n - 20], c.seqs[s].v[h][5:n - 20] = 0, 0
    check_window(c, out, q, 20, 5)


def test_window_decode_leaves_no_query_record():
    a, b = (Case(2, 2, 64, [60], feature_window=16) for _ in range(2))
    x = a.rand(1, 2), a.rand(1, 2), a.rand(1, 4)
    y = a.rand(1, 2), a.rand(1, 2), a.rand(1, 4)
    a.cache.append_decode_attn(0, x[0], x[1], x[2])
    a.cache.append_decode_attn_window(0, y[0], y[1], y[2], 8, 1)
    b.cache.append_decode_attn(0, x[0], x[1], x[2])
    b.cache.append(0, y[0], y[1])
    a.cache.update_features(0)
    b.cache.update_features(0)
    assert torch.equal(a.cache.export_features(0, 0), b.cache.export_features(0, 0))


# ------------------------------------------------------------------ refusals
def test_refusals():
    c = Case(2, 4, 64, [20, 10], cap=64)
    lib, h, st = binding.lib(), c.cache._h, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    k, v, q = c.chunk([3, 2])
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    p = lambda t, off=0: ctypes.c_void_p(t.data_ptr() + off)  # noqa: E731
    i2 = lambda *x: (ctypes.c_int32 * 2)(*x)                  # noqa: E731
    inval, capacity = -1, -3

    def append(layer=0, kk=p(k), vv=p(v), keep=None, lens=i2(3, 2)):
        return lib.fkv_append_chunk(h, layer, kk, vv, None, keep, lens, st)

    def attn(layer=0, qq=p(q), lens=i2(3, 2), window=0, sinks=0, scale=0.0, o=p(out)):
        return lib.fkv_chunk_attn(h, layer, qq, lens, window, sinks, scale, o, p(lse), st)

    for bad in [dict(layer=1), dict(layer=-1), dict(kk=None), dict(vv=None), dict(kk=p(k, 2)), dict(vv=p(v, 8)), dict(lens=None),
                dict(lens=i2(-1, 2)), dict(keep=i2(21, 10)), dict(keep=i2(-1, 10)), dict(lens=i2(1 << 24, 1))]:
        assert append(**bad) == inval, bad
    assert append(lens=i2(45, 0)) == capacity and append(keep=i2(20, 10), lens=i2(0, 55)) == capacity
    for bad in [dict(layer=1), dict(qq=None), dict(qq=p(q, 2)), dict(o=None), dict(o=p(out, 4)), dict(lens=None), dict(lens=i2(-1, 0)),
                dict(lens=i2(21, 0)), dict(window=-1), dict(sinks=-1), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(scale=1e-32), dict(scale=1e32)]:
        assert attn(**bad) == inval, bad
    assert attn(lens=i2(0, 0), qq=None, o=None) == 0 and append(lens=i2(0, 0), kk=None, vv=None) == 0
    assert lib.fkv_append_chunk_attn(h, 0, p(k), p(v), None, None, i2(3, 2), p(q, 2), 0, 0, 0.0, p(out), None, st) == inval
    assert lib.fkv_append_chunk_attn(h, 0, p(k), p(v), None, None, i2(50, 2), p(q), 0, 0, 0.0, p(out), None, st) == capacity
    qd, od = c.rand(2, 8), c.rand(2, 8)
    for window, sinks in [(0, 0), (-3, 0), (4, -1)]:
        assert lib.fkv_decode_attn_window(h, 0, p(qd), None, window, sinks, p(od), 0.0, st) == inval
        assert lib.fkv_append_decode_attn_window(h, 0, p(k), p(v), None, None, p(qd), window, sinks, p(od), 0.0, st) == inval
    assert lib.fkv_decode_attn_window(h, 0, None, None, 4, 0, p(od), 0.0, st) == inval
    assert lib.fkv_export_features(h, 0, 2, p(out), st) == inval and lib.fkv_export_features(h, 0, 0, None, st) == inval
    with pytest.raises(ValueError):
        c.cache.chunk_attn(0, q, [3])
    with pytest.raises(ValueError):
        c.cache.chunk_attn(0, q, [3, 3])
    with pytest.raises(ValueError):
        c.cache.append_chunk(0, k, v[:4], [3, 2])
    with pytest.raises(ValueError):
        c.cache.chunk_attn(0, q, [3, 2], lse=lse.double())
    c.check_stored()   # nothing was stored by a refused call
    assert c.status() == 0


def test_misaligned_tensors_are_refused():
    c = Case(2, 4, 64, [20, 10], cap=64)
    lib, h, st = binding.lib(), c.cache._h, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    k, v, q = c.chunk([3, 2])
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    pos, feat = torch.arange(100, 105, dtype=torch.int32, device="cuda"), torch.zeros(2, 20, 24, device="cuda")
    lens = (ctypes.c_int32 * 2)(3, 2)
    p = lambda t, off=0: ctypes.c_void_p(t.data_ptr() + off)  # noqa: E731
    good = dict(k=p(k), v=p(v), q=p(q), out=p(out), pos=p(pos), lse=p(lse))

    def calls(**x):
        return (lib.fkv_append_chunk(h, 0, x["k"], x["v"], x["pos"], None, lens, st) if not {"q", "out", "lse"} & set(x["bad"]) else -1,
                lib.fkv_append_chunk_attn(h, 0, x["k"], x["v"], x["pos"], None, lens, x["q"], 0, 0, 0.0, x["out"], x["lse"], st),
                lib.fkv_append_decode_attn_window(h, 0, x["k"], x["v"], x["pos"], None, x["q"], 4, 0, x["out"], 0.0, st)
                if "lse" not in x["bad"] else -1)

    for name, offs in [("k", (2, 8)), ("v", (2, 8)), ("q", (2, 8)), ("out", (2, 8)), ("pos", (1, 2)), ("lse", (1, 2))]:
        for off in offs:
            assert calls(**{**good, name: ctypes.c_void_p(good[name].value + off)}, bad=[name]) == (-1, -1, -1), (name, off)
    for off in (2, 8):
        assert lib.fkv_decode_attn_window(h, 0, p(q, off), None, 4, 0, p(out), 0.0, st) == -1
        assert lib.fkv_decode_attn_window(h, 0, p(q), None, 4, 0, p(out, off), 0.0, st) == -1
    assert lib.fkv_decode_attn_window(h, 0, p(q), p(pos, 2), 4, 0, p(out), 0.0, st) == -1
    assert lib.fkv_chunk_attn(h, 0, p(q), lens, 0, 0, 0.0, p(out), p(lse, 2), st) == -1
    assert lib.fkv_export_features(h, 0, 0, p(feat, 2), st) == -1
    c.check_stored()
    assert c.status() == 0 and not out.any() and not lse.any() and not feat.any()
