"""Speculative steps as a decoder makes them: masks, attention in every layer, verification, the accepted path, and what may follow."""
import pytest
import torch

import tree_ref
from paper_2602_03203_b200 import binding

pytestmark = pytest.mark.gpu

L, HKV, G, D, BATCH, VOCAB = 2, 2, 4, 64, 3, 97


class Model:
    """A stand-in for a model: keys, values, queries and probabilities as functions of a token and its position."""

    def __init__(self, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.k, self.v = (torch.randn((L, VOCAB, HKV, D), generator=g, device="cuda") for _ in range(2))
        self.q = torch.randn((L, VOCAB, HKV * G, D), generator=g, device="cuda")
        self.head = torch.randn((HKV * G * D, VOCAB), generator=g, device="cuda") * 0.1

    def rows(self, layer, tokens):
        return tuple(x[layer][tokens.long()].to(torch.bfloat16).contiguous() for x in (self.k, self.v, self.q))

    def probs(self, out):
        return (out.float().flatten(1) @ self.head).softmax(1)


def caches(n, **kw):
    return [binding.Cache(L, HKV, G, D, BATCH, 64, 600, **kw) for _ in range(n)]


def prompt(cache, m, lens=(37, 64, 5)):
    g = torch.Generator(device="cuda").manual_seed(11)
    tokens = torch.randint(0, VOCAB, (sum(lens),), generator=g, device="cuda")
    for layer in range(L):
        k, v, _ = m.rows(layer, tokens)
        cache.append_chunk(layer, k, v, list(lens))


def test_steps_give_the_cache_and_outputs_of_plain_decoding():
    """Greedy steps over random trees: the tokens are those of one-by-one decoding, whatever the drafts were, and so is the cache."""
    m = Model()
    a, b = caches(2)
    for c in (a, b):
        prompt(c, m)
    # One by one.
    tok = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    plain = [[] for _ in range(BATCH)]
    for _ in range(40):
        for layer in range(L):
            k, v, q = m.rows(layer, tok)
            out = b.append_chunk_attn(layer, k, v, q, [1] * BATCH)
        tok = m.probs(out).argmax(1).to(torch.int32)
        for s, t in enumerate(tok.tolist()):
            plain[s].append(t)
    # In steps: drafts that know the answer in part.
    root, given = [1, 2, 3], [[] for _ in range(BATCH)]
    step = 0
    while min(len(x) for x in given) < 30:
        step += 1
        trees, tokens = [], []
        for s in range(BATCH):
            t = 1 + (step * 7 + s * 5) % 20
            parents = tree_ref.tree(t, 3, step * 31 + s, near=6)
            trees.append(parents)
            for j, p in enumerate(parents):
                d = len(given[s]) + tree_ref.depth(parents, j) - 1
                tokens.append(root[s] if p < 0 else plain[s][d] if d < 40 and (j + step) % 3 else (7 * j + step) % VOCAB)
        lens = [len(t) for t in trees]
        tokens = torch.tensor(tokens, dtype=torch.int32, device="cuda")
        parents = torch.tensor([p for t in trees for p in t], dtype=torch.int32, device="cuda")
        masks = a.tree_masks(parents, lens)
        for layer in range(L):
            k, v, q = m.rows(layer, tokens)
            out = a.append_tree_attn(layer, k, v, q, lens, masks)
        path, n, new = a.verify_tree_greedy(tokens, parents, lens, m.probs(out).argmax(1).to(torch.int32))
        a.commit_tree(lens, path, n)
        a.sync_lengths()
        for s in range(BATCH):
            given[s] += new[s, :n[s]].tolist()
            root[s] = given[s][-1]
    assert a.device_status()[0] == 0
    # Two decodings of the same function differ by rounding: a near tie may go the other way, and from there on the tokens differ.
    for s in range(BATCH):
        same = 0
        while same < 30 and given[s][same] == plain[s][same]:
            same += 1
        assert same == 30
    for layer in range(L):
        n = [min(x, y) for x, y in zip(a.lengths(layer), b.lengths(layer))]
        for s in range(BATCH):
            for h in range(HKV):
                for x, y in zip(a.export_head(layer, s, h), b.export_head(layer, s, h)):
                    assert torch.equal(x[:n[s]], y[:n[s]])


def sampled_step(cache, m, x, base, eager=None):
    """One step on the tensors of x; returns what it gives."""
    masks = cache.tree_masks(x["parents"], x["lens"])
    outs = []
    for layer in range(L):
        lse = torch.empty((sum(x["lens"]), HKV * G), device="cuda")
        out = cache.append_tree_attn(layer, *x["rows"][layer], x["lens"], masks, lse=lse)
        outs += [out, lse]
    found = cache.verify_tree(x["tokens"], x["parents"], x["lens"], m.probs(out), x["u"], x["us"], draft=x["draft"])
    cache.commit_tree(x["lens"], found[0], found[1])
    return outs + list(found)


def inputs(m, seed, lens):
    g = torch.Generator(device="cuda").manual_seed(seed)
    total = sum(lens)
    trees = [tree_ref.tree(t, 3, seed + s) for s, t in enumerate(lens)]
    tokens = torch.randint(0, VOCAB, (total,), generator=g, device="cuda", dtype=torch.int32)
    return dict(lens=lens, tokens=tokens, parents=torch.tensor([p for t in trees for p in t], dtype=torch.int32, device="cuda"),
                rows=[m.rows(i, tokens) for i in range(L)], u=torch.rand(total, generator=g, device="cuda") * 0.3, us=torch.rand(BATCH, generator=g, device="cuda"),
                draft=torch.rand((total, VOCAB), generator=g, device="cuda").softmax(1))


def test_a_captured_step_equals_eager_ones():
    m, lens = Model(1), [12, 0, 30]
    a, b = caches(2)
    for c in (a, b):
        prompt(c, m)
    x = inputs(m, 5, lens)
    sampled_step(b, m, x, None)   # (warm: kernels of both ways have run)
    b.reset()
    prompt(b, m)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = sampled_step(a, m, x, None)
    for seed in (5, 6, 7):   # other inputs in the same tensors
        new = inputs(m, seed, lens)
        for name in ("tokens", "u", "us", "draft", "parents"):
            x[name].copy_(new[name])
        for i in range(L):
            for to, frm in zip(x["rows"][i], new["rows"][i]):
                to.copy_(frm)
        graph.replay()
        want = sampled_step(b, m, new, None)
        b.sync_lengths()
        torch.cuda.synchronize()
        for p, q in zip(outs, want):
            assert torch.equal(p, q)
    a.sync_lengths()
    assert a.device_status()[0] == 0 and [a.lengths(i) for i in range(L)] == [b.lengths(i) for i in range(L)]
    for layer in range(L):
        for x1, y1 in zip(a.export_chunk(layer, a.lengths(layer)), b.export_chunk(layer, b.lengths(layer))):
            assert torch.equal(x1, y1)


def test_features_of_the_accepted_path_and_an_eviction_follow():
    """The accepted nodes' queries and log-sum-exps give the features that the same tokens give as a chunk."""
    m, lens = Model(2), [14, 9, 0]
    a, b = caches(2)
    for c in (a, b):
        prompt(c, m)
    x = inputs(m, 9, lens)
    paths = [[0, 1], [0], []]
    outs = []
    masks = a.tree_masks(x["parents"], lens)
    for layer in range(L):
        lse = torch.empty((sum(lens), HKV * G), device="cuda")
        out = a.append_tree_attn(layer, *x["rows"][layer], lens, masks, lse=lse)
        outs.append((out, lse))
    path = torch.full((BATCH, 14), -1, dtype=torch.int32)
    for s, p in enumerate(paths):
        path[s, :len(p)] = torch.tensor(p, dtype=torch.int32)
    n = [len(p) for p in paths]
    a.commit_tree(lens, path.cuda(), torch.tensor(n, dtype=torch.int32, device="cuda"))
    a.sync_lengths()
    rows = torch.tensor([0, 1, 14], device="cuda")   # packed indices of the accepted nodes
    for layer in range(L):
        k, v, q = (y[rows].contiguous() for y in x["rows"][layer])
        lse = torch.empty((3, HKV * G), device="cuda")
        out = b.append_chunk_attn(layer, k, v, q, n, lse=lse)
        assert float((out.float() - outs[layer][0][rows].float()).abs().max()) < 2e-2 and float((lse - outs[layer][1][rows]).abs().max()) < 1e-5
        a.chunk_features(layer, q, outs[layer][1][rows].contiguous(), n)
        b.chunk_features(layer, q, lse, n)
        for s in range(2):
            f, h = a.export_features(layer, s), b.export_features(layer, s)
            assert f.shape == h.shape and float((f - h).abs().max()) < 1e-5 * float(h.abs().max())
    for c in (a, b):
        c.set_budget(1, 40)
        c.evict_by_feature(4)
    assert [a.lengths(i) for i in range(L)] == [b.lengths(i) for i in range(L)] == [[39, 40, 5]] * L
    k, v, q = (y[:BATCH].contiguous() for y in x["rows"][0])
    assert float((a.append_decode_attn(0, k, v, q).float() - b.append_decode_attn(0, k, v, q).float()).abs().max()) < 2e-2
    assert a.device_status()[0] == 0


def test_decode_queries_of_dropped_trees_leave_the_record():
    """A decode token behind a tree that is then committed: its query saw pairs that are gone, so it leaves the record."""
    m = Model(3)
    a, b = caches(2, feature_window=16)
    for c in (a, b):
        prompt(c, m)
    tok = torch.tensor([4, 5, 6], dtype=torch.int32, device="cuda")
    k, v, q = m.rows(0, tok)
    for c in (a, b):
        c.append_decode_attn(0, k, v, q)
    lens = [6, 0, 3]
    x = inputs(m, 3, lens)
    n = a.lengths(0)
    masks = a.tree_masks(x["parents"], lens)
    kk, vv, _ = x["rows"][0]
    a.append_tree(0, kk, vv, lens, masks)
    a.append_decode_attn(0, k, v, q, seq_mask=0b101)   # (with the pair it appends, 7 and 4 behind the first token's)
    a.commit_tree([7, 0, 4], torch.full((BATCH, 8), -1, dtype=torch.int32, device="cuda"), torch.zeros(BATCH, dtype=torch.int32, device="cuda"), layer=0)
    a.sync_lengths()
    assert a.lengths(0) == n
    for c in (a, b):
        c.update_features(0)
    for s in range(BATCH):
        assert torch.equal(a.export_features(0, s), b.export_features(0, s))
