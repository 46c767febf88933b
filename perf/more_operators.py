"""Cases and plain forms of the operators of a speculative decoder on the paged cache.

  tree    attention of the nodes of a draft tree, stored behind a sequence's pairs: a node sees the pairs before the tree
          (optionally only a sliding window of positions and a few first positions, the sinks), its ancestors and itself;
  verify  which drafted tokens stand, and the token after them: from the root down, a child of node a with token x is
          accepted if u q_a(x) < R(x), R being the target's probabilities after a; a rejection makes R the normalised
          positive part of R - q_a; behind the last child the next token is drawn from R.  Without draft probabilities the
          children are point masses: u m < p_a(x) with m the mass that no rejected sibling holds;
  step    one step of a decoder over several layers: tree attention, verification, and the accepted path's pairs moved
          together behind the pairs before the tree, in all layers;
  fork    every sequence becomes what another one was, or empty: one prompt for several samples, beams, finished requests.

``run`` computes them in elementary torch operations over dense padded tensors; with ``own`` set it calls the library.
A tree's nodes are in an order in which parents come first; node 0 is its root, the token that the step before gave.
"""
import math
import random

import torch

own = False


def _tree(name, kind, seqs, n, nodes, fan, kv_heads, group, dim, window=0, sinks=0, ragged=False, layers=1, vocab=0, sampled=True,
          dtype="float32"):
    c = {"kind": kind, "seqs": seqs, "n": n, "nodes": nodes, "fan": fan, "kv_heads": kv_heads, "group": group, "dim": dim,
         "window": window, "sinks": sinks, "ragged": ragged, "layers": layers, "vocab": vocab, "sampled": sampled, "dtype": dtype}
    return {"name": name, **c} if name else c


def _verify(name, seqs, nodes, fan, vocab, sampled=True, dtype="float32", ragged=False):
    c = {"kind": "verify", "seqs": seqs, "nodes": nodes, "fan": fan, "vocab": vocab, "sampled": sampled, "dtype": dtype, "ragged": ragged}
    return {"name": name, **c} if name else c


def _fork(name, seqs, n, kv_heads, group, dim, layers, shape, ragged=False):
    c = {"kind": "fork", "seqs": seqs, "n": n, "kv_heads": kv_heads, "group": group, "dim": dim, "layers": layers, "shape": shape,
         "ragged": ragged}
    return {"name": name, **c} if name else c


def listed():
    return [
        # A tree of 16 drafts of one sequence over an 8K cache, one layer: latency of the smallest call.
        _tree("tree of 16, one sequence", "tree", 1, 8192, 16, 3, 8, 4, 128),
        # Trees of up to 64 nodes for a batch of 16 uneven long caches, seven query heads to a KV head: the largest call.
        _tree("trees of 64, batch of 16", "tree", 16, 32768, 64, 4, 4, 7, 128, ragged=True),
        # The widest tree, in a layer with a sliding window and four sinks.
        _tree("tree of 256, window 4096", "tree", 1, 30720, 256, 6, 8, 4, 128, window=4096, sinks=4),
        # Uneven trees behind small caches with 64 channels.
        _tree("small trees, small caches", "tree", 3, 512, 33, 2, 2, 4, 64, ragged=True),
        # Five drafts in a row of one sequence, drawn from a draft model: latency.
        _verify("drafts of 5, one sequence", 1, 6, 1, 130001),
        # Trees whose siblings are drawn from one distribution: several passes over a node's rows.
        _verify("trees of 32, batch of 16", 16, 32, 4, 130001, ragged=True),
        # Likeliest tokens of a draft head as drafts, probabilities in 16 bits, a large batch.
        _verify("likeliest 7, batch of 64", 64, 8, 1, 130001, sampled=False, dtype="bfloat16"),
        # A step of one sequence over four layers, with the host reading the lengths at its end.
        _tree("step, one sequence", "step", 1, 8192, 16, 3, 8, 4, 128, layers=4, vocab=32003),
        # A step of a batch of uneven sequences.
        _tree("step, batch of 8", "step", 8, 8192, 32, 4, 4, 7, 128, ragged=True, layers=2, vocab=32003, sampled=False),
        # A prompt of 8K for four samples.
        _fork("fork, one to four", 4, 8192, 8, 4, 128, 2, "one"),
        # A batch of beams: some go on twice, some end.
        _fork("beams, batch of 16", 16, 4096, 4, 7, 128, 1, "beams", ragged=True),
        # A small pruned cache: latency.
        _fork("fork, small cache", 3, 300, 2, 4, 64, 1, "one"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("tree", "tree", "verify", "step", "fork"))
    heads, group, dim, dtype = rng.choice((1, 2, 4, 8)), rng.randint(1, 8), rng.choice((64, 128)), rng.choice(("float32", "bfloat16"))
    ragged, sampled = rng.random() < 0.7, rng.random() < 0.6
    if kind == "verify":
        seqs, nodes, vocab = log(1, 64), log(1, 256), log(1000, 130001)
        while seqs * nodes * vocab > 2 ** 26:
            seqs, nodes = (seqs + 1) // 2, (nodes + 1) // 2
        return _verify("", seqs, nodes, rng.randint(1, 6), vocab, sampled, dtype, ragged)
    if kind == "fork":
        seqs, n, layers = log(2, 16), log(1, 8192), rng.randint(1, 4)
        while seqs * n * heads * dim * layers > 2 ** 26:
            n = (n + 1) // 2
        return _fork("", seqs, n, heads, group, dim, layers, rng.choice(("one", "beams")), ragged)
    seqs, n, nodes, layers = log(1, 16), log(1, 32768), log(1, 256), rng.randint(2, 4) if kind == "step" else 1
    window = log(max(256, nodes), 8192) if rng.random() < 0.3 else 0
    while seqs * heads * group * nodes * (n + nodes) * layers > 2 ** 29 or seqs * heads * (n + nodes) * dim * layers > 2 ** 28:
        seqs, n = (seqs + 1) // 2, (n + 1) // 2
    return _tree("", kind, seqs, n, nodes, rng.randint(1, 6), heads, group, dim, window, rng.choice((0, 1, 4, 16, 64)) if window else 0,
                 ragged, layers, log(1000, 32003) if kind == "step" else 0, sampled, dtype)


def _lengths(case):
    """Pairs stored before the call, and nodes of the tree, of every sequence."""
    n, t = case.get("n", 0), case.get("nodes", 0)
    if not case["ragged"]:
        return [n] * case["seqs"], [t] * case["seqs"]
    # (every fifth slot of a ragged batch has no tree in this step)
    return ([n * (100 - s * 29 % 88) // 100 for s in range(case["seqs"])],
            [0 if s % 5 == 3 else max(1, t * (100 - s * 37 % 75) // 100) for s in range(case["seqs"])])


def _parents(case):
    """Per sequence the parent of every node: at most `fan` children to a node, shallow trees and deep ones."""
    rng = random.Random("%(seqs)s %(nodes)s %(fan)s" % case)
    trees = []
    for t in _lengths(case)[1]:
        children, parents, near = [], [], rng.choice((2, 6, 1000))
        for j in range(t):
            free = [i for i in range(j) if children[i] < case["fan"]][-near:]
            parents.append(rng.choice(free) if j else -1)
            if j:
                children[parents[j]] += 1
            children.append(0)
        trees.append(parents)
    return trees


def _sources(case):
    """For every sequence the one that it becomes (the same again when it is applied twice), -1: empty."""
    if case["shape"] == "one":
        return [0] * case["seqs"]
    return [s if s % 4 == 0 else -1 if s % 8 == 7 else s // 4 * 4 if s % 4 < 3 else s // 8 * 8 for s in range(case["seqs"])]


def _depths(parents):
    d = []
    for p in parents:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 29)
    dev, bf, kind = "cuda", torch.bfloat16, case["kind"]
    st = {"case": case}
    stored, nodes = _lengths(case)
    if kind != "fork":
        trees = _parents(case)
        total = sum(nodes)
        st["lens"], st["keep"] = nodes, stored
        st["parents"] = torch.tensor([p for t in trees for p in t], dtype=torch.int32, device=dev)
        st["t_len"] = torch.tensor(nodes, device=dev)
        st["first"] = st["t_len"].cumsum(0) - st["t_len"]
        st["row_seq"] = torch.repeat_interleave(torch.arange(case["seqs"], device=dev), st["t_len"])
        st["row_node"] = torch.arange(total, device=dev) - st["first"][st["row_seq"]]
        st["deepest"] = 1 + max(max(_depths(t), default=-1) for t in trees)   # nodes on the longest path
    if kind in ("verify", "step"):
        # The target agrees with the draft model up to some noise.
        v, dt = case["vocab"], getattr(torch, case["dtype"])
        logits = torch.randn((total, v), generator=g, device=dev) * 3
        draft = logits.softmax(1)
        logits += torch.randn(logits.shape, generator=g, device=dev) * 0.7
        st["target"] = logits.softmax(1).to(dt)
        up = st["parents"].long() + st["first"][st["row_seq"]]
        rank = [sum(q == p for q in t[:j]) for t in trees for j, p in enumerate(t)]
        if case["sampled"]:
            st["draft"] = draft = draft.to(dt)
            near = torch.multinomial(draft.float(), case["fan"], replacement=True, generator=g) if total else None
        else:
            near = draft.topk(case["fan"], dim=1).indices if total else None
        del logits, draft
        st["tokens"] = near[up.clamp(min=0), torch.tensor(rank, device=dev)].to(torch.int32) if total else torch.empty(0, dtype=torch.int32, device=dev)
        st["u_accept"] = torch.rand(total, generator=g, device=dev)
        st["u_sample"] = torch.rand(case["seqs"], generator=g, device=dev)
    if kind == "verify":
        if own:
            from paper_2602_03203_b200 import binding
            st["cache"] = binding.Cache(1, 1, 1, 64, case["seqs"], 16, 16)
        return st
    # The cache: keys carry a scale of their own in every channel, as rotated keys do.
    b, hk, grp, dim, layers = case["seqs"], case["kv_heads"], case["group"], case["dim"], case["layers"]
    width = max(stored) + (max(nodes) if nodes else 0)
    scale = torch.exp(torch.randn((1, hk, 1, dim), generator=g, device=dev))
    k = [(torch.randn((b, hk, width, dim), generator=g, device=dev) * scale).to(bf) for _ in range(layers)]
    v = [torch.randn((b, hk, width, dim), generator=g, device=dev).to(bf) for _ in range(layers)]
    s_len = torch.tensor(stored, device=dev)
    # Positions of a pruned cache have gaps; the first ones have none.
    step = torch.randint(1, 4, (b, width), generator=g, device=dev)
    step[:, : 65] = 1
    pos = (step.cumsum(1) - 1).to(torch.int32)
    st["stored"] = s_len
    if kind == "fork":
        st["source"] = _sources(case)
        st["new_lens"] = [stored[r] if r >= 0 else 0 for r in st["source"]]
        f = [torch.rand((b, hk, width, 6 * grp), generator=g, device=dev) for _ in range(layers)]
    else:
        f = [None] * layers
        st["q"] = [torch.randn((total, hk * grp, dim), generator=g, device=dev).to(bf) for _ in range(layers)]
        st["k_new"] = [(torch.randn((total, hk, dim), generator=g, device=dev) * scale[0, :, 0]).to(bf) for _ in range(layers)]
        st["v_new"] = [torch.randn((total, hk, dim), generator=g, device=dev).to(bf) for _ in range(layers)]
    if own:
        from paper_2602_03203_b200 import binding
        cache = binding.Cache(layers, hk, grp, dim, b, 16, width)
        for i in range(layers):
            for s, m in enumerate(stored):
                if m:
                    cache.prefill(i, s, k[i][s, :, :m].contiguous(), v[i][s, :, :m].contiguous(),
                                  None if f[i] is None else f[i][s, :, :m].contiguous(), pos[s, :m].contiguous())
        st["cache"] = cache
        if kind == "tree":   # a program that runs the layers of a step has the tree's masks in hand
            st["masks"] = cache.tree_masks(st["parents"], nodes)
    else:
        st["k"], st["v"], st["f"], st["pos"] = k, v, f, pos
        if kind == "tree":
            st["ancestors"] = _ancestors(st)
    return st


def _ancestors(st):
    """[row][node]: whether a node is on the path from a row's node up to the root; packed rows."""
    t = max(st["lens"], default=0)
    at = st["row_node"].clone()
    seen = torch.zeros((len(at), t), dtype=torch.bool, device=at.device)
    for _ in range(st["deepest"]):
        seen[torch.arange(len(at), device=at.device), at] = True
        up = st["parents"][st["first"][st["row_seq"]] + at].long()
        at = torch.where(up < 0, at, up)
    return seen


def _attend(st, layer, ancestors):
    """Stores the tree's pairs and attends, in 32 bits: out and log-sum-exp, packed."""
    c, row, node = st["case"], st["row_seq"], st["row_node"]
    b, hk, grp, dim, t, w = c["seqs"], c["kv_heads"], c["group"], c["dim"], max(st["lens"]), c["window"]
    k, v, pos = st["k"][layer], st["v"][layer], st["pos"].long()
    width, slot = k.shape[2], st["stored"][row] + node
    k[row, :, slot] = st["k_new"][layer]
    v[row, :, slot] = st["v_new"][layer]
    # Own position: behind the last stored pair, one further with every step down the tree.
    last = torch.where(st["stored"] > 0, pos.gather(1, (st["stored"] - 1).clamp(min=0)[:, None])[:, 0], torch.full_like(st["stored"], -1))
    own_pos = last[row] + ancestors.sum(1)
    at = torch.arange(width, device=k.device)
    before = at < st["stored"][row][:, None]
    if w:
        before = before & ((own_pos[:, None] - pos[row] < w) | (pos[row] < c["sinks"]))
    in_tree = at - st["stored"][row][:, None]
    inside = (in_tree >= 0) & (in_tree < st["t_len"][row][:, None])
    seen = before | (inside & ancestors.gather(1, in_tree.clamp(0, t - 1)))
    q = st["q"][layer].float().new_zeros((b, t, hk * grp, dim))
    q[row, node] = st["q"][layer].float()
    mask = torch.zeros((b, t, width), dtype=torch.bool, device=k.device)
    mask[row, node] = seen
    q = q.reshape(b, t, hk, grp, dim).permute(0, 2, 3, 1, 4).reshape(b, hk, grp * t, dim)
    s = (q @ k.float().transpose(2, 3)).mul_(dim ** -0.5).reshape(b, hk, grp, t, width)
    s.masked_fill_(~mask[:, None, None], -math.inf)
    m = s.amax(4, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    total = p.sum(4, keepdim=True)
    o = (p.reshape(b, hk, grp * t, width) @ v.float()).reshape(b, hk, grp, t, dim)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (m + total.log())[..., 0]
    o = o.permute(0, 3, 1, 2, 4).reshape(b, t, hk * grp, dim)[row, node]
    return [o.to(torch.bfloat16), lse.permute(0, 3, 1, 2).reshape(b, t, hk * grp)[row, node], own_pos]


def _verified(st):
    """Accepted nodes [sequence][path] (-1 behind the last), their number, and the tokens that the step gives; in 64 bits."""
    c, dev = st["case"], st["parents"].device
    b, t, fan = c["seqs"], max(st["lens"]), c["fan"]
    seq, row, node, up = torch.arange(b, device=dev), st["row_seq"], st["row_node"], st["parents"].long()
    # child[sequence][node][rank]: packed row of that child, or -1.
    same = (up[:, None] == up[None]) & (row[:, None] == row[None])
    rank = torch.tril(same, -1).sum(1)
    child = torch.full((b, t, max(fan, 1)), -1, device=dev)
    below = up >= 0
    child[row[below], up[below], rank[below]] = torch.arange(len(up), device=dev)[below]
    target, draft = st["target"], st.get("draft")
    alive = st["t_len"] > 0
    cur = torch.zeros(b, dtype=torch.long, device=dev)
    final = torch.zeros((b, c["vocab"]), dtype=torch.float64, device=dev)
    path = torch.full((b, t), -1, dtype=torch.int32, device=dev)
    tokens = torch.full((b, t), -1, dtype=torch.int32, device=dev)
    count = torch.zeros(b, dtype=torch.long, device=dev)
    for _ in range(st["deepest"]):
        path[seq[alive], count[alive]] = cur[alive].to(torch.int32)
        count = count + alive
        at = (st["first"] + cur).clamp(max=len(up) - 1)
        p = target[at].double()
        r, q = p, None if draft is None else draft[at].double()
        mass, done, nxt = torch.ones(b, dtype=torch.float64, device=dev), torch.zeros_like(alive), cur
        for i in range(fan):
            ch = child[seq, cur, i]
            has = alive & ~done & (ch >= 0)
            x = st["tokens"][ch.clamp(min=0)].long()[:, None]
            px, u = r.gather(1, x)[:, 0], st["u_accept"][ch.clamp(min=0)].double()
            ok = has & (u * (mass if q is None else q.gather(1, x)[:, 0]) < px)
            lost = has & ~ok
            if q is None:
                mass = torch.where(lost, mass - px, mass)
                r = torch.where(lost[:, None], r.scatter(1, x, 0.0), r)
            else:
                left = (r - q).clamp(min=0)
                z = left.sum(1, keepdim=True)
                r = torch.where(lost[:, None], torch.where(z > 0, left / z, p), r)
            nxt = torch.where(ok, node[ch.clamp(min=0)], nxt)
            token = torch.where(ok, x[:, 0], torch.full_like(nxt, -1)).to(torch.int32)
            tokens[seq[ok], count[ok] - 1] = token[ok]
            done = done | ok
        final = torch.where((alive & ~done)[:, None], r, final)
        alive, cur = alive & done, nxt
    sums = final.cumsum(1)
    last = c["vocab"] - 1 - (final > 0).flip(1).to(torch.uint8).argmax(1)
    drawn = torch.minimum((sums <= st["u_sample"].double()[:, None] * sums[:, -1:]).sum(1), last)
    drawn = torch.where(sums[:, -1] > 0, drawn, torch.full_like(drawn, -1)).to(torch.int32)
    some = st["t_len"] > 0
    tokens[seq[some], count[some] - 1] = drawn[some]
    return [path, count.to(torch.int32), tokens]


def _step(st):
    ancestors = _ancestors(st)
    outs, c = [], st["case"]
    layers = range(c["layers"])
    for i in layers:
        o, lse, own_pos = _attend(st, i, ancestors)
        outs += [o, lse]
    path, count, tokens = _verified(st)
    # The accepted pairs move together, in every layer.
    seq, j = (path >= 0).nonzero(as_tuple=True)
    src = path[seq, j].long()
    packed = st["first"][seq] + src
    for i in layers:   # (as many rows as there are nodes, zeros behind the accepted ones)
        for x, new in ((st["k"][i], st["k_new"][i]), (st["v"][i], st["v_new"][i])):
            x[seq, :, st["stored"][seq] + j] = new[packed]
            outs.append(torch.zeros_like(new))
            outs[-1][: len(seq)] = x[seq, :, st["stored"][seq] + j]
    pos = st["parents"].new_zeros((len(own_pos), c["kv_heads"]))
    pos[: len(seq)] = own_pos[packed, None].to(torch.int32)
    return outs + [pos, path, count, tokens, count + st["stored"].to(torch.int32)]


def run(st):
    c, kind = st["case"], st["case"]["kind"]
    if own:
        cache = st["cache"]
        if kind == "tree":
            lse = torch.empty(st["q"][0].shape[:2], device="cuda")
            out = cache.append_tree_attn(0, st["k_new"][0], st["v_new"][0], st["q"][0], st["lens"], st["masks"], keep_lens=st["keep"],
                                         window=c["window"], sinks=c["sinks"], lse=lse)
            return [out, lse]
        if kind == "fork":
            cache.fork(st["source"])
            return [x for i in range(c["layers"]) for x in cache.export_chunk(i, st["new_lens"])]
        checked = dict(draft=st.get("draft"))
        if kind == "verify":
            return list(cache.verify_tree(st["tokens"], st["parents"], st["lens"], st["target"], st["u_accept"], st["u_sample"], **checked))
        masks = cache.tree_masks(st["parents"], st["lens"])
        outs = []
        for i in range(c["layers"]):
            lse = torch.empty(st["q"][i].shape[:2], device="cuda")
            outs += [cache.append_tree_attn(i, st["k_new"][i], st["v_new"][i], st["q"][i], st["lens"], masks, keep_lens=st["keep"],
                                            window=c["window"], sinks=c["sinks"], lse=lse), lse]
        found = cache.verify_tree(st["tokens"], st["parents"], st["lens"], st["target"], st["u_accept"], st["u_sample"], **checked)
        cache.commit_tree(st["lens"], found[0], found[1])
        cache.sync_lengths()   # the host reads how far every sequence has come
        now = cache.lengths(0)
        accepted = [m - n for m, n in zip(now, st["keep"])]
        m, pos = sum(accepted), st["parents"].new_zeros((len(st["parents"]), c["kv_heads"]))
        for i in range(c["layers"]):   # (as many rows as there are nodes, zeros behind the accepted ones)
            k, v = torch.zeros_like(st["k_new"][i]), torch.zeros_like(st["v_new"][i])
            cache.export_chunk(i, accepted, (k[:m], v[:m], None, pos[:m]))
            outs += [k, v]
        return outs + [pos, *found, torch.tensor(now, dtype=torch.int32)]
    if kind == "tree":
        return _attend(st, 0, st["ancestors"])[:2]
    if kind == "verify":
        return _verified(st)
    if kind == "step":
        outs = _step(st)
        return outs[:-1] + [outs[-1].cpu()]
    src = torch.tensor([max(r, 0) for r in st["source"]], device="cuda")
    new = torch.tensor(st["new_lens"], device="cuda")
    seq = torch.repeat_interleave(torch.arange(c["seqs"], device="cuda"), new)
    slot = torch.arange(len(seq), device="cuda") - (new.cumsum(0) - new)[seq]
    outs = []
    for i in range(c["layers"]):
        outs += [x[i][src][seq, :, slot] for x in (st["k"], st["v"], st["f"])] + [st["pos"][src][seq, slot, None].expand(-1, c["kv_heads"])]
    return outs


def work(case):
    kind = case["kind"]
    stored, nodes = _lengths(case)
    size = 2 if case.get("dtype") == "bfloat16" else 4
    nbytes = flops = 0
    if kind in ("verify", "step"):
        # A sequence's last node has its row read (with the draft's); its path depends on the numbers.
        rows = sum(t > 0 for t in nodes) * (2 if case["sampled"] else 1)
        nbytes += rows * case["vocab"] * size + sum(nodes) * (12 + 2 * size) + sum(t > 0 for t in nodes) * 4 + case["seqs"] * (8 * max(nodes) + 4)
        flops += 2 * rows * case["vocab"]
    if kind in ("tree", "step"):
        hk, grp, dim, w = case["kv_heads"], case["group"], case["dim"], case["window"]
        for n, t, parents in zip(stored, nodes, _parents(case)):
            if not t:
                continue
            seen = min(n, w // 2 + min(case["sinks"], n)) if w else n   # (positions are two apart in the mean)
            scores = sum(seen + d + 1 for d in _depths(parents))
            per = hk * (seen + t) * dim * 4 + 2 * t * hk * grp * dim * 2 + t * (hk * dim * 4 + hk * grp * 4) + t * (4 if kind == "step" else 32)
            if kind == "step":
                per += hk * dim * 8   # one pair at least comes back
            nbytes += per * case["layers"]
            flops += 4 * hk * grp * scores * dim * case["layers"]
    if kind == "fork":
        pair = case["kv_heads"] * (case["dim"] * 4 + case["group"] * 24) + 4
        source = _sources(case)
        copied = [r for s, r in enumerate(source) if r not in (-1, s)]
        new = sum(stored[r] for r in source if r >= 0)
        # The sources that are copied once, their copies, and the read-out.
        nbytes += case["layers"] * pair * (sum(stored[r] for r in set(copied)) + sum(stored[r] for r in copied) + 2 * new)
    return {"bytes": nbytes, "flops": flops}


def _exact_attention(st, layer, trees):
    """Per sequence and head in 64 bits, a node's own path walked."""
    case = st["case"]
    hk, grp, dim, w = case["kv_heads"], case["group"], case["dim"], case["window"]
    outs, lses, row = [], [], 0
    for s, parents in enumerate(trees):
        n, t = st["keep"][s], len(parents)
        pos = st["pos"][s, :n].double()
        o = torch.zeros((t, hk * grp, dim), dtype=torch.float64, device="cuda")
        lse = torch.zeros((t, hk * grp), dtype=torch.float64, device="cuda")
        hidden = torch.ones((t, n + t), dtype=torch.bool, device="cuda")
        depth = _depths(parents)
        here = torch.tensor(depth, dtype=torch.float64, device="cuda") + ((pos[-1] if n else -1) + 1)
        hidden[:, :n] = ((here[:, None] - pos >= w) & (pos >= case["sinks"])) if w else False
        on = [(j, i) for j in range(t) for i in _path_up(parents, j)]
        if on:
            a, b = torch.tensor(on, device="cuda").T
            hidden[a, n + b] = False
        for h in range(hk * grp if t else 0):
            keys = torch.cat([st["k"][layer][s, h // grp, :n], st["k_new"][layer][row: row + t, h // grp]]).double()
            vals = torch.cat([st["v"][layer][s, h // grp, :n], st["v_new"][layer][row: row + t, h // grp]]).double()
            z = torch.einsum("td,nd->tn", st["q"][layer][row: row + t, h].double(), keys) / math.sqrt(dim)
            z[hidden] = -math.inf
            lse[:, h] = torch.logsumexp(z, 1)
            o[:, h] = torch.exp(z - lse[:, h: h + 1]) @ vals
        row += t
        outs.append(o)
        lses.append(lse)
    return [torch.cat(outs), torch.cat(lses)]


def _path_up(parents, j):
    while j >= 0:
        yield j
        j = parents[j]


def exact(case, seed):
    """The attention's definition in 64 bits, and a fork's copies one sequence after another.  What a verification gives is whole
    numbers, and the accepted pairs are copies of the new ones: they have no rounded value."""
    global own
    if case["kind"] == "verify":
        return None
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "fork":
        outs = []
        for i in range(case["layers"]):
            kept = [(r, n) for r, n in zip(st["source"], st["new_lens"]) if n]
            outs += [torch.cat([x[i][r, :, :n].transpose(0, 1).double() for r, n in kept]) for x in (st["k"], st["v"], st["f"])] + [None]
        return outs
    trees = _parents(case)
    outs = [x for i in range(case["layers"]) for x in _exact_attention(st, i, trees)]
    return outs if case["kind"] == "tree" else outs + [None] * (2 * case["layers"] + 5)
