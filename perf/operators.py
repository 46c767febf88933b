"""Cases and plain forms of the chunk and window operators of the paged cache.

Three operators work on one layer of a cache of (key, value) pairs, stored per sequence and KV head in position order:

  chunk     store a chunk of new tokens behind the pairs that stay, and attend from every one of them over all pairs up
            to its own (optionally only a sliding window of positions and a few first positions, the sinks);
  window    attention of one decode token per sequence over a sliding window of positions and the sinks;
  features  the attention features of every pair (means over the last 8 / 16 / 32 queries and over the chunk, the sum
            and the decayed sum over chunks) from the queries of a chunk and their log-sum-exp.

``run`` computes them in elementary torch operations in 32 bits, over dense padded tensors; with ``own`` set it calls
the library.  A query of position p sees a stored pair of position x if the pair is not behind the query's own pair and
(window == 0, or p - x < window, or x < sinks).
"""
import math

import torch

own = False

#: Last 8 / 16 / 32 queries; the fourth window of the features is the whole chunk.
WINDOWS = (8, 16, 32)
DECAY = 0.9


def _case(name, kind, seqs, n, chunk, kv_heads, group, dim, window=0, sinks=0, gap=1, ragged=False):
    c = {"kind": kind, "seqs": seqs, "n": n, "chunk": chunk, "kv_heads": kv_heads, "group": group, "dim": dim,
         "window": window, "sinks": sinks, "gap": gap, "ragged": ragged}
    return {"name": name, **c} if name else c


def listed():
    return [
        # Five draft tokens of a speculative decoder are checked against an 8K cache: latency of the smallest call.
        _case("drafts, one sequence", "chunk", 1, 8192, 5, 8, 4, 128),
        # The same for a batch of 16 sequences of uneven lengths and drafts, seven query heads to a KV head.
        _case("drafts, batch of 16", "chunk", 16, 32768, 8, 4, 7, 128, ragged=True),
        # Uneven short chunks behind small caches with 64 channels.
        _case("short chunks, small caches", "chunk", 3, 512, 33, 2, 4, 64, ragged=True),
        # One update length of prompt behind an 8K cache.
        _case("256 tokens at 8K", "chunk", 1, 8192, 256, 8, 4, 128),
        # A chunk of a long prompt: the largest call.
        _case("2048 tokens at 32K", "chunk", 1, 30720, 2048, 8, 4, 128),
        # A chunk of a long prompt in a layer with a sliding window and four sinks.
        _case("2048 tokens, window 4096", "chunk", 1, 14336, 2048, 8, 4, 128, window=4096, sinks=4),
        # A decode token in a layer with a sliding window: latency.
        _case("window step, one sequence", "window", 1, 32768, 1, 8, 4, 128, window=4096, sinks=4),
        # A decode token for 16 pruned caches: positions with gaps, uneven lengths.
        _case("window step, pruned batch", "window", 16, 32768, 1, 4, 7, 128, window=4096, sinks=4, gap=3, ragged=True),
        # A decode token for a large batch.
        _case("window step, batch of 64", "window", 64, 8192, 1, 8, 4, 128, window=4096, sinks=4),
        # The features of an 8K cache after a chunk of 128 queries.
        _case("features, 128 at 8K", "features", 1, 8192, 128, 8, 4, 128),
        # The features of a long prompt's cache after its last chunk: what a one-shot compression scores.
        _case("features, 2048 at 32K", "features", 1, 30720, 2048, 8, 4, 128),
        # Uneven chunks over pruned caches in a layer with a window, seven heads of 64 channels.
        _case("features, window, ragged", "features", 3, 4096, 300, 2, 7, 64, window=1024, sinks=4, gap=2, ragged=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("chunk", "window", "features"))
    seqs, n, chunk = log(1, 16), log(1, 30720), log(1, 2048)
    if kind == "window":
        seqs, chunk = log(1, 64), 1
    elif rng.random() < 0.1:
        n = 0   # the first chunk of a prompt
    heads, group, dim = rng.choice((1, 2, 4, 8)), rng.randint(1, 8), rng.choice((64, 128))
    window = log(1, 8192) if kind == "window" or rng.random() < 0.5 else 0
    sinks = rng.choice((0, 1, 4, 16, 64)) if window else 0
    gap = rng.choice((1, 1, 2, 3))
    while True:   # no larger than the largest listed case
        if seqs * heads * group * chunk * (n + chunk) > 2 ** 31:
            if seqs > 1:
                seqs = (seqs + 1) // 2
            else:
                chunk = (chunk + 1) // 2
        elif seqs * heads * (n + chunk) * dim > 2 ** 29:
            seqs = (seqs + 1) // 2
        else:
            break
    return _case("", kind, seqs, n, chunk, heads, group, dim, window, sinks, gap, seqs > 1 and rng.random() < 0.7)


def _lengths(case):
    """Pairs stored before the call and new tokens of every sequence."""
    n, t, kind = case["n"], case["chunk"], case["kind"]
    if not case["ragged"]:
        stored, fresh = [n] * case["seqs"], [t] * case["seqs"]
    else:
        stored = [n * (100 - s * 29 % 88) // 100 for s in range(case["seqs"])]
        # (every fifth slot of a ragged batch has no new tokens in this step)
        fresh = [0 if s % 5 == 3 else max(1, t * (100 - s * 37 % 75) // 100) for s in range(case["seqs"])]
    if kind == "window":
        return [max(1, x) for x in stored], [0] * case["seqs"]
    return stored, fresh


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 17)
    dev, bf = "cuda", torch.bfloat16
    b, hk, grp, dim = case["seqs"], case["kv_heads"], case["group"], case["dim"]
    stored, fresh = _lengths(case)
    n, t = max(stored), max(fresh)
    width, total = n + t, sum(fresh)
    # Keys carry a scale of their own in every channel, as rotated keys do.
    scale = torch.exp(torch.randn((1, hk, 1, dim), generator=g, device=dev))
    k = (torch.randn((b, hk, width, dim), generator=g, device=dev) * scale).to(bf)
    v = torch.randn((b, hk, width, dim), generator=g, device=dev).to(bf)
    # Positions of a pruned cache have gaps; the first ones and the chunk's own have none.
    step = torch.randint(1, 2 * case["gap"], (b, width), generator=g, device=dev)
    step[:, : case["sinks"] + 1] = 1
    at = torch.arange(width, device=dev)
    s_len = torch.tensor(stored, device=dev)
    t_len = torch.tensor(fresh, device=dev)
    step = torch.where(at[None] >= s_len[:, None], torch.ones_like(step), step)
    pos = (step.cumsum(1) - 1).to(torch.int32)
    state = {"case": case, "pos": pos, "stored": s_len, "fresh": t_len, "lens": fresh, "keep": stored}
    if case["kind"] == "window":
        state["q"] = torch.randn((b, hk * grp, dim), generator=g, device=dev).to(bf)
        state["row_seq"] = torch.arange(b, device=dev)
        state["row_slot"] = s_len - 1
        state["row_tok"] = torch.zeros(b, dtype=torch.long, device=dev)
    else:
        state["q"] = torch.randn((total, hk * grp, dim), generator=g, device=dev).to(bf)
        state["row_seq"] = torch.repeat_interleave(torch.arange(b, device=dev), t_len)
        state["row_tok"] = torch.arange(total, device=dev) - (t_len.cumsum(0) - t_len)[state["row_seq"]]
        state["row_slot"] = s_len[state["row_seq"]] + state["row_tok"]
    if case["kind"] == "chunk":
        state["k_new"] = k[state["row_seq"], :, state["row_slot"]].contiguous()
        state["v_new"] = v[state["row_seq"], :, state["row_slot"]].contiguous()
    if case["kind"] == "features":
        # Mean attention is 1 / width; the rows of the chunk's own pairs are new and hold zeros.
        f = torch.exp(torch.randn((b, hk, width, 6 * grp), generator=g, device=dev)) / width
        f = torch.where((at[None] < s_len[:, None])[:, None, :, None], f, torch.zeros_like(f))
        lse = torch.empty((total, hk * grp), device=dev)
        seen = _seen(state, torch.arange(b, device=dev), width)
        for h in range(hk * grp):
            s = _pad(state, state["q"][:, h].float()) @ k[:, h // grp].float().transpose(1, 2) * dim ** -0.5
            s = torch.where(seen, s, torch.full_like(s, -math.inf)).logsumexp(2)
            lse[:, h] = s[state["row_seq"], state["row_tok"]]
        state["lse"] = lse
        del seen
    if own:
        from paper_2602_03203_b200 import binding
        cache = binding.Cache(1, hk, grp, dim, b, 16, width)
        whole = case["kind"] != "chunk"   # the chunk operator stores the new pairs itself
        for s in range(b):
            m = stored[s] + (fresh[s] if whole else 0)
            if m:
                cache.prefill(0, s, k[s, :, :m].contiguous(), v[s, :, :m].contiguous(),
                              f[s, :, :m].contiguous() if case["kind"] == "features" else None, pos[s, :m].contiguous())
        state["cache"] = cache
    else:
        state["k"], state["v"] = k, v
        if case["kind"] == "features":
            state["f"] = f
    return state


def _pad(state, rows):
    """Packed rows [total][...] as [sequence][token][...], zeros behind the last token of a sequence."""
    t = 1 if state["case"]["kind"] == "window" else max(state["lens"])
    out = rows.new_zeros((state["case"]["seqs"], t) + rows.shape[1:])
    out[state["row_seq"], state["row_tok"]] = rows
    return out


def _seen(state, seqs, width):
    """[sequence][token][slot]: the pairs that the query of a token sees."""
    c, pos = state["case"], state["pos"][seqs].long()
    own_slot = _pad(state, state["row_slot"][:, None])[seqs]
    at = torch.arange(width, device=pos.device)
    seen = at <= own_slot
    if c["window"]:
        p = pos.gather(1, own_slot[:, :, 0])[:, :, None]
        seen = seen & ((p - pos[:, None] < c["window"]) | (pos[:, None] < c["sinks"]))
    return seen


def _attend(state, k, v):
    """Softmax attention of the packed queries over the padded cache, in 32 bits: out and log-sum-exp, packed."""
    c = state["case"]
    b, hk, grp, dim = c["seqs"], c["kv_heads"], c["group"], c["dim"]
    q = _pad(state, state["q"].float())
    t, width = q.shape[1], k.shape[2]
    q = q.reshape(b, t, hk, grp, dim).permute(0, 2, 3, 1, 4).reshape(b, hk, grp * t, dim)
    s = (q @ k.float().transpose(2, 3)).mul_(dim ** -0.5).reshape(b, hk, grp, t, width)
    s.masked_fill_(~_seen(state, torch.arange(b, device=q.device), width)[:, None, None], -math.inf)
    m = s.amax(4, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    total = p.sum(4, keepdim=True)
    o = (p.reshape(b, hk, grp * t, width) @ v.float()).reshape(b, hk, grp, t, dim)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (m + total.log())[..., 0]
    o = o.permute(0, 3, 1, 2, 4).reshape(b, t, hk * grp, dim)[state["row_seq"], state["row_tok"]]
    lse = lse.permute(0, 3, 1, 2).reshape(b, t, hk * grp)[state["row_seq"], state["row_tok"]]
    return o.to(torch.bfloat16), lse


def _features(state, k, f):
    """The feature rows after the chunk, in 32 bits and in place, of the sequences that have new tokens."""
    c = state["case"]
    b, hk, grp, dim = c["seqs"], c["kv_heads"], c["group"], c["dim"]
    q, lse = _pad(state, state["q"].float()), _pad(state, state["lse"])
    t, width = q.shape[1], k.shape[2]
    q = q.reshape(b, t, hk, grp, dim).permute(0, 2, 3, 1, 4).reshape(b, hk, grp * t, dim)
    p = (q @ k.float().transpose(2, 3)).mul_(dim ** -0.5).reshape(b, hk, grp, t, width)
    p.sub_(lse.reshape(b, t, hk, grp).permute(0, 2, 3, 1)[..., None]).exp_()
    age = (state["fresh"][:, None] - 1 - torch.arange(t, device=q.device))[:, :, None]
    seen = _seen(state, torch.arange(b, device=q.device), width) & (age >= 0)
    p.masked_fill_(~seen[:, None, None], 0.0)
    f = f.reshape(b, hk, width, grp, 6)
    active = (state["fresh"] > 0)[:, None, None, None]
    for i, w in enumerate(WINDOWS):
        mean = torch.where((age < w)[:, None, None], p, torch.zeros_like(p)).sum(3).transpose(2, 3) / w
        f[..., i] = torch.where(active, mean, f[..., i])
    mean = p.sum(3).transpose(2, 3) / state["fresh"].clamp(min=1)[:, None, None, None]
    f[..., 3] = torch.where(active, mean, f[..., 3])
    f[..., 4] = torch.where(active, f[..., 4] + mean, f[..., 4])
    f[..., 5] = torch.where(active, DECAY * f[..., 5] + mean, f[..., 5])
    return f.reshape(b, hk, width, 6 * grp)


def run(state):
    c = state["case"]
    if own:
        cache = state["cache"]
        if c["kind"] == "chunk":
            # keep_lens: the pairs that stay; a pass after another one drops the chunk that the one before stored,
            # as a decoder does whose drafts were rejected.
            lse = torch.empty(state["q"].shape[:2], device="cuda")
            out = cache.append_chunk_attn(0, state["k_new"], state["v_new"], state["q"], state["lens"],
                                          keep_lens=state["keep"], window=c["window"], sinks=c["sinks"], lse=lse)
            return [out, lse]
        if c["kind"] == "window":
            return cache.decode_attn_window(0, state["q"], c["window"], sinks=c["sinks"])
        cache.chunk_features(0, state["q"], state["lse"], state["lens"], window=c["window"], sinks=c["sinks"])
        return [cache.export_features(0, s) for s in range(c["seqs"])]
    if c["kind"] == "chunk":
        state["k"][state["row_seq"], :, state["row_slot"]] = state["k_new"]
        state["v"][state["row_seq"], :, state["row_slot"]] = state["v_new"]
        return list(_attend(state, state["k"], state["v"]))
    if c["kind"] == "window":
        return _attend(state, state["k"], state["v"])[0]
    f = _features(state, state["k"], state["f"])
    return [x[:, : n + t] for x, n, t in zip(f, state["keep"], state["lens"])]


def work(case):
    hk, grp, dim, w, kind = case["kv_heads"], case["group"], case["dim"], case["window"], case["kind"]
    hq = hk * grp
    nbytes = flops = 0
    for n, t in zip(*_lengths(case)):
        rows = 1 if kind == "window" else t
        if not rows:
            if kind == "features":   # its rows come back as they are
                nbytes += 2 * hk * n * 6 * grp * 4
            continue
        # Visible pairs by slots; a window of positions holds 1 / gap of them in the pruned part.
        inside = max(1, w // case["gap"]) if w else 0
        first = n if kind == "window" else n + 1   # pairs up to the first query's own
        ends = range(first, first + rows)
        if w:
            scores = sum(min(e, inside + min(case["sinks"], max(0, e - inside))) for e in ends)
            keys = min(ends[-1], inside + rows - 1 + min(case["sinks"], max(0, first - inside)))
        else:
            scores, keys = rows * (ends[0] + ends[-1]) // 2, ends[-1]
        if kind == "features":
            nbytes += hk * keys * dim * 2 + rows * hq * (dim * 2 + 4) + 2 * hk * (n + t) * 6 * grp * 4
            flops += 2 * hq * scores * dim
        else:
            nbytes += hk * keys * dim * 4 + 2 * rows * hq * dim * 2
            flops += 4 * hq * scores * dim
            if kind == "chunk":
                nbytes += rows * (hk * dim * 4 + hq * 4)   # the new rows are read once more to be stored; log-sum-exp
    return {"bytes": nbytes, "flops": flops}


def exact(case, seed):
    """The operators' definitions, one sequence and KV head after another, in 64 bits."""
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    hk, grp, dim, w = case["kv_heads"], case["group"], case["dim"], case["window"]
    kind = case["kind"]
    stored, fresh = _lengths(case)
    outs, lses, feats, row = [], [], [], 0
    for s in range(case["seqs"]):
        n, t = stored[s], fresh[s]
        rows, m = (1, n) if kind == "window" else (t, n + t)
        first = n - 1 if kind == "window" else n
        q = st["q"][row: row + rows].double()
        row += rows
        pos = st["pos"][s, :m].double()
        own_pos = pos[first: first + rows]
        order = torch.arange(m, device="cuda")
        hidden = order[None, :] > first + torch.arange(rows, device="cuda")[:, None]
        if w:
            hidden |= (own_pos[:, None] - pos[None, :] >= w) & (pos[None, :] >= case["sinks"])
        o = torch.zeros((rows, hk * grp, dim), dtype=torch.float64, device="cuda")
        lse = torch.zeros((rows, hk * grp), dtype=torch.float64, device="cuda")
        f = st["f"][s, :, :m].double() if kind == "features" else None
        for h in range(hk * grp if rows else 0):
            keys = st["k"][s, h // grp, :m].double()
            z = torch.einsum("td,nd->tn", q[:, h], keys) / math.sqrt(dim)
            z[hidden] = -math.inf
            lse[:, h] = torch.logsumexp(z, 1)
            a = torch.exp(z - lse[:, h: h + 1])
            if kind != "features":
                o[:, h] = a @ st["v"][s, h // grp, :m].double()
                continue
            col = f[h // grp, :, 6 * (h % grp): 6 * (h % grp) + 6]
            for i, last in enumerate(WINDOWS):
                col[:, i] = a[-last:].sum(0) / last
            col[:, 3] = a.mean(0)
            col[:, 4] += col[:, 3]
            col[:, 5] = DECAY * col[:, 5] + col[:, 3]
        outs.append(o)
        lses.append(lse)
        feats.append(f)
    if kind == "features":
        return feats
    out = torch.cat(outs)
    return out if kind == "window" else [out, torch.cat(lses)]
