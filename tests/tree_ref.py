"""Plain implementations of the draft-tree operators: trees, masks, acceptance in 64 bits, forks."""
import random

import numpy as np


def tree(t, fan, seed, near=1000):
    """Parents of t nodes, parents first, at most `fan` children to a node, the parent among the last `near` that have room."""
    rng = random.Random(seed)
    parents, children = [], []
    for j in range(t):
        free = [i for i in range(j) if children[i] < fan][-near:]
        parents.append(rng.choice(free) if j else -1)
        if j:
            children[parents[j]] += 1
        children.append(0)
    return parents


def path_up(parents, j):
    while j >= 0:
        yield j
        j = parents[j]


def depth(parents, j):
    return len(list(path_up(parents, j))) - 1


def mask_words(parents):
    """[nodes][8] int64: the bits of every node's ancestors and itself."""
    m = np.zeros((len(parents), 8), dtype=np.int64)
    for j in range(len(parents)):
        for i in path_up(parents, j):
            m[j, i // 32] |= 1 << (i % 32)
    return m


def verify(tokens, parents, p, q, u, us):
    """One sequence: accepted nodes and given tokens.  p, q [nodes][vocab] (q None: point masses), in 64 bits, by the definition."""
    p = np.maximum(np.nan_to_num(p.astype(np.float64), nan=0.0), 0.0)
    q = None if q is None else q.astype(np.float64)
    V = p.shape[1]
    cur, path, out = 0, [0], []
    while True:
        R, m, nxt = p[cur].copy(), 1.0, -1
        for c in range(len(parents)):
            if parents[c] != cur or c <= cur or nxt >= 0:
                continue
            x = int(tokens[c])
            if not 0 <= x < V:
                continue
            if q is None:
                if float(u[c]) * m < R[x]:
                    nxt = c
                else:
                    m -= R[x]
                    R[x] = 0.0
            elif float(u[c]) * q[cur][x] < R[x]:
                nxt = c
            else:
                left = np.maximum(R - q[cur], 0.0)
                R = left / left.sum() if left.sum() > 0 else p[cur].copy()
        if nxt < 0:
            break
        cur = nxt
        path.append(cur)
        out.append(int(tokens[cur]))
    R = np.maximum(R, 0.0)
    run = np.cumsum(R)
    if not run[-1] > 0:
        return path, out + [-1]
    past = np.nonzero(run > float(us) * run[-1])[0]
    return path, out + [int(past[0]) if len(past) else int(np.nonzero(R)[0][-1])]


def greedy(tokens, parents, choice):
    cur, path, out = 0, [0], []
    while True:
        out.append(int(choice[cur]))
        nxt = [c for c in range(cur + 1, len(parents)) if parents[c] == cur and tokens[c] == choice[cur]]
        if not nxt:
            return path, out
        cur = nxt[0]
        path.append(cur)
