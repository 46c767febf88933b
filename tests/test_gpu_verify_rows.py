"""Acceptance with rows that hold what no probability is: NaN, infinities and negative numbers, in rows that count and in rows that do not."""
import numpy as np
import pytest
import torch

from test_gpu_verify import problem, run, small

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def clean(x):
    return np.maximum(np.nan_to_num(x.astype(np.float64), nan=0.0, posinf=INF, neginf=0.0), 0.0)


def verify(tokens, parents, p, q, u, us):
    """One sequence by the definition, in 64 bits: NaN and negative entries count as 0, a draft of probability NaN is rejected."""
    p, raw, q = clean(p), q, clean(q)
    cur, path, out = 0, [0], []
    while True:
        R, nxt = p[cur].copy(), -1
        for c in range(cur + 1, len(parents)):
            if parents[c] != cur or nxt >= 0:
                continue
            x = int(tokens[c])
            if not np.isnan(raw[cur][x]) and (q[cur][x] < INF and float(u[c]) * q[cur][x] < R[x]):
                nxt = c
                continue
            left = np.maximum(R - q[cur], 0.0)
            R = left / left.sum() if left.sum() > 0 else p[cur].copy()
        if nxt < 0:
            break
        cur = nxt
        path.append(cur)
        out.append(int(tokens[cur]))
    run_ = np.cumsum(R)
    if not run_[-1] > 0:
        return path, out + [-1]
    past = np.nonzero(run_ > float(us) * run_[-1])[0]
    return path, out + [int(past[0]) if len(past) else int(np.nonzero(R)[0][-1])]


def check(x):
    p, q = x["target"].float().cpu().numpy(), x["draft"].float().cpu().numpy()
    tok, u, us = x["tokens"].cpu().numpy(), x["u"].cpu().numpy(), x["us"].cpu().numpy()
    width, row, want = max(x["lens"]), 0, ([], [], [])
    for s, t in enumerate(x["trees"]):
        part = slice(row, row + len(t))
        path, given = verify(tok[part], t, p[part], q[part], u[part], us[s])
        for o, v in zip(want, (path + [-1] * (width - len(path)), len(path), given + [-1] * (width - len(given)))):
            o.append(v)
        row += len(t)
    assert run(x) == (list(want), 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_draft_rows_that_were_never_filled(dtype, bad):
    """Rows of nodes without children: the next token comes from the target's row alone."""
    for seed in range(3):
        x = problem([6, 1, 20, 33], 3001, 3, True, dtype, seed, noise=0.2)
        row = 0
        for t in x["trees"]:
            for j in range(len(t)):
                if j not in t:
                    x["draft"][row + j] = bad
            row += len(t)
        check(x)


def test_an_accepted_leaf_goes_by_the_target_alone():
    p = [[0.5, 0.5], [0.25, 0.75]]
    for bad in (NAN, INF, -INF, -1.0, 7.0):
        q = [[0.5, 0.5], [bad, bad]]
        assert small([-1, 0], [0, 1], p, q, [0, 0.5], 0.2)[:3] == ([0, 1], 2, [1, 0])
        assert small([-1, 0], [0, 1], p, q, [0, 0.5], 0.3)[:3] == ([0, 1], 2, [1, 1])
        assert small([-1], [0], p[1:], q[1:], us=0.3)[:3] == ([0], 1, [1])   # (a root alone)


def test_entries_of_the_draft_that_are_no_probabilities():
    # A negative one counts as 0: nothing is accepted that the target does not hold, and a rejection adds nothing.
    p = [[0.0, 1.0, 0.0, 0.0]] * 3
    assert small([-1, 0], [9, 0], p[:2], [[-0.5, 0.5, 0.5, 0.5]] * 2, [0, 0.5], 0.5)[:3] == ([0, -1], 1, [1, -1])
    assert small([-1, 0], [9, 1], p[:2], [[0.0, -0.5, 0.5, 0.5]] * 2, [0, 0.999], 0.5)[:3] == ([0, 1], 2, [1, 1])
    got = small([-1, 0, 0], [9, 2, 0], [[0.25, 0.5, 0.25, 0.0]] * 3, [[-8.0, 0.25, 0.75, NAN]] * 3, [0, 0.9, 0.9], 0.4)
    assert got[:3] == ([0, 2, -1], 2, [0, 1, -1])   # R behind the rejection: 0.5, 0.5, 0, 0; 0.9 * 0 < 0.5; then the target's own 0.25, 0.5, 0.25
    # An infinite one is never accepted, and its token is gone from R.
    assert small([-1, 0], [9, 0], [[0.5, 0.5]] * 2, [[INF, 0.0]] * 2, [0, 0.0], 0.1)[:3] == ([0, -1], 1, [1, -1])
    assert small([-1, 0], [9, 0], [[0.5, 0.5]] * 2, [[INF, INF]] * 2, [0, 0.5], 0.1)[:3] == ([0, -1], 1, [0, -1])   # nothing left: p itself
    # NaN: the draft is rejected, and the next token is the target's own.
    assert small([-1, 0], [0, 1], [[0.5, 0.5]] * 2, [[NAN, NAN]] * 2, us=0.6)[:3] == ([0, -1], 1, [1, -1])
    assert small([-1, 0], [0, 1], [[0.5, 0.5]] * 2, [[NAN, NAN]] * 2, us=0.4)[:3] == ([0, -1], 1, [0, -1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lens,vocab,fan", [([16, 33, 5], 257, 4), ([64, 9], 3001, 3), ([30, 30, 30], 7, 6)])
def test_entries_all_over_the_rows(dtype, lens, vocab, fan):
    for seed in range(6):
        x = problem(lens, vocab, fan, True, dtype, seed, noise=(0.3, 2.0)[seed % 2], pad=(0, 3)[seed % 2])
        g = torch.Generator(device="cuda").manual_seed(seed)
        for name, values in (("draft", (NAN, INF, -INF, -0.25)), ("target", (NAN, -INF, -0.25))):
            for v in values:
                x[name].masked_fill_(torch.rand(x[name].shape, generator=g, device="cuda") < 0.03, v)
        check(x)
