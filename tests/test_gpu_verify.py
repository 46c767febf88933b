"""Acceptance of drafts: against the definition in 64 bits, with given uniform numbers."""
import numpy as np
import pytest
import torch

import tree_ref
from paper_2602_03203_b200 import binding

pytestmark = pytest.mark.gpu


def handle(batch):
    return binding.Cache(1, 1, 1, 64, batch, 16, 16)


def problem(lens, vocab, fan, sampled, dtype, seed, near=1000, noise=0.7, pad=0):
    """Trees whose drafts come from q, and a target that agrees with it up to noise.  pad: unused elements behind every row."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    trees = [tree_ref.tree(t, fan, seed + s, near) for s, t in enumerate(lens)]
    total = sum(lens)
    logits = torch.randn((total, vocab), generator=g, device="cuda") * 3
    q = logits.softmax(1)
    p = (logits + noise * torch.randn((total, vocab), generator=g, device="cuda")).softmax(1)
    tokens, row = [], 0
    for t in trees:
        for j, parent in enumerate(t):
            if parent < 0:
                tokens.append(0)
            elif sampled:
                tokens.append(int(torch.multinomial(q[row + parent], 1, generator=g)))
            else:
                rank = sum(x == parent for x in t[:j])
                tokens.append(int(q[row + parent].topk(min(fan, vocab)).indices[rank % vocab]))
        row += len(t)

    def rows(x):
        x = x.to(dtype)
        if not pad:
            return x
        wide = torch.full((total, vocab + pad), 9.0, dtype=dtype, device="cuda")   # (more than any probability)
        wide[:, :vocab] = x
        return wide[:, :vocab]

    return dict(trees=trees, lens=lens, tokens=torch.tensor(tokens, dtype=torch.int32, device="cuda"),
                parents=torch.tensor([x for t in trees for x in t], dtype=torch.int32, device="cuda"), target=rows(p),
                draft=rows(q) if sampled else None, u=torch.rand(total, generator=g, device="cuda"),
                us=torch.rand(len(lens), generator=g, device="cuda"))


def run(x, cache=None, **kw):
    cache = cache or handle(len(x["lens"]))
    got = cache.verify_tree(x["tokens"], x["parents"], x["lens"], x["target"], x["u"], x["us"], draft=x["draft"], **kw)
    status = cache.device_status()[0]
    return [t.cpu().tolist() for t in got], status


def want(x):
    p, q = x["target"].float().cpu().numpy(), None if x["draft"] is None else x["draft"].float().cpu().numpy()
    tok, u, us = x["tokens"].cpu().numpy(), x["u"].cpu().numpy(), x["us"].cpu().numpy()
    width, row, out = max(1, max(x["lens"])), 0, ([], [], [])
    for s, t in enumerate(x["trees"]):
        part = slice(row, row + len(t))
        path, given = tree_ref.verify(tok[part], t, p[part], None if q is None else q[part], u[part], us[s]) if t else ([], [])
        for o, v in zip(out, (path + [-1] * (width - len(path)), len(path), given + [-1] * (width - len(given)))):
            o.append(v)
        row += len(t)
    return list(out)


CASES = [([6], 1000, 1), ([1, 0, 16, 33], 32003, 3), ([256, 0, 100], 257, 6), ([2, 2, 2, 2, 2], 1, 2), ([12, 5], 255, 4),
         ([40, 7, 0, 0, 9], 130001, 5), ([3, 9], 256, 2), ([64, 64], 8, 8), ([20, 20], 5, 3)]


@pytest.mark.parametrize("lens,vocab,fan", CASES)
@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_paths_and_tokens(lens, vocab, fan, sampled, dtype):
    for seed in range(3):
        x = problem(lens, vocab, fan, sampled, dtype, seed, near=(1000, 3, 1)[seed], noise=(0.7, 0.05, 3.0)[seed], pad=(0, 3, 8)[seed])
        got, status = run(x)
        assert got == want(x) and status == 0


def test_batches_of_every_cluster_size():
    for batch in (1, 18, 19, 37, 38, 74, 75, 148, 149, 256):
        lens = [(s * 7) % 5 for s in range(batch)]
        x = problem(lens, 3001, 2, True, torch.float32, batch)
        got, status = run(x)
        assert got == want(x) and status == 0
        if batch == 18:   # the same rows alone
            rows = [sum(lens[:s]) for s in range(batch + 1)]
            for s in (3, 11):
                part = slice(rows[s], rows[s + 1])
                one = dict(x, trees=[x["trees"][s]], lens=[lens[s]], us=x["us"][s:s + 1],
                           **{k: x[k][part] for k in ("tokens", "parents", "target", "draft", "u")})
                alone, _ = run(one)
                n = got[1][s]
                assert alone[1] == [n] and alone[0][0][:n] == got[0][s][:n] and alone[2][0][:n] == got[2][s][:n]


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("vocab", [300, 40000])
def test_as_many_siblings_as_a_tree_holds(sampled, vocab):
    """255 children of one node, most of them rejected; many tokens come twice or more in the small vocabulary."""
    for seed in range(4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x = problem([256, 256], vocab, 255, sampled, torch.float32, seed, noise=6.0)
        x["trees"] = [[-1] + [0] * 255, [-1] + [0] * 200 + [200] * 55]
        x["parents"] = torch.tensor([p for t in x["trees"] for p in t], dtype=torch.int32, device="cuda")
        x["tokens"] = torch.randint(0, vocab, (512,), generator=g, device="cuda", dtype=torch.int32)
        if seed == 0:
            x["u"] = torch.full_like(x["u"], 0.9999)
        got, status = run(x)
        assert got == want(x) and status == 0


def small(parents, tokens, p, q=None, u=None, us=0.5, **kw):
    """One sequence from lists."""
    t = len(parents)
    f = lambda a: torch.tensor(a, dtype=torch.float32, device="cuda")  # noqa: E731
    i = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    x = dict(trees=[parents], lens=[t], tokens=i(tokens), parents=i(parents), target=f(p), draft=None if q is None else f(q),
             u=f(u or [0.5] * t), us=f([us]))
    got, status = run(x, **kw)
    return got[0][0], got[1][0], got[2][0], status


def test_equality_is_a_rejection_and_zero_is_accepted():
    p, q = [[0.5, 0.5]] * 2, [[1.0, 0.0]] * 2
    assert small([-1, 0], [0, 0], p, q, [0, 0.5])[:3] == ([0, -1], 1, [1, -1])           # u q = p
    assert small([-1, 0], [0, 0], p, q, [0, np.nextafter(np.float32(0.5), np.float32(0)).item()], 0.75)[:3] == ([0, 1], 2, [0, 1])
    assert small([-1, 0], [0, 0], p, q, [0, 0.0], 0.0)[:3] == ([0, 1], 2, [0, 0])
    assert small([-1, 0], [0, 0], [[0.0, 1.0]] * 2, q, [0, 0.0])[:3] == ([0, -1], 1, [1, -1])   # 0 < 0 is no acceptance


def test_running_sums_pick_the_first_token_past_the_number():
    p = [[0.25, 0.0, 0.25, 0.5]]
    for us, x in ((0.0, 0), (0.2499, 0), (0.25, 2), (0.49, 2), (0.5, 3), (0.999999, 3)):
        assert small([-1], [0], p, us=us)[2] == [x]


def test_a_rejection_takes_the_draft_probabilities_away():
    # p - q leaves token 2 alone after the first rejection; the second sibling holds it.
    p, q = [[0.25, 0.25, 0.5, 0.0]] * 4, [[0.5, 0.25, 0.25, 0.0]] * 4
    assert small([-1, 0, 0, 0], [0, 0, 1, 2], p, q, [0, 0.75, 0.1, 0.99])[:3] == ([0, 3, -1, -1], 2, [2, 2, -1, -1])
    got = small([-1, 0, 0], [0, 0, 0], p[:3], q[:3], [0, 0.9, 0.0], 0.7)
    assert got[:3] == ([0, -1, -1], 1, [2, -1, -1])


def test_point_masses_leave_the_other_tokens():
    p = [[0.5, 0.25, 0.25]] * 4
    # 0.6 >= 0.5: rejected; 0.4 * 0.5 < 0.25: accepted.
    assert small([-1, 0, 0], [0, 0, 2], p[:3], None, [0, 0.6, 0.4], 0.1)[:3] == ([0, 2, -1], 2, [2, 0, -1])
    # All three tried: a token a second time has nothing left; token 1 is what remains.
    assert small([-1, 0, 0, 0], [0, 0, 0, 2], p, None, [0, 0.6, 0.0, 0.9], 0.99)[:3] == ([0, -1, -1, -1], 1, [1, -1, -1, -1])


def test_rows_that_are_equal_or_empty():
    same = [[0.5, 0.5]] * 2
    assert small([-1, 0], [0, 1], same, same, [0, 0.999], 0.2)[:3] == ([0, 1], 2, [1, 0])
    # A rejection that leaves nothing (here q is more than p everywhere): p itself serves.
    assert small([-1, 0], [0, 0], [[0.25, 0.5]] * 2, [[0.5, 0.5]] * 2, [0, 0.9], 0.1)[:3] == ([0, -1], 1, [0, -1])
    assert small([-1, 0], [0, 0], [[0.25, 0.5]] * 2, [[0.5, 0.5]] * 2, [0, 0.9], 0.9)[:3] == ([0, -1], 1, [1, -1])
    assert small([-1, 0], [0, 0], [[0.0, 0.0]] * 2, None)[:3] == ([0, -1], 1, [-1, -1])
    assert small([-1, 0], [0, 0], [[0.0, 0.0]] * 2, [[0.5, 0.5]] * 2)[:3] == ([0, -1], 1, [-1, -1])


def test_numbers_that_are_no_probabilities():
    nan = float("nan")
    assert small([-1, 0], [0, 0], [[nan, 0.5, nan]] * 2, [[0.5, 0.25, 0.25]] * 2)[:3] == ([0, -1], 1, [1, -1])
    assert small([-1, 0], [0, 0], [[nan, -1.0, 0.5]] * 2, None)[:3] == ([0, -1], 1, [2, -1])
    assert small([-1, 0], [0, 1], [[0.5, 0.5]] * 2, [[nan, nan]] * 2, us=0.6)[:2] == ([0, -1], 1)


def test_bad_tokens_and_parents():
    p, q = [[0.25, 0.75]] * 4, [[0.25, 0.75]] * 4
    for bad in (-1, 2, 2 ** 30):
        path, n, out, status = small([-1, 0, 0, 1], [7, bad, 1, 0], p, q, [0, 0.1, 0.1, 0.1], 0.5)
        assert (path, n, out, status) == ([0, 2, -1, -1], 2, [1, 1, -1, -1], 0)
    for bad in (1, 3, -2, 2 ** 20):
        path, n, out, status = small([-1, bad, 0, 1], [0, 0, 1, 0], p, q, [0, 0.1, 0.1, 0.1], 0.5)
        assert (path, n, status) == ([0, 2, -1, -1], 2, binding.DEV_BAD_INDEX)
    # A second root is no child of the first.
    assert small([-1, -1, 0], [0, 0, 1], p[:3], q[:3], [0, 0.1, 0.1], 0.1)[:2] == ([0, 2, -1], 2)


def test_the_tokens_follow_the_targets_distribution():
    """20000 sequences of one tree each over four tokens: frequencies of the first token within five standard deviations of p."""
    g = torch.Generator(device="cuda").manual_seed(5)
    batch, runs, n = 250, 80, 4
    cache = handle(batch)
    p = torch.tensor([0.1, 0.2, 0.3, 0.4], device="cuda")
    q = torch.tensor([0.4, 0.3, 0.2, 0.1], device="cuda")
    parents = torch.tensor([-1, 0, 0, 0] * batch, dtype=torch.int32, device="cuda")
    for sampled in (True, False):
        count = torch.zeros(4, device="cuda")
        for _ in range(runs):
            tokens = (torch.multinomial(q, n * batch, replacement=True, generator=g) if sampled else
                      torch.tensor([0, 3, 1, 3] * batch, device="cuda")).to(torch.int32)
            _, _, out = cache.verify_tree(tokens, parents, [n] * batch, p.repeat(n * batch, 1).contiguous(), torch.rand(n * batch, generator=g, device="cuda"),
                                          torch.rand(batch, generator=g, device="cuda"), draft=q.repeat(n * batch, 1).contiguous() if sampled else None)
            count += torch.bincount(out[:, 0], minlength=4)
        total = batch * runs
        dev = (count - total * p).abs() / (total * p * (1 - p)).sqrt()
        assert float(dev.max()) < 5, (sampled, dev.tolist())


def test_greedy():
    gen = torch.Generator().manual_seed(2)
    lens = [1, 0, 16, 256, 33, 5]
    for vocab, fan in ((2, 3), (4, 6), (1000, 2)):
        trees = [tree_ref.tree(t, fan, s) for s, t in enumerate(lens)]
        tokens, choice = (torch.randint(0, vocab, (sum(lens),), generator=gen, dtype=torch.int32) for _ in range(2))
        if vocab == 1000:
            choice = tokens.roll(-1)
        cache = handle(6)
        parents = torch.tensor([x for t in trees for x in t], dtype=torch.int32)
        out = tuple(torch.full(s, 9, dtype=torch.int32, device="cuda") for s in ((6, 260), (6,), (6, 260)))
        got = cache.verify_tree_greedy(tokens.cuda(), parents.cuda(), lens, choice.cuda(), out=out)
        row = 0
        for s, t in enumerate(trees):
            part = slice(row, row + len(t))
            path, given = tree_ref.greedy(tokens[part].tolist(), t, choice[part].tolist()) if t else ([], [])
            assert got[1][s] == len(path)
            assert got[0][s].tolist() == path + [-1] * (260 - len(path)) and got[2][s].tolist() == given + [-1] * (260 - len(given))
            row += len(t)
        assert cache.device_status()[0] == 0


def test_refusals():
    x = problem([5, 3], 100, 2, True, torch.float32, 1)
    cache = handle(2)
    call = lambda **kw: run(dict(x, **kw), cache)  # noqa: E731
    assert call()[1] == 0
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    bad = [dict(tokens=x["tokens"][:-1]), dict(tokens=x["tokens"].long()), dict(parents=x["parents"].cpu()), dict(u=x["u"].double()),
           dict(us=x["us"][:1]), dict(target=x["target"][:-1]), dict(target=x["target"].half()), dict(draft=x["draft"].bfloat16()),
           dict(draft=x["draft"][:, :-1]), dict(target=x["target"].t().contiguous().t()), dict(lens=[5, 3, 0]), dict(lens=[6, 3]),
           dict(lens=[2 ** 32 + 5, 3])]
    for kw in bad:
        with pytest.raises((ValueError, binding.FkvError)):
            call(**kw)
    for out in ((i32(2, 4), i32(2), i32(2, 4)), (i32(2, 5), i32(2), i32(2, 6)), (i32(1, 5), i32(2), i32(1, 5)), (i32(2, 5), i32(3), i32(2, 5))):
        with pytest.raises((ValueError, binding.FkvError)):
            run(x, cache, out=out)
    wide = torch.zeros((8, 2 ** 20 + 1), device="cuda")
    with pytest.raises(binding.FkvError):
        call(target=wide, draft=None)
    n = 257
    with pytest.raises((ValueError, binding.FkvError)):
        cache.verify_tree(i32(n), i32(n), [n, 0], torch.zeros((n, 4), device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(2, device="cuda"))
    assert cache.device_status()[0] == 0


def test_the_largest_vocabulary_and_far_rows():
    """Rows past 4 GB: 64-bit offsets."""
    v, t = 2 ** 20, 600
    cache = handle(3)
    target = torch.zeros((t * 2, v), device="cuda")   # 5 GB, every other row used
    target[:, 1] = 1.0
    target[598 * 2, 1] = 0.0
    target[598 * 2, v - 1] = 0.5
    parents = torch.tensor([-1] + [0] * 199 + [-1] + [0] * 199 + [-1] + list(range(199)), dtype=torch.int32, device="cuda")
    tokens = torch.ones(600, dtype=torch.int32, device="cuda")
    tokens[599] = 5
    got = cache.verify_tree(tokens, parents, [200, 200, 200], target[::2], torch.full((600,), 0.5, device="cuda"), torch.full((3,), 0.9, device="cuda"))
    assert got[1].tolist() == [2, 2, 199]
    assert got[2][2].tolist()[:200] == [1] * 198 + [v - 1] + [-1] and got[0][0].tolist()[:3] == [0, 1, -1]
