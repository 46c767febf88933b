"""Calls that the documentation allows beside the usual ones: tensors that begin anywhere they may, steps without the host's lengths."""
import pytest
import torch

import tree_ref
from test_gpu_chunk import Case
from test_gpu_tree import check, commit, extend, make_trees, packed, path_tensors
from test_gpu_verify import problem, run, want

pytestmark = pytest.mark.gpu


def shifted(t, n):
    """The same values n elements behind the beginning of an allocation."""
    flat = torch.full((t.numel() + n + 8,), 1, dtype=t.dtype, device="cuda")
    out = flat[n:n + t.numel()].view(t.shape)
    out.copy_(t)
    return out


@pytest.mark.parametrize("D,g,lens,window", [(128, 4, [16, 3], 0), (64, 3, [40, 1], 64), (128, 8, [100, 60], 0), (64, 8, [256, 200], 256)])
def test_tensors_at_the_least_alignment(D, g, lens, window):
    """k, v, q and out 16 bytes into an allocation, everything of 32 bits 4 bytes (masks 16, as they are written)."""
    for stored in ([100, 0], [37, 500]):
        c = Case(8, g, D, stored, cap=800)
        trees = make_trees(lens, near=4)
        k, v, q = (shifted(x, 8) for x in c.chunk(lens))
        masks = c.cache.tree_masks(shifted(packed(trees), 1), lens, out=shifted(torch.zeros((sum(lens), 8), dtype=torch.int32, device="cuda"), 4))
        lse, out = shifted(torch.zeros(q.shape[:2], device="cuda"), 1), shifted(torch.zeros_like(q), 8)
        c.cache.append_tree_attn(0, k, v, q, lens, masks, window=window, out=out, lse=lse)
        extend(c, k, v, trees)
        check(c, out, lse, q, trees, window)
        again, lse2 = shifted(torch.zeros_like(q), 8), shifted(torch.zeros(q.shape[:2], device="cuda"), 1)
        c.cache.tree_attn(0, q, lens, shifted(masks, 1), window=window, out=again, lse=lse2)
        check(c, again, lse2, q, trees, window)
        assert c.status() == 0
        c.check_stored()
        got = c.cache.export_chunk(0, lens)
        into = (shifted(torch.zeros_like(got[0]), 8), shifted(torch.zeros_like(got[1]), 8), shifted(torch.zeros_like(got[2]), 2), shifted(torch.zeros_like(got[3]), 1))
        c.cache.export_chunk(0, lens, into)
        for x, y in zip(got, into):
            assert torch.equal(x, y)


@pytest.mark.parametrize("sampled", [True, False])
def test_rows_of_probabilities_at_any_address(sampled):
    for dtype in (torch.float32, torch.bfloat16):
        x = problem([7, 12], 1003, 3, sampled, dtype, 5)
        for n in (1, 3):
            y = dict(x, target=shifted(x["target"], n), draft=None if x["draft"] is None else shifted(x["draft"], n), u=shifted(x["u"], n),
                     us=shifted(x["us"], n), tokens=shifted(x["tokens"], n), parents=shifted(x["parents"], n))
            assert run(y) == (want(x), 0)


def test_steps_that_never_ask_for_the_lengths():
    """Commits followed at once by the next tree: the device's lengths count, and the host learns them at the end."""
    c = Case(2, 4, 128, [30, 0, 100], cap=900)
    for step in range(8):
        lens = [9, 3, 17]
        trees = make_trees(lens, seed=step, near=4)
        k, v, q = c.chunk(lens)
        masks = c.cache.tree_masks(packed(trees), lens)
        lse = torch.empty(q.shape[:2], device="cuda")
        out = c.cache.append_tree_attn(0, k, v, q, lens, masks, lse=lse)
        extend(c, k, v, trees)
        check(c, out, lse, q, trees)
        paths = [sorted(tree_ref.path_up(t, (5 * step + 2) % len(t))) for t in trees]
        c.cache.commit_tree(lens, *path_tensors(paths, 17))
        commit(c, trees, paths)
        if step == 4:   # the host gives lengths that it knows to be there
            lens, keep = [2, 0, 5], [31, 0, 100]
            k, v, _ = c.chunk(lens)
            c.cache.append_chunk(0, k, v, lens, keep_lens=keep)
            c.extend(k, v, lens, keep=keep)
    c.cache.sync_lengths()
    assert c.status() == 0
    c.check_stored()
