"""Argument checks of the tree, verification and fork calls that need no device."""
import ctypes

import pytest
import torch

from paper_2602_03203_b200 import binding

BIG = (2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1, -2 ** 32)


def test_null_handles_are_refused():
    lib, lens = binding.lib(), (ctypes.c_int32 * 1)(1)
    assert lib.fkv_tree_masks(None, None, lens, None, None) == -1
    assert lib.fkv_append_tree(None, 0, None, None, None, None, lens, None, None) == -1
    assert lib.fkv_tree_attn(None, 0, None, lens, None, 0, 0, 0.0, None, None, None) == -1
    assert lib.fkv_append_tree_attn(None, 0, None, None, None, None, lens, None, None, 0, 0, 0.0, None, None, None) == -1
    assert lib.fkv_verify_tree(None, None, None, lens, None, 8, None, 8, 0, 8, None, None, None, None, None, 4, None) == -1
    assert lib.fkv_verify_tree_greedy(None, None, None, lens, None, None, None, None, 4, None) == -1
    assert lib.fkv_commit_tree(None, 0, lens, None, None, 4, None) == -1
    assert lib.fkv_fork(None, lens, None) == -1
    assert lib.fkv_export_chunk(None, 0, lens, None, None, None, None, None) == -1


@pytest.fixture
def cache(monkeypatch):
    """A handle that no library call has made: every call here has to end ahead of the library."""
    c = binding.Cache.__new__(binding.Cache)
    c._h, c.feat_dim = None, 12
    c.cfg = binding.FkvConfig(1, 2, 2, 64, 3, 16, 16, 0, 32, 0, 64, 0, 0)
    c.workspace = torch.empty(1, dtype=torch.uint8, device="meta")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: c.workspace.device.index)
    return c


def t(*s, dtype=torch.bfloat16, device="meta"):
    return torch.empty(s, dtype=dtype, device=device)


def ints(*s, device="meta"):
    return t(*s, dtype=torch.int32, device=device)


def floats(*s, device="meta"):
    return t(*s, dtype=torch.float32, device=device)


@pytest.mark.parametrize("big", BIG)
def test_integers_past_32_bits(cache, big):
    k, q, m, lens = t(3, 2, 64), t(3, 4, 64), ints(3, 8), [1, 2, 0]
    for call in (lambda: cache.append_tree(big, k, k, lens, m), lambda: cache.tree_attn(0, q, lens, m, window=big),
                 lambda: cache.append_tree_attn(0, k, k, q, lens, m, sinks=big), lambda: cache.commit_tree(lens, ints(3, 2), ints(3), layer=big),
                 lambda: cache.fork([0, big, 1]), lambda: cache.export_chunk(big, lens)):
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_tensors_of_other_sizes_or_devices(cache):
    k, q, m, lens = t(3, 2, 64), t(3, 4, 64), ints(3, 8), [1, 2, 0]
    p, n = ints(3, 2), ints(3)
    nodes = dict(tokens=ints(3), parents=ints(3), tree_lens=lens, target=floats(3, 9), u_accept=floats(3), u_sample=floats(3))
    greedy = dict(tokens=ints(3), parents=ints(3), tree_lens=lens, choice=ints(3))
    calls = [lambda: cache.tree_masks(ints(4), lens), lambda: cache.tree_masks(ints(3), lens, out=ints(3, 7)),
             lambda: cache.tree_masks(ints(3, device="cpu"), lens), lambda: cache.append_tree(0, k, k, lens, ints(2, 8)),
             lambda: cache.append_tree(0, k, t(3, 2, 63), lens, m), lambda: cache.tree_attn(0, q, lens, ints(3, 8, device="cpu")),
             lambda: cache.append_tree_attn(0, k, k, q, lens, m, lse=floats(3, 3)), lambda: cache.commit_tree(lens, ints(2, 2), n),
             lambda: cache.commit_tree(lens, p, ints(2)), lambda: cache.commit_tree(lens, p, ints(3, device="cpu")),
             lambda: cache.fork([0, 1]), lambda: cache.export_chunk(0, lens, (t(2, 2, 64), None, None, None)),
             lambda: cache.export_chunk(0, lens, (None, None, floats(3, 2, 11), None)),
             lambda: cache.export_chunk(0, lens, (None, None, None, ints(3, 2, device="cpu")))]
    calls += [lambda kw=kw: cache.verify_tree(**{**nodes, **kw}) for kw in (
        dict(tokens=ints(2)), dict(parents=ints(4)), dict(u_accept=floats(2)), dict(u_sample=floats(2)), dict(target=floats(2, 9)),
        dict(target=t(3, 9, dtype=torch.float16)), dict(target=floats(3)), dict(draft=floats(3, 8)), dict(draft=t(3, 9)),
        dict(target=floats(9, 3).t()), dict(tree_lens=[3, 0]), dict(out=(ints(3, 2), ints(3), ints(3, 3))),
        dict(out=(ints(2, 2), ints(3), ints(2, 2))), dict(target=floats(3, 9, device="cpu")), dict(u_sample=floats(3, device="cpu")))]
    calls += [lambda kw=kw: cache.verify_tree_greedy(**{**greedy, **kw}) for kw in (
        dict(choice=ints(2)), dict(tokens=ints(3, device="cpu")), dict(tree_lens=[1, 2, 1]))]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(str(i))


def test_tree_constants_match_the_header():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "fkv.h")).read()
    assert int(re.search(r"#define FKV_TREE_NODES (\d+)", text).group(1)) == binding.TREE_NODES == 32 * binding.TREE_WORDS
