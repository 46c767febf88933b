"""Roll-backs of chunks in captured graphs."""
import pytest
import torch

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
